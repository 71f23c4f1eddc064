"""Paged caches in plain numpy, 64 bits, one row at a time: what the calls on them are defined to do."""
import numpy as np


class Pool:
    """Pools of one layer and a page table; slot s of sequence b is row s % page of page table[b, s // page]."""

    def __init__(self, k, v, pos, mass, table):
        self.k, self.v, self.pos, self.mass, self.table = k, v, pos, mass.astype(np.float64), table
        self.n_pages, self.Hkv, self.page = k.shape[:3]
        self.G = mass.shape[1]
        self.slots = table.shape[1] * self.page

    def copy(self):
        return Pool(self.k.copy(), self.v.copy(), self.pos.copy(), self.mass.copy(), self.table)

    def at(self, b, s):
        """(page, row) of a slot, or None."""
        if not 0 <= s < self.slots:
            return None
        p = int(self.table[b, s // self.page])
        return (p, s % self.page) if 0 <= p < self.n_pages else None


def store(pool, k, v, pos, mass, start, n_rows, T):
    for b in range(pool.table.shape[0]):
        for r in range(min(max(int(n_rows[b]), 0), T)):
            at = pool.at(b, int(start[b]) + r)
            if at is None:
                continue
            p, o = at
            if k is not None:
                pool.k[p, :, o], pool.v[p, :, o] = k[b, :, r], v[b, :, r]
            if pos is not None:
                pool.pos[p, :, o] = pos[b, :, r]
            if mass is not None:
                pool.mass[p, :, o] = mass[b, :, r]


def step(pool, q, kn, vn, lens, new_pos, scale, scored):
    """out [B,H,D] and what its tolerance is made of: |out| <= A = sum p |v|, and the largest sum_d |q_d k_d| of a row's score. Appends the new
    rows, and adds the masses where `scored`."""
    B, H, D = q.shape
    g = H // pool.Hkv
    out, A, big = np.zeros((B, H, D)), np.zeros((B, H, D)), np.zeros((B, H))
    for b in range(B):
        n = int(lens[b])
        if not 0 <= n < pool.slots:
            continue
        places = [pool.at(b, s) for s in range(n)]
        held = [s for s in range(n) if places[s] is not None]
        pp, oo = (np.array([places[s][i] for s in held], dtype=int) for i in (0, 1))
        total = np.zeros((pool.Hkv, len(held) + 1))
        for h in range(H):
            hk = h // g
            K = np.concatenate([pool.k[pp, hk, oo], kn[b, hk][None]]).astype(np.float64)
            V = np.concatenate([pool.v[pp, hk, oo], vn[b, hk][None]]).astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                x = scale * (K @ q[b, h])
                w = np.exp(x - x.max())
                w /= w.sum()
                out[b, h], A[b, h], big[b, h] = w @ V, w @ np.abs(V), scale * (np.abs(K) @ np.abs(q[b, h])).max()
                total[hk] += w / g
        at = pool.at(b, n)
        if at is not None:
            pool.k[at[0], :, at[1]], pool.v[at[0], :, at[1]] = kn[b], vn[b]
            if new_pos is not None:
                pool.pos[at[0], :, at[1]] = new_pos[b]
        if scored:
            add = total if pool.G == pool.Hkv else total.mean(0, keepdims=True)
            pool.mass[pp, :, oo] += add[:, :-1].T
            if at is not None:
                pool.mass[at[0], :, at[1]] = add[:, -1]
    return out, A, big


def evict(pool, lens, keep, seen, max_evict, first, recent):
    for b in range(pool.table.shape[0]):
        n = min(max(int(lens[b]), 0), pool.slots)
        gone = min(max(n - max(int(keep[b]), 0), 0), max_evict)
        places = [pool.at(b, s) for s in range(n)]
        for g in range(pool.G):
            def rank(s):
                if places[s] is None:
                    return (2, 0.0, s)
                p, o = places[s]
                at, m = int(pool.pos[p, g, o]), float(pool.mass[p, g, o])
                if (first and at < first) or (recent and at >= int(seen[b]) - recent):
                    return (2, 0.0, s)
                return (1, 0.0, s) if np.isnan(m) else (0, m + 0.0, s)
            away = set(sorted(range(n), key=rank)[:gone])
            holes = [s for s in range(n - gone) if s in away]
            movers = [s for s in range(n - gone, n) if s not in away]
            heads = [g] if pool.G > 1 else range(pool.Hkv)
            for to, come in zip(holes, movers):
                t, f = places[to], places[come]
                if t is None or f is None:
                    continue
                for h in heads:
                    pool.k[t[0], h, t[1]], pool.v[t[0], h, t[1]] = pool.k[f[0], h, f[1]], pool.v[f[0], h, f[1]]
                pool.pos[t[0], g, t[1]], pool.mass[t[0], g, t[1]] = pool.pos[f[0], g, f[1]], pool.mass[f[0], g, f[1]]


def attention_tolerance(dtype, out, A, big, n, D):
    """How far a step's output may be off, with u = 2^-24 for every fp32 operation:
      scores: a sum of D products, scaled, and its exponent's argument: (D + 8) u big, twice (the row's and the maximum's)
      weights, their sum and the weighted sum: an exponential of 4 u, sums of n terms (n + 16) u together with the rescalings
      bf16: weights as the sum of two bf16 numbers, 2^-16 relative
      the output's own rounding, half a step."""
    u = 2.0 ** -24
    rel = 2 * (D + 8) * u * big[..., None] + (n + 24) * u + (2.0 ** -16 if dtype == "bf16" else 0.0)
    return A * rel + np.abs(out) * (2.0 ** -8 if dtype == "bf16" else u) + 1e-37


def mass_tolerance(big, n, D, old):
    """Relative to a probability of at most 1: its score and normalisation as above, the mean over at most 64 heads; plus one addition to `old` (NaN in it: a new row's
    place, where nothing is added to)."""
    u = 2.0 ** -24
    return 2 * (D + 8) * u * big.max() + (n + 24 + 64) * u + np.abs(np.nan_to_num(old)) * u
