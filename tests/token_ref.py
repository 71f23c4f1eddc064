"""Several new tokens of a sequence over paged caches in plain numpy, 64 bits: what the three calls are defined to do, and how far each number may be off."""
import numpy as np

U = 2.0 ** -24  # half a step of fp32, the most that one operation is off
STEP = {"bf16": 2.0 ** -8, "f32": U}  # half a step of the type


def pages(rows, page):
    return -(-rows // page)


class Planned:
    """Page tables and a stack of free pages on the host; plan() is one step, sequence by sequence, page by page."""

    def __init__(self, B, page, n_pages, max_pages, free):
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.table, self.held = np.full((B, max_pages), -1, np.int32), np.zeros(B, np.int32)
        self.stack, self.n_free = np.full(n_pages, -1, np.int32), len(free)
        self.stack[:len(free)] = free

    def plan(self, length, new, seen, T):
        """(start, len after, seen after, token_start, rows, pos)"""
        B, page = len(length), self.page
        n = [max(int(x), 0) for x in new]
        ends = np.cumsum(n)
        goal = []
        for b in range(B):
            L = int(length[b])
            fits = L >= 0 and ends[b] <= T and pages(L + n[b], page) <= self.max_pages
            goal.append(pages(L + n[b], page) if fits else None)
            while self.held[b] > (goal[b] if fits else pages(max(L, 0), page)):
                self.held[b] -= 1
                self.stack[self.n_free] = self.table[b, self.held[b]]
                self.table[b, self.held[b]] = -1
                self.n_free += 1
        start, after, seen_after, short = np.full(B, -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32), False
        for b in range(B):
            L = int(length[b])
            miss = max(goal[b] - self.held[b], 0) if goal[b] is not None else 0
            short |= miss > self.n_free
            granted = goal[b] is not None and not (miss and short)
            for _ in range(miss if granted else 0):
                self.n_free -= 1
                self.table[b, self.held[b]] = self.stack[self.n_free]
                self.held[b] += 1
            start[b] = L if granted else -1
            after[b] = -1 if L < 0 else L + n[b] if granted else L
            seen_after[b] = (0 if seen is None else int(seen[b])) + (n[b] if granted else 0)
        rows, pos = np.full(T, -1, np.int64), np.zeros(T, np.int32)
        for b in range(B):
            for i in range(n[b] if start[b] >= 0 else 0):
                t, slot = ends[b] - n[b] + i, start[b] + i
                p = int(self.table[b, slot // page])
                if 0 <= p < self.n_pages:
                    rows[t] = p * page + slot % page
                pos[t] = slot if seen is None else int(seen[b]) + i
        return start, after, seen_after, np.minimum(np.concatenate([[0], ends]), T).astype(np.int32), rows, pos


def turned(x, pos, freq, mscale, neighbours, dtype):
    """x [T,heads,D] with the positions in it, and its tolerance: the cosine and the sine are off by four steps at 1 and by the angle's own
    error (its reduction in 64 bits, the rest of an eighth of a turn rounded to fp32), mscale, two products and a sum by one each."""
    y, rot = x.astype(np.float64), 2 * len(freq)
    angle = pos.astype(np.float64)[:, None] * freq.astype(np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if neighbours else (np.arange(rot // 2), np.arange(rot // 2, rot))
    out, tol = y.copy(), np.zeros(y.shape)
    out[..., a], out[..., b] = mscale * (y[..., a] * c - y[..., b] * s), mscale * (y[..., b] * c + y[..., a] * s)
    off = abs(mscale) * (np.abs(y[..., a]) + np.abs(y[..., b])) * (8 * U + 4 * U + np.abs(angle)[:, None] * 2.0 ** -50)
    tol[..., a], tol[..., b] = off, off
    tol[..., :rot] += np.abs(out[..., :rot]) * STEP[dtype] + 1e-37
    return out, tol


def chunk(pool, q, start, token_start, scale, dtype, before_out=None):
    """(out, its tolerance, lse, its tolerance) of every token; rows of tokens of no sequence are NaN.

    Relative to a row's weight p_j, with S_j = scale * sum_d |q_d k_jd| and n rows seen:
      score      a sum of as many products as q has elements that are not 0 (`terms`), scaled, less the maximum, which is such a score itself:
                 (terms + 8) U (S_j + max S)
      weight     an exponential of 4 U; rescaled where the maximum rises and where partial results meet; the sum of the weights: n additions at
                 most, and the rescalings go with them; a division:  (n + 40) U
      weighted V fp32: n additions; bf16, up to 32 rows (tokens times query heads of a key/value head): the weight in three parts, 2 U off, 3 n
                 additions; more rows: the weight rounded to bf16, half a step off, n additions"""
    T, H, D = q.shape
    g, slots = H // pool.Hkv, pool.slots
    out, tol = np.full((T, H, D), np.nan), np.zeros((T, H, D))
    lse, lse_tol = np.full((T, H), np.nan), np.zeros((T, H))
    for b in range(len(start)):
        t0, t1, L = int(token_start[b]), int(token_start[b + 1]), int(start[b])
        n = t1 - t0
        if n <= 0:
            continue
        if not 0 <= L < slots:
            out[t0:t1], lse[t0:t1] = 0, -np.inf
            continue
        s = np.arange(min(L + n, slots))
        ids = pool.table[b, s // pool.page]
        here = (ids >= 0) & (ids < pool.n_pages)
        pp, oo, s = ids[here], s[here] % pool.page, s[here]
        parts, w_off = (1, 0.0) if dtype == "f32" else (3, 2 * U) if n * g <= 32 else (1, 2.0 ** -8)
        sees = s[None] <= (L + np.arange(n))[:, None]
        count = sees.sum(1)[:, None]
        for h in range(H):
            K, V = pool.k[pp, h // g, oo].astype(np.float64), pool.v[pp, h // g, oo].astype(np.float64)
            x = q[t0:t1, h].astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                score = np.where(sees, scale * (x @ K.T).astype(np.float32).astype(np.float64), -np.inf)  # (beyond fp32: infinite)
                S = np.where(sees & np.isfinite(score), scale * (np.abs(x) @ np.abs(K).T), 0.0)
                top = score.max(1, keepdims=True, initial=-np.inf)
                none = top == -np.inf
                w = np.exp(score - np.where(none, 0.0, top))
                total = w.sum(1, keepdims=True)
                w = w / np.where(total == 0, 1.0, total)
                lse[t0:t1, h] = np.where(none, -np.inf, top + np.log(total))[:, 0]
                rel = (((x != 0).sum(1) + 8) * U)[:, None] * (S + S.max(1, keepdims=True, initial=0)) + (count + 40) * U
                lse_tol[t0:t1, h] = rel.max(1, initial=0) + np.abs(np.where(none[:, 0], 0.0, lse[t0:t1, h])) * 8 * U + 8 * U
                wv = w * (rel + w_off + parts * (count + 1) * U)
                for lo in range(0, n, 64):  # every token by the rows that it sees: 0 times infinity is not among them
                    hi = min(lo + 64, n)
                    m = int(sees[lo:hi].any(0).sum())
                    part, finite = V[:m], np.isfinite(V[:m]).all()
                    if finite:
                        out[t0 + lo:t0 + hi, h], tol[t0 + lo:t0 + hi, h] = w[lo:hi, :m] @ part, wv[lo:hi, :m] @ np.abs(part)
                    else:
                        for i in range(lo, hi):
                            c = sees[i, :m] & (w[i, :m] > 0)
                            out[t0 + i, h], tol[t0 + i, h] = w[i, :m][c] @ part[c], wv[i, :m][c] @ np.abs(part[c])
                tol[t0:t1, h] += np.abs(out[t0:t1, h]) * STEP[dtype] + 1e-37
    return out, tol, lse, lse_tol


def fits(got, want, tol):
    """Where the definition gives an infinity or NaN the output has to have the same, everywhere else a number within the tolerance."""
    finite = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        return np.where(finite, np.abs(got - want) <= tol, (got == want) | (np.isnan(got) & np.isnan(want)))
