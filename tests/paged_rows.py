"""What a step over paged caches computes, row by row in 64 bits, and how far each number may be off: bounds relative to the row's own probability."""
import numpy as np

import paged_ref as ref

U = 2.0 ** -24  # half a step of fp32, the most that one operation is off


def step(pool, q, kn, vn, lens, new_pos, scale, dtype):
    """(out, its tolerance, masses added [n_pages,G,page], their tolerance); new rows and masses are in the pool afterwards.

    Relative to a row's probability p_j, with S_j = scale * sum_d |q_d k_jd| and the sequence's n rows:
      score      a sum of as many products as q has elements that are not 0 (`terms`), scaled, less the maximum, which is such a score itself:
                 (terms + 8) U (S_j + max S)
      weight     an exponential of 4 U; rescaled where the maximum rises, once a tile at most, and once where partial results meet; the sum of the
                 weights: n additions at most, and the rescalings go with them; a division:  (n + 40) U
      weighted V bf16: the weight in three parts, 2^-24 + 2^-25 < 2^-23 off, 3 n additions at most;  fp32: n additions
      mass       the mean over `heads`: as many additions and a division
    A mass is added to what was there (one rounding) and an output rounded to its type (half a step)."""
    B, H, D = q.shape
    g, heads = H // pool.Hkv, H // pool.G
    parts, w_off = (3, 2 * U) if dtype == "bf16" else (1, 0.0)
    out, tol = np.zeros((B, H, D)), np.zeros((B, H, D))
    add, add_tol = np.zeros(pool.mass.shape), np.zeros(pool.mass.shape)
    for b in range(B):
        n = int(lens[b])
        if not 0 <= n < pool.slots:
            continue
        slots = np.arange(n)
        ids = pool.table[b, slots // pool.page]
        here = (ids >= 0) & (ids < pool.n_pages)
        pp, oo = ids[here], slots[here] % pool.page
        new = pool.at(b, n)
        for h in range(H):
            hk = h // g
            K = np.concatenate([pool.k[pp, hk, oo], kn[b, hk][None]]).astype(np.float64)
            V = np.concatenate([pool.v[pp, hk, oo], vn[b, hk][None]]).astype(np.float64)
            x, S = scale * (K @ q[b, h]), scale * (np.abs(K) @ np.abs(q[b, h]))
            p = np.exp(x - x.max())
            p /= p.sum()
            rel = ((q[b, h] != 0).sum() + 8) * U * (S + S.max()) + (n + 1 + 40) * U
            with np.errstate(invalid="ignore"):
                out[b, h] = p @ V
                tol[b, h] = (p * (rel + w_off + parts * (n + 1) * U)) @ np.abs(V)
            at = hk if pool.G > 1 else 0
            share = p / heads
            np.add.at(add, (pp, at, oo), share[:-1])
            np.add.at(add_tol, (pp, at, oo), (share * (rel + (heads + 2) * U))[:-1])
            if new is not None:
                add[new[0], at, new[1]] += share[-1]
                add_tol[new[0], at, new[1]] += share[-1] * (rel[-1] + (heads + 2) * U)
        if new is not None:
            pool.k[new[0], :, new[1]], pool.v[new[0], :, new[1]] = kn[b], vn[b]
            pool.mass[new[0], :, new[1]] = 0.0
            if new_pos is not None:
                pool.pos[new[0], :, new[1]] = new_pos[b]
    with np.errstate(invalid="ignore"):
        tol += np.abs(out) * (2.0 ** -8 if dtype == "bf16" else U) + 1e-37
        pool.mass = np.where(add > 0, pool.mass + add, pool.mass)  # junk of rows that are no sequence's stays
        add_tol = np.where(add > 0, add_tol + np.abs(pool.mass) * U + 1e-37, 0.0)
    return out, tol, add, add_tol


def outputs_fit(got, want, tol):
    """Where the definition gives an infinity or NaN the output has to have the same, everywhere else a number within the tolerance."""
    finite = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        return np.where(finite, np.abs(got - want) <= tol, (got == want) | (np.isnan(got) & np.isnan(want)))


__all__ = ["U", "step", "outputs_fit", "ref"]
