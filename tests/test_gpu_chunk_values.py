"""Attention of several new tokens over paged caches at the ends of the numbers' range: large scores, small weights, values that are no numbers."""
import numpy as np
import pytest
import torch

import paged_ref
import token_ref as ref
from paper_2407_18121_amd import binding as ec
from util import quantize, to_dev, to_host, torch_dtype

pytestmark = pytest.mark.gpu


def run(k, v, q, L, dtype, scale, page=16):
    """k, v [slots,D] of one sequence and key/value head, its last len(q) rows those of the tokens; (out, lse) on the host."""
    n, H, D = q.shape
    N = -(-len(k) // page)
    pools = []
    for x in (k, v):
        x = np.concatenate([x, np.zeros((N * page - len(x), D), x.dtype)]).reshape(N, 1, page, D)
        pools.append(to_dev(x, dtype))
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse = torch.full((n, H, D), 5.5, dtype=torch_dtype(dtype), device="cuda"), torch.full((n, H), 6.5, device="cuda")
    ws = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, n, D, ec.dtype_code(out))
    ec.ec_paged_chunk_step(to_dev(q, dtype), *pools, i([list(range(N))]), i([L]), i([0, n]), scale, out, ws, lse)
    return to_host(out), to_host(lse)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,n,H", [(0, 3, 1), (100, 20, 1), (10, 100, 1), (100, 200, 2), (0, 70, 64), (3000, 150, 2)])
@pytest.mark.parametrize("score", [1.25 * 2.0 ** 14, 1.25 * 2.0 ** 24, 1.25 * 2.0 ** 34, 1.75 * 2.0 ** 36, 1.125 * 2.0 ** 60, 1.5 * 2.0 ** 125])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(dtype, D, L, n, H, score, sign):
    """One element of q and k is not 0, so that scores are exact however large: the rows of the largest one weigh the same, the others, 128 and more below, nothing. A
    sum of m numbers of V then, m additions, and a division; weights of 1 are not rounded."""
    rng = np.random.default_rng(n)
    slots = L + n
    q, k = np.zeros((n, H, D), np.float32), np.zeros((slots, D), np.float32)
    power = 2.0 ** np.floor(np.log2(score))
    half = 2.0 ** (np.log2(power) // 2)
    q[:, :, 0] = half
    k[:, 0] = sign * score / half
    k[slots // 2:, 0] += power / half * 2.0 ** -7  # the larger one
    v = quantize(rng.standard_normal((slots, D)), dtype)
    assert np.array_equal(k, quantize(k, dtype))
    out, lse = run(k, v, q, L, dtype, 1.0)
    s = k[:, 0].astype(np.float64) * half
    for i in range(n):
        top = s[:L + i + 1].max()
        rows = v[:L + i + 1][s[:L + i + 1] == top].astype(np.float64)
        want, m = rows.mean(0), len(rows)
        tol = (m + 40) * ref.U * np.abs(rows).mean(0) + np.abs(want) * ref.STEP[dtype]
        assert (np.abs(out[i] - want) <= tol).all(), (i, np.abs(out[i] - want).max())
        assert (np.abs(lse[i] - (top + np.log(m))) <= 2 * ref.U * abs(top) + (m + 40) * ref.U).all()


def definition(k, v, q, L, dtype, scale, page=16):
    """ref.chunk of one sequence and key/value head whose pages lie in order."""
    N = -(-len(k) // page)
    pages = [np.concatenate([x, np.zeros((N * page - len(x), x.shape[1]), x.dtype)]).reshape(N, 1, page, -1) for x in (k, v)]
    z = np.zeros((N, 1, page))
    pool = paged_ref.Pool(pages[0], pages[1], z.astype(np.int32), z, np.arange(N, dtype=np.int32)[None])
    return ref.chunk(pool, q, [L], [0, len(q)], scale, dtype)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,H", [(1, 1), (3, 1), (20, 1), (5, 16), (100, 1), (200, 1)])
@pytest.mark.parametrize("below", [90, 105, 115, 124])
def test_infinite_values_of_small_weights(dtype, D, n, H, below):
    """Rows of weight 2^-below of the others', one that all tokens see and one that comes with the first of them: their infinities stay infinite, beside those of
    ordinary rows too."""
    rng = np.random.default_rng(n + below)
    L = 130
    q, k = np.zeros((n, H, D), np.float32), np.zeros((L + n, D), np.float32)
    q[:, :, 0] = 1
    v = quantize(rng.standard_normal((L + n, D)), dtype)
    k[[37, L], 0] = -below
    v[37, [2, 3, 4, 5]] = np.inf, -np.inf, np.inf, np.nan
    v[L, [4, 6, 7, 8]] = -np.inf, np.inf, -np.inf, np.nan
    v[36, [9, 4]] = np.inf, np.inf
    v[L + n - 1, 10] = -np.inf
    out, lse = run(k, v, q, L, dtype, float(np.log(2)))
    want, tol, want_lse, lse_tol = definition(k, v, q, L, dtype, float(np.log(2)))
    ok = ref.fits(out, want, tol)
    assert ok.all(), (np.argwhere(~ok)[:6].tolist(), out[~ok][:6], want[~ok][:6])
    assert (np.abs(lse - want_lse) <= lse_tol).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,H", [(1, 16), (2, 16), (16, 2)])
@pytest.mark.parametrize("below", [60, 104, 118, 124])
def test_small_weights_are_held_in_24_bits(dtype, D, n, H, below):
    """Two rows of weights near 2^-below of the others', large enough in V to be all that comes out, nearly cancel in the features of a head or two: what their weights are off by shows."""
    rng = np.random.default_rng(7)
    L = 40
    q, k, v = np.zeros((n, H, D), np.float32), np.zeros((L + n, D), np.float32), np.zeros((L + n, D), np.float32)
    u = quantize(rng.uniform(0.1, 1.0, (n, H)), dtype)
    q[:, :, 0], q[:, :, 1] = 1, u
    k[[5, 30], 0], k[5, 1] = -below, -1
    v[5] = 2.0 ** 100
    w = np.resize(u, D)
    v[30] = -quantize(2.0 ** 100 * np.exp2(-w.astype(np.float64)), dtype)
    out, _ = run(k, v, q, L, dtype, float(np.log(2)))
    want, tol, _, _ = definition(k, v, q, L, dtype, float(np.log(2)))
    ok = np.abs(out - want) <= tol
    assert ok.all(), (np.argwhere(~ok)[:6].tolist(), out[~ok][:6], want[~ok][:6], tol[~ok][:6])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,n,H", [(0, 2, 1), (130, 1, 1), (130, 3, 1), (130, 20, 1), (100, 5, 16), (100, 100, 1), (130, 200, 1), (3000, 5, 2), (3000, 200, 2)])
@pytest.mark.parametrize("scores", ["2^-200", "-inf"])
def test_values_of_no_weight(dtype, D, L, n, H, scores):
    """Rows that weigh 0: what is infinite or no number in their V gives NaN to every token that sees them, 0 times infinity, whichever tile they lie in, and to no other."""
    rng = np.random.default_rng(n + L)
    slots = L + n
    q, k = np.zeros((n, H, D), np.float32), np.zeros((slots, D), np.float32)
    q[:, :, 0] = 4 if scores == "-inf" else 1
    v = quantize(rng.standard_normal((slots, D)), dtype)
    rows = sorted({r for r in (1, L // 2 + 1, L + 1, L + n // 2, slots - 2, slots - 1) if 1 <= r < slots})  # (row 0 has a weight for everybody)
    k[rows, 0] = quantize(np.float32(-2.9e38), dtype) if scores == "-inf" else -200
    scale = 1.0 if scores == "-inf" else float(np.log(2))
    want, tol, want_lse, lse_tol = definition(k, v, q, L, dtype, scale)
    for i, r in enumerate(rows):
        v[r, [3 * i, 3 * i + 1, 3 * i + 2]] = np.inf, -np.inf, np.nan
        want[[t for t in range(n) if r <= L + t], :, 3 * i:3 * i + 3] = np.nan
    out, lse = run(k, v, q, L, dtype, scale)
    ok = ref.fits(out, want, tol)
    assert ok.all(), (np.argwhere(~ok)[:6].tolist(), out[~ok][:6], want[~ok][:6])
    assert ref.fits(lse, want_lse, lse_tol).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("n,H", [(1, 1), (20, 1), (100, 1), (300, 2)])
def test_the_largest_scales(dtype, D, n, H):
    """A scale beyond the range of fp32 in units of a power of two: rows of the largest score weigh the same, all others nothing."""
    rng = np.random.default_rng(n)
    L = 300
    q, k = np.zeros((n, H, D), np.float32), np.zeros((L + n, D), np.float32)
    q[:, :, 0] = 1
    k[:, 0] = np.where(rng.random(L + n) < 0.5, 0.0, -1.0)
    v = quantize(rng.standard_normal((L + n, D)), dtype)
    out, lse = run(k, v, q, L, dtype, 3.3e38)
    for i in range(n):
        rows = v[:L + i + 1][k[:L + i + 1, 0] == 0].astype(np.float64)
        tol = (len(rows) + 40) * ref.U * np.abs(rows).mean(0) + np.abs(rows.mean(0)) * ref.STEP[dtype]
        assert (np.abs(out[i] - rows.mean(0)) <= tol).all()
        assert (np.abs(lse[i] - np.log(len(rows))) <= (len(rows) + 40) * ref.U).all()
