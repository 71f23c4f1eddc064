"""Infinite values and the precision of weights in the attention over paged caches, where rows do not fill a tile and where they do."""
import numpy as np
import pytest
import torch

import paged_rows as rows
from paper_2407_18121_amd import binding as ec
from test_gpu_paged import Dev, ints, make
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu


def run(pool, dtype, lens, q, kn, vn, scale, scored=False):
    B, H, D = q.shape
    dev = Dev(pool, dtype)
    out = torch.full((B, H, D), 3.0, device="cuda", dtype=dev.k.dtype)
    ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, B, H, pool.slots, D, ec.dtype_code(dev.k))
    args = [to_dev(x, dtype) for x in (q, kn, vn)] + [dev.k, dev.v, dev.pos]
    print("step", dtype, q.shape, pool.k.shape, list(lens)[:8], scored, flush=True)
    if scored:
        ec.ec_paged_decode_score_step(*args, dev.mass, dev.table, ints(lens), ints([7000] * B), scale, out, ws)
    else:
        ec.ec_paged_decode_step(*args, dev.table, ints(lens), ints([7000] * B), scale, out, ws)
    got = to_host(out)
    want, tol, _, _ = rows.step(pool, q.astype(np.float64), kn, vn, lens, [7000] * B, scale, dtype)
    ok = rows.outputs_fit(got, want, tol)
    assert ok.all(), (np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4], tol[~ok][:4])
    return got


def inputs(seed, dtype, B, H, Hkv, D):
    rng = np.random.default_rng(seed)
    return [quantize(rng.standard_normal(s), dtype) for s in ((B, H, D), (B, Hkv, D), (B, Hkv, D))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [0, 1, 11, 15, 16, 20, 31, 32, 40, 63, 64, 75, 200, 333])
@pytest.mark.parametrize("scored", [False, True])
def test_infinite_values_stay_infinite(dtype, D, n, scored):
    """In the new row, in the last and the first row of the cache and in one in between, +inf and -inf; both in one feature give NaN."""
    pool = make(np.random.default_rng(n), dtype, 2, 2, 1, D, 16, 22, [n, n], junk=0.0)
    q, kn, vn = inputs(n, dtype, 2, 6, 2, D)
    vn[0, 0, 3], vn[1, 1, 5] = np.inf, -np.inf
    for s, d, x in ((n - 1, 7, -np.inf), (0, 11, np.inf), (n // 2, 13, -np.inf), (0, 17, np.inf), (n // 2, 17, -np.inf)):
        if n > 2:
            p, o = pool.at(0, s)
            pool.v[p, 1, o, d] = x
    run(pool, dtype, [n, n], q, kn, vn, D ** -0.5, scored)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("below", [90, 105, 120, 140])
@pytest.mark.parametrize("n", [19, 47, 63, 100])
def test_infinite_values_beside_small_weights(dtype, D, below, n):
    """One row's weight is 2^-below of the others' and one of the infinities is its own: neither takes part in the other's product as 0 times infinity."""
    pool = make(np.random.default_rng(n), dtype, 1, 1, 1, D, 8, 16, [n], junk=0.0)
    pool.k[:] = 0
    q, kn = np.zeros((1, 3, D), np.float32), np.zeros((1, 1, D), np.float32)
    _, _, vn = inputs(n, dtype, 1, 3, 1, D)
    q[:, :, 0] = 1
    (p, o), (p2, o2) = pool.at(0, 18), pool.at(0, 17)  # in one tile
    pool.k[p, 0, o, 0] = -0.5 * below
    pool.v[p, 0, o, 2], pool.v[p, 0, o, 4] = np.inf, -np.inf   # of the small weight
    pool.v[p2, 0, o2, 3], pool.v[p2, 0, o2, 4] = -np.inf, -np.inf  # of an ordinary one
    pool.v[p2, 0, o2, 5], pool.v[p, 0, o, 5] = np.inf, -np.inf
    pool.v[p2, 0, o2, 6] = np.nan
    vn[0, 0, 8] = np.inf
    run(pool, dtype, [n], q, kn, vn, 2 * float(np.log(2)))

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3])
def test_weights_are_held_in_24_bits(D, n):
    """Sums that nearly cancel show what a weight is off by: with weights of 16 bits about a hundredth of these heads is out of bounds. q has one element that
    is not 0, so that the scores are nearly exact."""
    H, rng = 2048, np.random.default_rng(7)
    pool = make(rng, "bf16", 1, 1, 1, D, 16, 4, [n], junk=0.0)
    q, kn, vn = np.zeros((1, H, D), np.float32), np.zeros((1, 1, D), np.float32), np.zeros((1, 1, D), np.float32)
    q[0, :, 0] = quantize(rng.uniform(0.1, 1.0, H), "bf16")
    pool.k[:], pool.v[:] = 0, 0
    p, o = pool.at(0, 0)
    pool.k[p, 0, o, 0], pool.v[p, 0, o] = -1.0, 1.0
    # V of the new row: -w of the d-th head, so that its sum and its neighbours' are small
    vn[0, 0] = quantize(-np.exp(-q[0, :D, 0].astype(np.float64)), "bf16")
    run(pool, "bf16", [n], q, kn, vn, 1.0)
