"""Attention of several new tokens over paged caches at the ends of the numbers' range: large scores, small weights, values that are no numbers."""
import numpy as np
import pytest
import torch

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
