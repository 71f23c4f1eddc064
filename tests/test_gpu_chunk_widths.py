"""Attention of several new tokens over page tables that are wider than their sequences: the same bits, whatever room there is behind the last page."""
import numpy as np
import pytest
import torch

import token_ref as ref
from paper_2407_18121_amd import binding as ec
from test_gpu_chunk_pages import make
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu
WIDTHS = (8192, 65536, 1 << 26)  # slots; in the last the sums over the batch have 64 bits


def check(dtype, H, Hkv, D, L, news, page=64):
    rng = np.random.default_rng(len(L) + sum(news) + H)
    pool = make(rng, dtype, Hkv, D, page, [a + n if a >= 0 else 0 for a, n in zip(L, news)], spare=0)
    starts = np.concatenate([[0], np.cumsum(news)])
    T = int(starts[-1])
    q = quantize(rng.standard_normal((T, H, D)), dtype)
    dq, k, v = to_dev(q, dtype), to_dev(pool.k, dtype), to_dev(pool.v, dtype)
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    ws = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, len(L), H, T, D, ec.dtype_code(dq))
    got, used = [], -(-max(a + n for a, n in zip(L, news)) // page)  # pages of the longest
    for slots in (0,) + WIDTHS:
        table = torch.full((len(L), max(used, slots // page)), -1, dtype=torch.int32, device="cuda")
        table[:, :used] = i(pool.table[:, :used])
        out, lse = torch.empty_like(dq), torch.empty(T, H, device="cuda")
        ec.ec_paged_chunk_step(dq, k, v, table, i(L), i(starts), D ** -0.5, out, ws.fill_(255), lse)
        got.append((out, lse))
    want, tol, want_lse, lse_tol = ref.chunk(pool, q, L, starts, D ** -0.5, dtype)
    assert ref.fits(to_host(got[0][0]), want, tol).all() and ref.fits(to_host(got[0][1]), want_lse, lse_tol).all()
    for slots, (out, lse) in zip(WIDTHS, got[1:]):
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1]), slots


@pytest.mark.parametrize("H,Hkv,L,news", [
    (32, 32, [768], [512]),            # tiles of 64 rows, where 128 leave compute units without work
    (32, 8, [3000], [100]),
    (16, 16, [700, 33], [200, 470]),
    (32, 8, [2900], [32]),             # segments of tiles of 128 rows
    (32, 8, [2900, 40, -1, 700], [32, 1, 1, 90]),
    (40, 8, [9000], [32]),
    (32, 8, [3000], [5]),
    (32, 8, [870] * 6, [1] * 6),
    (8, 2, [2000, 10] * 40, [1] * 80),  # more sequences than lanes
    (4, 4, [300] * 70, [1] * 69 + [200]),
    (8, 8, [0, 100], [2048, 1])])
def test_128_features(H, Hkv, L, news):
    check("bf16", H, Hkv, 128, L, news)


@pytest.mark.parametrize("H,Hkv", [(32, 8), (8, 8), (32, 32)])
@pytest.mark.parametrize("rows", [200, 256, 257, 300, 400, 449, 512, 513, 900])
@pytest.mark.parametrize("n", [1, 5, 30, 60, 150])
def test_64_features(H, Hkv, rows, n):
    """Tables that just hold 257 to 512 rows are too short for a second launch: sequences of as many are not cut in wider ones either."""
    check("bf16", H, Hkv, 64, [rows - n], [n])


@pytest.mark.parametrize("D,L,news", [(128, [577, 100], [300, 7]), (64, [400], [5]), (64, [5000], [40]), (128, [0], [500]), (128, [3000, 20, 500], [1, 1, 2])])
def test_fp32(D, L, news):
    check("f32", 8, 2, D, L, news)


def test_replays_choose_anew():
    """One captured call whose lengths ask for tiles of 64 rows in one replay, of 128 in the next, and for few rows: what an eager call gives, bit for bit."""
    H, D, page, T, most = 32, 128, 64, 300, 3300
    rng = np.random.default_rng(3)
    pool = make(rng, "bf16", H, D, page, [most], spare=0)
    q = quantize(rng.standard_normal((T, H, D)), "bf16")
    dq, k, v = to_dev(q, "bf16"), to_dev(pool.k, "bf16"), to_dev(pool.v, "bf16")
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, start, starts = i(pool.table), i([0]), i([0, 0])
    size = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, T, D, ec.EC_BF16)
    out, ws = torch.zeros_like(dq), torch.full_like(size, 255)
    call = lambda out, ws: ec.ec_paged_chunk_step(dq, k, v, table, start, starts, 0.1, out, ws)  # noqa: E731
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for L, n in ((100, 300), (2900, 300), (0, 299), (3000, 20), (3000, 250), (100, 300), (700, 1)):
        start.copy_(i([L])), starts.copy_(i([0, n]))
        eager = torch.zeros_like(out)
        call(eager, torch.full_like(size, 255))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:n], eager[:n]), (L, n)
        want, tol, _, _ = ref.chunk(pool, q, [L], [0, n], 0.1, "bf16")
        assert (np.abs(to_host(out)[:n] - want[:n]) <= tol[:n]).all(), (L, n)
