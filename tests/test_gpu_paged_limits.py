"""Calls on paged caches near the largest sizes that their checks let through."""
import numpy as np
import pytest
import torch

import paged_rows as rows
from paged_ref import evict
from paper_2407_18121_amd import binding as ec
from test_gpu_paged import Dev, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("max_evict", [1, 8])
def test_eviction_over_many_heads(grouped, max_evict):
    """More heads than half of what a grid holds in its second dimension."""
    rng, Hkv, D = np.random.default_rng(1), 40000, 64
    G = Hkv if grouped else 1
    N = 3
    pool = rows.ref.Pool(*(rng.integers(-9, 9, (N, Hkv, 8, D)).astype(np.float32) for _ in range(2)), rng.permutation(N * G * 8).reshape(N, G, 8).astype(np.int32),
                         rng.random((N, G, 8)).astype(np.float32), np.array([[2, 0]]))
    dev = Dev(pool, "bf16")
    ws = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, 1, G, max_evict, D, ec.EC_BF16)
    print("evict", Hkv, G, max_evict, flush=True)
    ec.ec_paged_evict_min(dev.k, dev.v, dev.pos, dev.mass, dev.table, ints([13]), ints([5]), None, max_evict, 1, 0, ws)
    torch.cuda.synchronize()
    evict(pool, [13], [5], None, max_evict, 1, 0)
    dev.check(pool)


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 20, 2 ** 29 + 96])
def test_store_out_of_very_long_sources(T):
    """More rows than workgroups of 32 of them fit into a launch; nearly all lie behind the last slot or the sequence."""
    rng, page = np.random.default_rng(2), 8
    pos = torch.empty((1, 1, T), dtype=torch.int32, device="cuda")
    pos[0, 0, :200], pos[0, 0, -30:] = torch.arange(200, device="cuda"), 77
    for start, n, first in ((0, 40, 0), (30, 100, 0), (0, None, 0), (-(T - 25), None, T - 25)):
        pos_pages = torch.full((5, 1, page), -1, dtype=torch.int32, device="cuda")
        table = ints([[4, 1, 0, 2]])
        print("store", T, start, n, flush=True)
        ec.ec_paged_store(None, None, pos, None, table, None, None, pos_pages, None, ints([start]), None if n is None else ints([n]))
        want = torch.full((5 * page,), -1, dtype=torch.int32)
        for r in range(first, min(first + 64, T if n is None else n)):  # (rows before and behind have no slot)
            s = start + r
            if 0 <= s < 32:
                want[int(table[0, s // page]) * page + s % page] = int(pos[0, 0, r])
        assert torch.equal(pos_pages.cpu().view(-1), want), (start, n)
