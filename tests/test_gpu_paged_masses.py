"""The masses that a step over paged caches adds, every row's within a bound relative to its own probability: none can be left out unseen.
(A planted mistake shows that: test_paged_rows_cpu.py.)"""
import numpy as np
import pytest
import torch

import paged_rows as rows
from paper_2407_18121_amd import binding as ec
from test_gpu_paged import MASSES, STEPS, Dev, ints, make
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu

CASES = STEPS + MASSES + [  # dtype, D, H, Hkv, G, page, max_pages, lens
    ("bf16", 64, 8, 2, 1, 16, 313, [5000, 4100]),
    ("bf16", 64, 3, 3, 3, 64, 141, [9001]),
    ("f32", 64, 4, 1, 1, 8, 376, [3001, 2999]),
    ("bf16", 128, 64, 8, 1, 32, 9, [260, -1, 7, 255] * 5),
    ("bf16", 128, 24, 3, 3, 16, 140, [2239, 2047, 64]),
    ("f32", 128, 6, 2, 2, 256, 9, [2048, 2047, 1]),
]


def inputs(case):
    dtype, D, H, Hkv, G, page, max_pages, lens = CASES[case]
    rng = np.random.default_rng(300 + case)
    pool = make(rng, dtype, len(lens), Hkv, G, D, page, max_pages, lens)
    pool.mass = np.where(rng.random(pool.mass.shape) < 0.7, pool.mass * 0.0, pool.mass)  # of most rows none yet: what is added is all there is (NaN stays)
    if case % 4 == 1 and max_pages > 1:
        pool.table[0, 1] = -1  # rows that are not there
    return (pool, dtype, lens, *(quantize(rng.standard_normal(s), dtype) for s in ((len(lens), H, D), (len(lens), Hkv, D), (len(lens), Hkv, D))), D ** -0.5)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_row_gets_its_mass(case):
    pool, dtype, lens, q, kn, vn, scale = inputs(case)
    B, H, D = q.shape
    dev = Dev(pool, dtype)
    out = torch.empty((B, H, D), device="cuda", dtype=dev.k.dtype)
    ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, B, H, pool.slots, D, ec.dtype_code(dev.k))
    print("masses", CASES[case][:7], len(lens), flush=True)
    ec.ec_paged_decode_score_step(to_dev(q, dtype), to_dev(kn, dtype), to_dev(vn, dtype), dev.k, dev.v, dev.pos, dev.mass, dev.table, ints(lens),
                                  ints([7000] * B), scale, out, ws)
    got, mass = to_host(out), to_host(dev.mass)
    want, tol, _, mass_tol = rows.step(pool, q.astype(np.float64), kn, vn, lens, [7000] * B, scale, dtype)
    assert rows.outputs_fit(got, want, tol).all()
    ok = rows.outputs_fit(mass, pool.mass, mass_tol)
    assert ok.all(), (np.argwhere(~ok)[:4], mass[~ok][:4], pool.mass[~ok][:4], mass_tol[~ok][:4])
