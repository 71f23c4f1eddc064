"""Calls on paged caches against the plain 64-bit form (paged_ref.py)."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2407_18121_amd import binding as ec
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu
I32 = torch.int32


def ints(x):
    return torch.tensor(np.asarray(x), dtype=I32, device="cuda")


def make(rng, dtype, B, Hkv, G, D, page, max_pages, lens, extra=5, junk=float("nan")):
    """A pool whose sequences hold `lens` rows (and room for one more) in pages of any order; rows that are no sequence's hold `junk`, table
    entries that are not used lie outside the pool."""
    used = [min(max(n, -1) // page + 1 if n >= 0 else 0, max_pages) for n in lens]
    N = sum(used) + extra
    order = rng.permutation(N)
    table = rng.choice([-1, -7, N, N + 3, 2 ** 31 - 1, -2 ** 31], size=(B, max_pages)).astype(np.int64)
    i = 0
    for b, u in enumerate(used):
        table[b, :u] = order[i:i + u]
        i += u
    k, v = (np.full((N, Hkv, page, D), junk, np.float32) for _ in range(2))
    pos, mass = rng.integers(0, 5000, (N, G, page)).astype(np.int32), np.full((N, G, page), junk, np.float32)
    for b, n in enumerate(lens):
        for s in range(min(max(n, 0), max_pages * page)):
            p, o = table[b, s // page], s % page
            k[p, :, o] = quantize(rng.standard_normal((Hkv, D)) * (4.0 if rng.random() < 0.05 else 0.7), dtype)
            v[p, :, o] = quantize(rng.standard_normal((Hkv, D)), dtype)
            mass[p, :, o] = rng.random(G).astype(np.float32)
    return ref.Pool(k, v, pos, mass, table)


class Dev:
    """The same on the device."""

    def __init__(self, pool, dtype):
        self.k, self.v = to_dev(pool.k, dtype), to_dev(pool.v, dtype)
        self.pos, self.mass, self.table = ints(pool.pos), torch.from_numpy(pool.mass.astype(np.float32)).cuda(), ints(pool.table)

    def check(self, pool, mass_tol=None):
        """Rows, positions and masses are the pool's, bit for bit (masses within a tolerance where that is given), junk included."""
        assert np.array_equal(to_host(self.k), pool.k, equal_nan=True)
        assert np.array_equal(to_host(self.v), pool.v, equal_nan=True)
        assert np.array_equal(self.pos.cpu().numpy(), pool.pos)
        got, want = to_host(self.mass), pool.mass.astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        with np.errstate(invalid="ignore"):
            err = np.abs(got - want)
        assert (np.isnan(want) | (got == want) | (err <= (0 if mass_tol is None else mass_tol))).all(), np.nanmax(err)


def run_step(pool, dtype, H, lens, seed, scored=False, scale=None, q=None, kn=None, vn=None, with_pos=True, more=0.0, ws=None):
    rng = np.random.default_rng(seed)
    B, D = pool.table.shape[0], pool.k.shape[3]
    scale = D ** -0.5 if scale is None else scale
    q = quantize(rng.standard_normal((B, H, D)), dtype) if q is None else q
    kn = quantize(rng.standard_normal((B, pool.Hkv, D)), dtype) if kn is None else kn
    vn = quantize(rng.standard_normal((B, pool.Hkv, D)), dtype) if vn is None else vn
    new_pos = rng.integers(5000, 6000, B)
    dev, code = Dev(pool, dtype), ec.EC_F32 if dtype == "f32" else ec.EC_BF16
    out = torch.full((B, H, D), 3.0, device="cuda", dtype=dev.k.dtype)
    fn = ec.EC_FN_PAGED_DECODE_SCORE_STEP if scored else ec.EC_FN_PAGED_DECODE_STEP
    ws = ec.new_workspace(fn, B, H, pool.slots, D, code) if ws is None else ws
    tq, tk, tv, tl, tp = to_dev(q, dtype), to_dev(kn, dtype), to_dev(vn, dtype), ints(lens), ints(new_pos)
    pos = dev.pos if with_pos else None
    print("step", dtype, q.shape, pool.k.shape, list(lens)[:8], flush=True)
    if scored:
        ec.ec_paged_decode_score_step(tq, tk, tv, dev.k, dev.v, pos, dev.mass, dev.table, tl, tp, scale, out, ws)
    else:
        ec.ec_paged_decode_step(tq, tk, tv, dev.k, dev.v, pos, dev.table, tl, tp if with_pos else None, scale, out, ws)
    torch.cuda.synchronize()
    old = pool.mass.copy()
    want, A, big = ref.step(pool, q.astype(np.float64), kn, vn, lens, new_pos if with_pos else None, scale, scored)
    n = max(max(lens), 0) + 1
    tol = ref.attention_tolerance(dtype, want, A, big, n, D) + more
    got = to_host(out)
    with np.errstate(invalid="ignore"):
        err = np.abs(got - want)
    ok = (err <= tol) | (np.isnan(want) & np.isnan(got)) | (got == want)
    assert ok.all(), (np.argwhere(~ok)[:4], err[~ok][:4], tol[~ok][:4])
    dev.check(pool, ref.mass_tolerance(big, n, D, old) if scored else None)
    return dev


STEPS = [  # dtype, D, H, Hkv, G, page, max_pages, lens
    ("bf16", 128, 4, 4, 1, 16, 3, [0, 1, 15, 16, 17, 31, 32, 33, 47]),
    ("bf16", 128, 8, 2, 2, 8, 5, [7, 8, 9, 0, -1, 39, 40, 41, 24]),
    ("bf16", 64, 6, 2, 1, 64, 6, [127, 128, 129, 383, 255, 256, 257, -5, 1]),
    ("bf16", 128, 16, 1, 1, 32, 40, [1000, 1279]),
    ("bf16", 128, 20, 1, 1, 16, 20, [300, 63]),
    ("bf16", 64, 35, 5, 5, 256, 3, [511, 512, 700]),
    ("bf16", 128, 32, 8, 8, 128, 9, [1100]),
    ("bf16", 64, 1, 1, 1, 8, 1, [0, 7, 8]),
    ("f32", 64, 4, 4, 1, 16, 7, [0, 1, 15, 16, 17, 100, 111, 112]),
    ("f32", 128, 8, 2, 2, 8, 40, [9, 311, -1, 64, 65]),
    ("f32", 128, 5, 1, 1, 32, 20, [600, 0]),
    ("f32", 64, 33, 3, 3, 64, 4, [255, 31, 128]),
    ("f32", 128, 3, 3, 1, 256, 2, [400]),
]


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_step(case, scored):
    dtype, D, H, Hkv, G, page, max_pages, lens = STEPS[case]
    rng = np.random.default_rng(100 + case)
    pool = make(rng, dtype, len(lens), Hkv, G, D, page, max_pages, lens)
    run_step(pool, dtype, H, lens, case, scored, with_pos=case % 3 != 1 or scored)


@pytest.mark.parametrize("dtype,H,Hkv,B,n,page", [("bf16", 8, 2, 2, 5000, 16), ("bf16", 3, 3, 1, 9001, 64), ("f32", 4, 1, 1, 3001, 8),
                                                  ("bf16", 40, 40, 12, 150, 16), ("bf16", 64, 8, 33, 260, 32), ("f32", 16, 16, 20, 90, 16)])
@pytest.mark.parametrize("scored", [False, True])
def test_step_long_or_many(dtype, H, Hkv, B, n, page, scored):
    rng = np.random.default_rng(n)
    lens = [n] + [int(x) for x in rng.integers(-1, n + 1, B - 1)]
    pool = make(rng, dtype, B, Hkv, 1, 64 if n > 1000 else 128, page, -(-(n + 1) // page), lens)
    run_step(pool, dtype, H, lens, n, scored)


MASSES = [  # dtype, D, H, Hkv, G, page, max_pages, lens: groups of few and of many scores, of one pair and of several, cut and whole
    ("bf16", 128, 8, 2, 1, 16, 31, [400, -1, 495, 0]),      # two pairs a group
    ("bf16", 128, 20, 1, 1, 16, 12, [150, 191, 3]),         # two pairs of one key head
    ("bf16", 64, 68, 2, 2, 8, 14, [111, 30]),               # three pairs of a key head each
    ("bf16", 64, 51, 1, 1, 8, 9, [71, 2, 60]),              # four pairs
    ("bf16", 64, 65, 1, 1, 8, 7, [55, 17]),                 # five pairs
    ("bf16", 128, 4, 4, 4, 8, 256, [2047, 1500]),           # as many slots as one launch takes, one head a group
    ("bf16", 128, 4, 4, 4, 8, 257, [2055, 1500]),           # and a page more
    ("bf16", 128, 2, 1, 1, 32, 64, [2040]),                 # as many scores
    ("bf16", 64, 5, 1, 1, 32, 26, [831, 500]),              # and some more
    ("f32", 64, 9, 3, 1, 8, 40, [310, 311, 319, 255, 256]),
    ("f32", 128, 7, 1, 1, 64, 9, [500, 64, 63]),
    ("f32", 64, 512, 1, 1, 8, 1, [7, 6, 0, -1]),            # as many heads
    ("f32", 128, 3, 3, 3, 16, 20, [300] * 200),             # more groups than tickets, one pair each
    ("bf16", 64, 2, 2, 1, 8, 5, [33] * 520),                # and of two pairs
]


@pytest.mark.parametrize("case", range(len(MASSES)))
def test_masses(case):
    dtype, D, H, Hkv, G, page, max_pages, lens = MASSES[case]
    pool = make(np.random.default_rng(900 + case), dtype, len(lens), Hkv, G, D, page, max_pages, lens)
    if case % 2:
        pool.table[0, 1 if max_pages > 1 else 0] = -1  # rows that are not there
    run_step(pool, dtype, H, lens, case, True)


def test_one_workspace_for_calls_of_different_sizes():
    """What a call leaves in a workspace is what any other finds right, whichever way the masses are added up."""
    ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, 70, 64, 6000, 128, ec.EC_F32)
    for i, (dtype, D, H, Hkv, G, page, lens) in enumerate([("bf16", 128, 8, 2, 1, 16, [400, 300, 0]), ("bf16", 128, 8, 2, 1, 16, [5000, 300]),
                                                           ("f32", 64, 3, 3, 1, 8, [500] * 5), ("bf16", 64, 40, 4, 4, 32, [200] * 60),
                                                           ("bf16", 128, 8, 2, 1, 16, [400, 300, 0]), ("f32", 128, 64, 1, 1, 8, [50, 60])]):
        for scored in (True, False, True):
            run_step(quick(np.random.default_rng(i), dtype, Hkv, G, D, page, lens), dtype, H, lens, i, scored, ws=ws)


def quick(rng, dtype, Hkv, G, D, page, lens):
    """A pool of normal numbers all over: long sequences are made quickly."""
    used = [max(n, 0) // page + 1 for n in lens]
    N = sum(used)
    order, table, at = rng.permutation(N), np.full((len(lens), max(used)), -1, np.int64), 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    k, v = (quantize(rng.standard_normal((N, Hkv, page, D), np.float32), dtype) for _ in range(2))
    return ref.Pool(k, v, rng.integers(0, 5000, (N, G, page)).astype(np.int32), rng.random((N, G, page)).astype(np.float32), table)


@pytest.mark.parametrize("dtype,H,Hkv,D,page,B,n", [("bf16", 4, 2, 128, 16, 24, 4200), ("bf16", 2, 2, 64, 64, 30, 6000), ("f32", 4, 4, 64, 32, 40, 700),
                                                    ("bf16", 3, 1, 128, 8, 64, 3900), ("bf16", 2, 1, 128, 256, 63, 5000), ("bf16", 1, 1, 64, 16, 70, 2000), ("f32", 1, 1, 64, 8, 700, 40),
                                                    ("bf16", 1, 1, 64, 8, 1100, 60), ("bf16", 4, 2, 128, 16, 2, 640), ("f32", 8, 2, 64, 8, 3, 1100),
                                                    ("bf16", 2, 1, 128, 16, 70, 400)])
@pytest.mark.parametrize("spread", ["alike", "mixed", "one long"])
def test_batches_whose_sequences_are_cut(dtype, H, Hkv, D, page, B, n, spread):
    """Every rule by which a batch is divided over workgroups: no row is left out or counted twice."""
    rng = np.random.default_rng(B + n)
    lens = [n] * B if spread == "alike" else [int(x) for x in rng.integers(-1, n + 1, B)] if spread == "mixed" else [n * 3] + [int(x) for x in rng.integers(0, 200, B - 1)]
    pool = quick(rng, dtype, Hkv, 1, D, page, lens)
    run_step(pool, dtype, H, lens, n, with_pos=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scored", [False, True])
def test_pages_that_do_not_exist(dtype, scored):
    """Rows on them weigh nothing, also where nothing is left but the new row, which counts even if it cannot be stored."""
    rng = np.random.default_rng(5)
    lens = [100, 64, 40, 16, 33]
    pool = make(rng, dtype, 5, 2, 2, 64, 16, 8, lens)
    pool.table[0, [0, 3]] = -1          # the first page and one in between
    pool.table[1, :4] = 10 ** 9         # all of them, the new row's not
    pool.table[2, 2] = pool.n_pages     # the last one: the new row has no place
    pool.table[3, :2] = -3              # nothing at all
    run_step(pool, dtype, 6, lens, 6, scored)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_prefix(dtype):
    """Pages that are only read may be in several sequences."""
    rng = np.random.default_rng(8)
    lens = [70, 40, 64]
    pool = make(rng, dtype, 3, 2, 1, 64, 16, 6, lens)
    pool.table[1, :2] = pool.table[0, :2]
    pool.table[2, :4] = pool.table[0, [1, 1, 0, 2]]  # one of them twice in a sequence
    run_step(pool, dtype, 4, lens, 9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["large", "minus_inf", "nan_key", "nan_value", "inf_value", "tiny_scale", "equal", "all_minus_inf", "plus_inf"])
def test_values_at_the_ends_of_the_range(dtype, what):
    rng = np.random.default_rng(12)
    lens, D = [75, 12], 64
    pool = make(rng, dtype, 2, 2, 1, D, 16, 6, lens)
    q = quantize(np.abs(rng.standard_normal((2, 4, D))) + 0.1, dtype)
    kn = quantize(rng.standard_normal((2, 2, D)), dtype)
    (p, o), scale = pool.at(0, 41), 0.125
    if what == "large":
        q *= 512.0
    elif what == "minus_inf":
        pool.k[p, 0, o, 3] = -np.inf
    elif what == "nan_key":
        pool.k[p, 1, o, 7] = np.nan
    elif what == "nan_value":
        pool.v[p, 1, o, 7] = np.nan
    elif what == "inf_value":
        pool.v[p, 0, o, 9] = np.inf
    elif what == "tiny_scale":
        scale = 1e-30
    elif what == "equal":
        q[:] = 0
    elif what == "all_minus_inf":
        for s in range(12):
            at = pool.at(1, s)
            pool.k[at[0], :, at[1], 0] = -np.inf
        kn[1, :, 0] = -np.inf
    elif what == "plus_inf":
        pool.k[p, 0, o, 3] = np.inf
    run_step(pool, dtype, 4, lens, 13, scale=scale, q=q, kn=kn)


RANGES = {  # exponents of keys and of queries, scale
    "keys below the normal range": (-130, 123, 1.0),
    "queries below the normal range": (125, -130, 0.0884),
    "queries that scaling takes below it": (124, -124, 0.0884),
    "large queries": (-128, 127, 1.0),
    "large keys": (127, -128, 1.0),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", RANGES)
def test_queries_and_keys_at_the_ends_of_the_range(dtype, what):
    """The scores are of size one; neither their products nor their sums leave the range that q * scale stays in."""
    at_k, at_q, scale = RANGES[what]
    rng = np.random.default_rng(14)
    lens, D = [40, 300], 64
    pool = make(rng, dtype, 2, 2, 1, D, 16, 20, lens, junk=0.0)
    cut = lambda x, e: quantize(np.clip(x, -1.3, 1.3) * 2.0 ** e, dtype)  # noqa: E731
    pool.k = cut(pool.k, at_k)
    run_step(pool, dtype, 4, lens, 13, scale=scale, q=cut(rng.standard_normal((2, 4, D)), at_q), kn=cut(rng.standard_normal((2, 2, D)), at_k))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("below", [60, 110, 120, 130, 140])
def test_small_weights_of_large_rows(dtype, below):
    """A weight far below the normal range counts where its V decides the output: the other rows' V are zeros. A subnormal weight is off by 2^-150 at
    most, here of four rows of 2^120 times at most 5, divided by a sum of at least 1."""
    rng = np.random.default_rng(15)
    lens, D = [50, 10], 64
    pool = make(rng, dtype, 2, 2, 1, D, 16, 6, lens, junk=0.0)
    pool.k[:], pool.v[:] = 0, 0
    q, kn = np.zeros((2, 4, D), np.float32), np.zeros((2, 2, D), np.float32)
    q[:, :, 0] = 1
    for s in range(20, 24):
        p, o = pool.at(0, s)
        pool.k[p, :, o, 0] = -below * 0.5
        pool.v[p, :, o] = quantize(rng.standard_normal((2, D)) * 2.0 ** 120, dtype)
    run_step(pool, dtype, 4, lens, 13, scale=2 * float(np.log(2)), q=q, kn=kn, vn=np.zeros((2, 2, D), np.float32), more=4 * 5 * 2.0 ** (120 - 150))


def test_rows_beyond_four_gibibytes():
    """Pages whose offsets pass 32 bits: the rows there are read, written and moved."""
    Hkv, page, D, lens = 8, 64, 128, [100]
    N = (5 << 30) // (Hkv * page * D * 2)
    k, v = (torch.zeros((N, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, mass = torch.zeros((N, 1, page), dtype=I32, device="cuda"), torch.zeros((N, 1, page), device="cuda")
    rng = np.random.default_rng(3)
    small = make(rng, "bf16", 1, Hkv, 1, D, page, 2, lens, extra=0, junk=0.0)
    where = [N - 1, N - 3]
    for i, p in enumerate(small.table[0]):
        k[where[i]], v[where[i]] = to_dev(small.k[p], "bf16"), to_dev(small.v[p], "bf16")
        pos[where[i]], mass[where[i]] = ints(small.pos[p]), torch.from_numpy(small.mass[p]).cuda()
    table = ints([where])
    q, kn, vn = (quantize(rng.standard_normal(s), "bf16") for s in ((1, 8, D), (1, Hkv, D), (1, Hkv, D)))
    out, ws = torch.empty((1, 8, D), dtype=torch.bfloat16, device="cuda"), ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, 1, 8, 128, D, ec.EC_BF16)
    ec.ec_paged_decode_score_step(to_dev(q, "bf16"), to_dev(kn, "bf16"), to_dev(vn, "bf16"), k, v, pos, mass, table, ints(lens), ints([7000]), 0.1,
                                  out, ws)
    want, A, big = ref.step(small, q.astype(np.float64), kn, vn, lens, [7000], 0.1, True)
    assert (np.abs(to_host(out) - want) <= ref.attention_tolerance("bf16", want, A, big, 101, D)).all()
    small.mass = mass[torch.tensor([where[list(small.table[0]).index(p)] for p in range(2)])].cpu().numpy()
    ec.ec_paged_evict_min(k, v, pos, mass, table, ints([101]), ints([60]), ints([7001]), 60, 1, 5, ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, 1, 1, 60, D, ec.EC_BF16))
    ref.evict(small, [101], [60], [7001], 60, 1, 5)
    for i, p in enumerate(small.table[0]):
        assert np.array_equal(to_host(k[where[i]]), small.k[p]) and np.array_equal(to_host(v[where[i]]), small.v[p])
        assert np.array_equal(pos[where[i]].cpu().numpy(), small.pos[p]) and np.array_equal(mass[where[i]].cpu().numpy(), small.mass[p])
    assert not k[:where[1]].any() and not k[where[1] + 1:where[0]].any()
    # 5 GiB of a dense source as well
    src = torch.zeros((1, 1, (5 << 30) // 256, D), dtype=torch.bfloat16, device="cuda")
    src[0, 0, -40:] = to_dev(quantize(rng.standard_normal((40, D)), "bf16"), "bf16")
    T = src.shape[2]
    kp, vp = (torch.zeros((T // 64, 1, 64, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ec.ec_paged_store(src, src, None, None, torch.arange(T // 64, dtype=I32, device="cuda")[None].contiguous(), kp, vp, None, None)
    assert torch.equal(kp.view(-1, D), src[0, 0]) and torch.equal(vp.view(-1, D), src[0, 0])


STORES = [  # dtype, D, Hkv, G, page, max_pages, T, src_rows, start, n
    ("bf16", 128, 3, 1, 16, 4, 40, 40, [0, 5, 24, 63], [40, 40, 40, 40]),
    ("bf16", 64, 2, 2, 8, 9, 33, 50, [1, 70, -2, 0], [33, 12, 20, 0]),
    ("f32", 128, 1, 1, 32, 3, 1, 1, [31, 95, 96, 2 ** 31 - 1], [1, 9, 1, 1]),
    ("f32", 64, 5, 5, 256, 1, 200, 201, [3, 100, 255, -2 ** 31], [200, -4, 200, 200]),
    ("bf16", 128, 8, 8, 64, 20, 1203, 1300, [0, 7, 64, 77], [1203, 1202, 1000, 5]),
]


@pytest.mark.parametrize("case", range(len(STORES)))
@pytest.mark.parametrize("parts", ["all", "rows", "pos", "mass", "pos and mass"])
def test_store(case, parts):
    dtype, D, Hkv, G, page, max_pages, T, src_rows, start, n = STORES[case]
    rng = np.random.default_rng(case)
    B = len(start)
    pool = make(rng, dtype, B, Hkv, G, D, page, max_pages, [max_pages * page - 1] * B, junk=9.0)
    pool.table[2, max_pages // 2] = -1  # a page that is not there
    dev = Dev(pool, dtype)
    k, v = (quantize(rng.standard_normal((B, Hkv, src_rows, D)), dtype) for _ in range(2))
    pos, mass = rng.integers(0, 9999, (B, G, src_rows)).astype(np.int32), rng.random((B, G, src_rows)).astype(np.float32)
    rows, has_pos, has_mass = parts in ("all", "rows"), parts in ("all", "pos", "pos and mass"), parts in ("all", "mass", "pos and mass")
    print("store", STORES[case], parts, flush=True)
    ec.ec_paged_store(to_dev(k, dtype) if rows else None, to_dev(v, dtype) if rows else None, ints(pos) if has_pos else None,
                      torch.from_numpy(mass).cuda() if has_mass else None, dev.table, dev.k if rows else None, dev.v if rows else None,
                      dev.pos if has_pos else None, dev.mass if has_mass else None, ints(start), ints(n), T)
    ref.store(pool, k if rows else None, v, pos if has_pos else None, mass if has_mass else None, start, n, T)
    dev.check(pool)


def test_store_without_lengths():
    rng = np.random.default_rng(0)
    pool = make(rng, "bf16", 2, 2, 1, 64, 8, 3, [23, 23], junk=1.0)
    dev = Dev(pool, "bf16")
    k, v = (quantize(rng.standard_normal((2, 2, 17, 64)), "bf16") for _ in range(2))
    ec.ec_paged_store(to_dev(k, "bf16"), to_dev(v, "bf16"), None, None, dev.table, dev.k, dev.v, None, None)
    ref.store(pool, k, v, None, None, [0, 0], [17, 17], 17)
    dev.check(pool)


EVICTS = [  # dtype, D, Hkv, G, page, lens, keep, max_evict, first, recent
    ("bf16", 128, 2, 1, 16, [1, 2, 30, 31, 0, 64, 65], [1, 1, 29, 31, 0, 63, 64], 1, 1, 3),
    ("bf16", 64, 2, 2, 8, [100, 37, 5, 128], [40, 36, 9, 0], 128, 1, 10),
    ("f32", 64, 3, 3, 32, [700, 512, 33], [100, 511, -4], 600, 2, 25),
    ("f32", 128, 1, 1, 64, [1500, 1024, 1025], [1024, 700, 1], 2000, 0, 0),
    ("bf16", 128, 2, 1, 16, [3000, 2049, 64], [2999, 300, 64], 2700, 1, 25),
    ("bf16", 64, 1, 1, 256, [5000], [17], 3000, 4, 100),          # the cap on what may go is reached
    ("bf16", 64, 1, 1, 8, [20, 20], [3, 10], 20, 30, 500),        # more protected than kept
    ("f32", 64, 1, 1, 256, [70001], [30000], 65000, 1, 25),
    ("bf16", 64, 1, 1, 128, [32768], [20000], 12768, 3, 50),
    ("bf16", 64, 1, 1, 64, [8193], [8000], 1000, 1, 25),
    ("bf16", 64, 1, 1, 16, [16385], [1000], 15385, 1, 25),
    ("bf16", 64, 1, 1, 256, [32769], [32700], 100, 1, 25),
    ("bf16", 128, 1, 1, 32, [40009], [40008], 1, 1, 25),
    ("bf16", 64, 2, 2, 256, [8900, 3, 0, 1, 8192], [8899, 1, 0, 1, 9000], 1, 1, 25),   # in tables of 70 pages
]


@pytest.mark.parametrize("case", range(len(EVICTS)))
@pytest.mark.parametrize("masses", ["any", "ties", "ends", "same", "nan", "close"])
def test_evict(case, masses):
    dtype, D, Hkv, G, page, lens, keep, max_evict, first, recent = EVICTS[case]
    rng = np.random.default_rng(50 + case)
    max_pages = max(-(-max(lens) // page) + 1, -(-max_evict // page), 70 if max_evict == 1 and page == 256 else 0)
    pool = make(rng, dtype, len(lens), Hkv, G, D, page, max_pages, lens, junk=4.0) if max(lens) < 9000 else None
    if pool is None:  # a long one, quicker to make
        N = max_pages
        pool = ref.Pool(*(rng.integers(-9, 9, (N, Hkv, page, D)).astype(np.float32) for _ in range(2)), np.zeros((N, G, page), np.int32),
                        rng.random((N, G, page)).astype(np.float32), rng.permutation(N)[None].astype(np.int64))
    pool.pos = rng.permutation(pool.pos.size).reshape(pool.pos.shape).astype(np.int32)
    if masses == "ties":
        pool.mass = rng.integers(0, 4, pool.mass.shape).astype(np.float32)
    elif masses == "ends":
        pool.mass = rng.choice(np.float32([0.0, -0.0, 1e-45, -1e-45, np.inf, -np.inf, np.nan, -np.nan, 3.4e38, -2.0]), pool.mass.shape)
    elif masses == "same":
        pool.mass[:] = 0.25
    elif masses == "nan":
        pool.mass = np.where(rng.random(pool.mass.shape) < 0.5, np.nan, rng.random(pool.mass.shape).astype(np.float32))
    elif masses == "close":  # differ in their last bits only
        pool.mass = np.nextafter(np.float32(1.5), np.float32(2)) + rng.integers(0, 300, pool.mass.shape).astype(np.float32) * np.float32(2.0 ** -23)
    seen = [int(np.quantile(pool.pos, 0.9))] * len(lens)
    dev = Dev(pool, dtype)
    ws = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, len(lens), G, max_evict, D, ec.dtype_code(dev.k))
    ws.fill_(255)
    print("evict", EVICTS[case], masses, flush=True)
    ec.ec_paged_evict_min(dev.k, dev.v, dev.pos, dev.mass, dev.table, ints(lens), ints(keep), ints(seen), max_evict, first, recent, ws)
    torch.cuda.synchronize()
    ref.evict(pool, lens, keep, seen, max_evict, first, recent)
    dev.check(pool)


def test_evict_on_pages_that_do_not_exist():
    """Their rows go last, and are neither moved nor written."""
    rng = np.random.default_rng(2)
    lens = [64, 64, 40]
    pool = make(rng, "bf16", 3, 2, 1, 64, 16, 5, lens, junk=4.0)
    pool.table[0, 1], pool.table[1, 3], pool.table[2, :] = -1, pool.n_pages, -5
    dev = Dev(pool, "bf16")
    ws = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, 3, 1, 64, 64, ec.EC_BF16)
    ec.ec_paged_evict_min(dev.k, dev.v, None, dev.mass, dev.table, ints(lens), ints([30, 20, 10]), None, 64, 0, 0, ws)
    pos = pool.pos.copy()  # not given, so it stays as it was
    ref.evict(pool, lens, [30, 20, 10], None, 64, 0, 0)
    pool.pos = pos
    dev.check(pool)


@pytest.mark.parametrize("G", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_generation_under_the_frequency_policy(G, dtype):
    """A prompt's rows are stored, then every token is appended, attended with and the lightest row removed; caches differ in length, one is
    still below its budget. The masses' differences are far above what they may be off, so both sides remove the same rows."""
    rng = np.random.default_rng(21)
    B, H, Hkv, D, page, budget = 3, 4, 2, 64, 8, [40, 57, 60]
    lens, seen = [40, 57, 50], [90, 130, 50]
    pool = make(rng, dtype, B, Hkv, G, D, page, 9, [71] * B, junk=0.0)
    dev = Dev(pool, dtype)
    T = 57
    k, v = (quantize(rng.standard_normal((B, Hkv, T, D)), dtype) for _ in range(2))
    pos = np.tile(np.arange(T, dtype=np.int32), (B, G, 1))
    mass = np.ascontiguousarray(rng.permuted(pos, axis=-1) * np.float32(0.5), dtype=np.float32)
    ec.ec_paged_store(to_dev(k, dtype), to_dev(v, dtype), ints(pos), torch.from_numpy(mass).cuda(), dev.table, dev.k, dev.v, dev.pos, dev.mass, None,
                      ints(lens))
    ref.store(pool, k, v, pos, mass, [0] * B, lens, T)
    dev.check(pool)
    ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, B, H, pool.slots, D, ec.dtype_code(dev.k))
    ws_e = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, B, G, 1, D, ec.dtype_code(dev.k))
    out = torch.empty((B, H, D), dtype=dev.k.dtype, device="cuda")
    for token in range(20):
        q, kn, vn = (quantize(rng.standard_normal(s), dtype) for s in ((B, H, D), (B, Hkv, D), (B, Hkv, D)))
        ec.ec_paged_decode_score_step(to_dev(q, dtype), to_dev(kn, dtype), to_dev(vn, dtype), dev.k, dev.v, dev.pos, dev.mass, dev.table, ints(lens),
                                      ints(seen), 0.125, out, ws)
        want, A, big = ref.step(pool, q.astype(np.float64), kn, vn, lens, seen, 0.125, True)
        assert (np.abs(to_host(out) - want) <= ref.attention_tolerance(dtype, want, A, big, 80, D)).all(), token
        lens, seen = [n + 1 for n in lens], [n + 1 for n in seen]
        ec.ec_paged_evict_min(dev.k, dev.v, dev.pos, dev.mass, dev.table, ints(lens), ints(budget), ints(seen), 1, 1, 5, ws_e)
        ref.evict(pool, lens, budget, seen, 1, 1, 5)
        lens = [max(min(n, c), n - 1) for n, c in zip(lens, budget)]
        assert lens == [40, 57, min(51 + token, 60)]
    dev.check(pool, (token + 1) * ref.mass_tolerance(big * 4, 80, D, pool.mass))


def test_captured_and_replayed():
    """A token's calls in one graph, lengths read on the device: every replay against the same calls made eagerly."""
    rng = np.random.default_rng(31)
    B, H, Hkv, D, page = 5, 16, 4, 128, 16
    lens = [0, 300, 17, 1000, -1]
    pool = make(rng, "bf16", B, Hkv, 1, D, page, 70, [1050] * B, extra=0, junk=0.5)
    side, graph = [Dev(pool, "bf16") for _ in range(2)], torch.cuda.CUDAGraph()
    q, kn, vn = (to_dev(quantize(rng.standard_normal(s), "bf16"), "bf16") for s in ((B, H, D), (B, Hkv, D), (B, Hkv, D)))
    state = [dict(lens=ints(lens), len1=ints(lens), pos=ints([2000] * B), keep=ints([1, 200, 100, 900, 5]), seen=ints([2001] * B),
                  out=torch.zeros((B, H, D), dtype=torch.bfloat16, device="cuda"),
                  ws=ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, B, H, pool.slots, D, ec.EC_BF16),
                  we=ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, B, 1, 40, D, ec.EC_BF16)) for _ in range(2)]

    def token(d, s):
        ec.ec_paged_decode_score_step(q, kn, vn, d.k, d.v, d.pos, d.mass, d.table, s["lens"], s["pos"], 0.1, s["out"], s["ws"])
        torch.add(s["lens"], 1, out=s["len1"])
        ec.ec_paged_evict_min(d.k, d.v, d.pos, d.mass, d.table, s["len1"], s["keep"], s["seen"], 40, 1, 3, s["we"])
        s["lens"].copy_(torch.maximum(torch.minimum(s["len1"], s["keep"]), s["len1"] - 40))
        s["pos"].add_(1), s["seen"].add_(1)
        ec.ec_paged_decode_step(q, kn, vn, d.k, d.v, None, d.table, s["lens"], None, 0.1, s["out"], s["ws"])

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        token(Dev(pool, "bf16"), dict(state[1], **{n: state[1][n].clone() for n in ("lens", "pos", "seen")}))  # warm-up
        with torch.cuda.graph(graph, stream=stream):
            token(side[1], state[1])
    torch.cuda.current_stream().wait_stream(stream)
    for replay in range(6):
        token(side[0], state[0])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((state[0]["out"], state[1]["out"]), (state[0]["lens"], state[1]["lens"]), (side[0].k, side[1].k), (side[0].v, side[1].v),
                     (side[0].pos, side[1].pos), (side[0].mass, side[1].mass)):
            assert torch.equal(a, b), replay


def test_same_call_same_bits():
    """Results do not depend on which workgroup ends first."""
    rng = np.random.default_rng(33)
    lens = [4000, 130, 77]
    pool = make(rng, "bf16", 3, 2, 1, 128, 16, 260, lens, junk=0.0)
    q, kn, vn = (to_dev(quantize(rng.standard_normal(s), "bf16"), "bf16") for s in ((3, 8, 128), (3, 2, 128), (3, 2, 128)))
    ws = ec.new_workspace(ec.EC_FN_PAGED_DECODE_SCORE_STEP, 3, 8, pool.slots, 128, ec.EC_BF16)
    got = []
    for _ in range(20):
        d, out = Dev(pool, "bf16") if not got else d, torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda")
        d.mass.fill_(1.0)
        ec.ec_paged_decode_score_step(q, kn, vn, d.k, d.v, None, d.mass, d.table, ints(lens), None, 0.1, out, ws)
        got.append((out, d.mass.clone()))
    assert all(torch.equal(a, got[0][0]) and torch.equal(m, got[0][1]) for a, m in got)


def test_calls_on_two_streams():
    """Two batches at once, each with its own workspace and stream."""
    rng = np.random.default_rng(35)
    lens = [900, 40]
    pools = [make(rng, "bf16", 2, 4, 1, 128, 16, 60, lens, junk=0.0) for _ in range(2)]
    want, work = [], []
    for pool in pools:
        q, kn, vn = (quantize(rng.standard_normal(s), "bf16") for s in ((2, 8, 128), (2, 4, 128), (2, 4, 128)))
        d = Dev(pool, "bf16")
        work.append((d, to_dev(q, "bf16"), to_dev(kn, "bf16"), to_dev(vn, "bf16"), torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda"),
                     ec.new_workspace(ec.EC_FN_PAGED_DECODE_STEP, 2, 8, pool.slots, 128, ec.EC_BF16), torch.cuda.Stream()))
        want.append(ref.step(pool, q.astype(np.float64), kn, vn, lens, None, 0.1, False))
    tl = ints(lens)
    torch.cuda.synchronize()
    for _ in range(10):
        for d, q, kn, vn, out, ws, stream in work:
            with torch.cuda.stream(stream):
                ec.ec_paged_decode_step(q, kn, vn, d.k, d.v, None, d.table, tl, None, 0.1, out, ws)
    torch.cuda.synchronize()
    for (o, A, big), w in zip(want, work):
        assert (np.abs(to_host(w[4]) - o) <= ref.attention_tolerance("bf16", o, A, big, 901, 128)).all()
