"""Attention of several new tokens over paged caches against the definition in 64 bits (token_ref.chunk)."""
import numpy as np
import pytest
import torch

import paged_ref
import token_ref as ref
from paper_2407_18121_amd import binding as ec
from util import quantize, to_dev, to_host, torch_dtype

pytestmark = pytest.mark.gpu


def make(rng, dtype, Hkv, D, page, used, spare=2, gain=1.0, junk=np.nan):
    """A pool whose sequences use so many rows each, pages anywhere; `junk` in all rows that are no sequence's."""
    need = [-(-max(n, 0) // page) for n in used]
    N, most = sum(need) + spare, max(max(need), 1) + 1
    table, order, at = np.full((len(used), most), -1, np.int32), rng.permutation(N), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (np.full((N, Hkv, page, D), junk, np.float32) for _ in range(2))
    for b, n in enumerate(used):
        s = np.arange(max(n, 0))
        p, o = table[b, s // page], s % page
        # rows that draw much attention and others
        k[p, :, o] = quantize(rng.standard_normal((len(s), Hkv, D)) * np.where(rng.random(len(s)) < 0.1, 3.0, 0.7)[:, None, None] * gain, dtype)
        v[p, :, o] = quantize(rng.standard_normal((len(s), Hkv, D)), dtype)
    z = np.zeros((N, 1, page))
    return paged_ref.Pool(k, v, z.astype(np.int32), z, table)


def run(pool, dtype, H, start, news, scale=None, pad=0, seed=0, lse=True, q=None, ws=None):
    """A step over the pool; (out, lse) of the device. Rows of padding have to stay as they are."""
    rng = np.random.default_rng(seed)
    D, B = pool.k.shape[3], len(start)
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    T = int(starts[-1]) + pad
    scale = D ** -0.5 if scale is None else scale
    if q is None:
        q = quantize(rng.standard_normal((T, H, D)), dtype)
    out = torch.full((T, H, D), 5.5, dtype=torch_dtype(dtype), device="cuda")
    got_lse = torch.full((T, H), 6.5, device="cuda") if lse else None
    if ws is None:  # nothing in it counts
        ws = torch.full_like(ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, B, H, T, D, ec.EC_BF16 if dtype == "bf16" else ec.EC_F32), 255)
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    assert ec.ec_paged_chunk_step(to_dev(q, dtype), to_dev(pool.k, dtype), to_dev(pool.v, dtype), i(pool.table), i(start), i(starts), scale, out, ws, got_lse) == ec.EC_OK
    want, tol, want_lse, lse_tol = ref.chunk(pool, q, start, starts, scale, dtype)
    got = to_host(out)
    live = slice(0, int(starts[-1]))
    ok = ref.fits(got[live], want[live], tol[live])
    assert ok.all(), (np.argwhere(~ok)[:5].tolist(), got[live][~ok][:5], want[live][~ok][:5], tol[live][~ok][:5])
    assert (got[int(starts[-1]):] == 5.5).all()
    if lse:
        got_lse = to_host(got_lse)
        ok = ref.fits(got_lse[live], want_lse[live], lse_tol[live])
        assert ok.all(), (np.argwhere(~ok)[:5].tolist(), got_lse[live][~ok][:5], want_lse[live][~ok][:5])
        assert (got_lse[int(starts[-1]):] == 6.5).all()
    return out, got_lse


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,n", [(0, 1), (0, 5), (1, 1), (15, 2), (63, 1), (64, 1), (63, 3), (100, 5), (127, 17), (250, 40), (0, 300), (577, 129)])
def test_lengths(dtype, D, L, n):
    rng = np.random.default_rng(L + n)
    run(make(rng, dtype, 2, D, 16, [L + n]), dtype, 4, [L], [n], pad=2)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("rows", [257, 281, 384, 449, 500, 512, 513, 530])
def test_lengths_where_cutting_begins(dtype, D, rows):
    """Whether a table is long enough for tiles to be cut is the host's to say, how they are cut the device's."""
    rng = np.random.default_rng(rows)
    for news in ([1], [9], [60], [150], [2, 60, 1]):
        run(make(rng, dtype, 3, D, 16, [rows] * len(news), spare=0), dtype, 6, [rows - n for n in news], news)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("Hkv", [4, 32, 64])
@pytest.mark.parametrize("L,news", [([0], [600]), ([700, 33], [90, 470]), ([511], [577])])
def test_few_and_many_tiles(D, Hkv, L, news):
    """Batches with fewer tiles than half the compute units, fewer than all of them, and more: three ways to share rows and slots among a workgroup's waves."""
    rng = np.random.default_rng(Hkv + len(L))
    run(make(rng, "bf16", Hkv, D, 32, [a + b for a, b in zip(L, news)]), "bf16", Hkv, L, news, pad=1)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (3, 1), (10, 2), (14, 2), (16, 1), (33, 1), (32, 4), (64, 1)])
def test_query_groups(dtype, D, H, Hkv):
    rng = np.random.default_rng(H)
    news = [1, 2, 5, 11, 33, 70]
    L = [90, 0, 200, 7, 130, 64]
    run(make(rng, dtype, Hkv, D, 8, [a + b for a, b in zip(L, news)]), dtype, H, L, news)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_pages(dtype, page):
    rng = np.random.default_rng(page)
    news, L = [3, 140, 1, 31], [page * 2 - 1, page + 3, page * 3, 0]
    run(make(rng, dtype, 2, 128, page, [a + b for a, b in zip(L, news)]), dtype, 6, L, news)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [5, 64, 65, 200, 1100])
def test_batches(dtype, B):
    """Mixed batches: chunks beside single tokens, places without a sequence (their tokens are zeros) and sequences without tokens."""
    rng = np.random.default_rng(B)
    news = np.where(rng.random(B) < 0.2, rng.integers(2, 60, B), rng.integers(0, 2, B))
    L = rng.integers(0, 90, B)
    L[rng.random(B) < 0.1] = -1
    L[B // 2], news[B // 2] = 1 << 20, 4  # behind every table
    news[0], L[0] = 150, 10
    run(make(rng, dtype, 1, 64, 16, [0 if x < 0 or x > 1000 else x + n for x, n in zip(L, news)]), dtype, 2, L, news, pad=3)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("news", [[1], [4], [33], [200], [1, 130, 6], [300, 1, 1, 1]])
def test_long_caches(dtype, D, news):
    """Long enough to be cut into segments that another launch joins, also where only some sequences of a batch are."""
    rng = np.random.default_rng(len(news))
    L = [6000, 2500, 100, 17][:len(news)]
    run(make(rng, dtype, 2, D, 64, [a + b for a, b in zip(L, news)], gain=0.6), dtype, 8, L, news)


def test_many_segments():
    rng = np.random.default_rng(1)
    run(make(rng, "bf16", 1, 128, 256, [40003]), "bf16", 8, [40000], [3])
    run(make(rng, "bf16", 1, 64, 256, [40200]), "bf16", 4, [40000], [200])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages(dtype):
    """Rows on no page weigh nothing; a token that sees none but such rows gets zeros and an lse of -inf."""
    rng = np.random.default_rng(4)
    news, L = [40, 150, 3, 200], [0, 90, 500, 0]
    pool = make(rng, dtype, 2, 128, 16, [a + b for a, b in zip(L, news)])
    pool.table[0, 0] = -1                       # the first 16 tokens see nothing
    pool.table[1, [1, 4, 7]] = [pool.n_pages, -5, 2 ** 31 - 1]
    pool.table[2, :40] = -1                     # nothing at all
    pool.table[3, 0:9] = -1
    out, lse = run(pool, dtype, 4, L, news)
    assert not out[:16].any() and np.isneginf(lse[:16]).all() and not out[190:193].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_behind_the_table(dtype):
    """New tokens whose slots the table does not reach see all that it has."""
    rng = np.random.default_rng(4)
    pool = make(rng, dtype, 2, 64, 8, [40, 40, 40])
    pool.table = pool.table[:, :5]
    pool.slots = 40
    run(pool, dtype, 4, [30, 39, 38], [20, 1, 300])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("news", [[7], [30], [100], [200]])
def test_infinite_values_of_rows_that_are_not_seen_yet(dtype, D, news):
    """An infinite or NaN row of V reaches the tokens from its own on, feature by feature, and no earlier one; one before the chunk reaches all."""
    rng = np.random.default_rng(2)
    L = 70
    for which in range(2):
        pool = make(rng, dtype, 1, D, 16, [L + news[0]], gain=0.3)
        rows = [L + 2, L + 3, L + news[0] - 2, L + news[0] // 2, L + 4] + ([3] if which else [])
        for i, r in enumerate(rows):
            p, o = pool.at(0, r)
            pool.v[p, 0, o, 5 * i] = (np.inf, -np.inf, np.nan, np.inf, -np.inf, np.inf)[i]
            pool.v[p, 0, o, 33] = (np.inf, np.inf, np.inf, -np.inf, np.inf, np.inf)[i]  # both signs from some token on: NaN
        run(pool, dtype, 2, [L], news, pad=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 150])
def test_scores_of_minus_infinity(dtype, n):
    """Scores beyond the range weigh nothing; tokens that see nothing else get zeros. Large finite ones are compared as they are."""
    rng = np.random.default_rng(9)
    L = 20
    pool = make(rng, dtype, 1, 64, 8, [L + n])
    q = np.zeros((n, 2, 64), np.float32)
    q[:, 0, 0], q[:, 1, 0] = 4.0, 1.0
    pool.k[:] = 0
    s = np.arange(L + n)
    p, o = pool.table[0, s // 8], s % 8
    low = quantize(np.float32(-2.9e38), dtype)
    pool.k[p, 0, o, 0] = np.where(s < L + 2, low, quantize(rng.uniform(-2, 2, len(s)), dtype))  # head 0: -inf for the first two tokens, head 1: finite
    out, _ = run(pool, dtype, 2, [L], [n], scale=1.0, q=q)
    assert not out[:2, 0].any() and out[:2, 1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales(dtype):
    rng = np.random.default_rng(6)
    for scale in (1e-3, 1.0, 3.7):
        run(make(rng, dtype, 2, 64, 32, [150, 300], gain=0.4), dtype, 4, [100, 10], [50, 290], scale=scale)


def test_shared_prefix():
    rng = np.random.default_rng(7)
    pool = make(rng, "bf16", 2, 128, 16, [96, 96, 96])
    pool.table[1, :4] = pool.table[2, :4] = pool.table[0, :4]
    run(pool, "bf16", 8, [64, 64, 90], [32, 5, 6])


def test_pools_beyond_4_gib():
    N, Hkv, page, D, H = 2100, 8, 256, 128, 16
    k, v = (torch.full((N, Hkv, page, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(3)
    ids = [N - 1, 0, N - 2, 1234]
    rows = [quantize(rng.standard_normal((len(ids), Hkv, page, D)), "bf16") for _ in range(2)]
    for i, p in enumerate(ids):
        k[p], v[p] = (to_dev(x[i], "bf16") for x in rows)
    L, n = 880, 140
    small = paged_ref.Pool(rows[0], rows[1], np.zeros((4, 1, page), np.int32), np.zeros((4, 1, page)), np.array([[0, 1, 2, 3]], np.int32))
    q = quantize(rng.standard_normal((n, H, D)), "bf16")
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, ws = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda"), ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, n, D, ec.EC_BF16)
    for m in (2, n):
        ec.ec_paged_chunk_step(to_dev(q[:m], "bf16"), k, v, i([ids]), i([L]), i([0, m]), D ** -0.5, out[:m], ws)
        want, tol, _, _ = ref.chunk(small, q[:m], [L], [0, m], D ** -0.5, "bf16")
        assert (np.abs(to_host(out[:m]) - want) <= tol).all()


def test_same_bits_every_time():
    rng = np.random.default_rng(5)
    pool, (L, news) = make(rng, "bf16", 2, 128, 32, [3005, 900, 401]), ([3000, 700, 400], [5, 200, 1])
    first = run(pool, "bf16", 8, L, news)
    for _ in range(3):
        again = run(pool, "bf16", 8, L, news)
        assert torch.equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_replays_and_streams():
    """A captured step follows the lengths on the device; two steps on two streams with workspaces of their own do not disturb each other."""
    rng = np.random.default_rng(11)
    B, H, Hkv, D, page, T = 4, 8, 2, 128, 16, 300
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    sets = []
    for seed in range(2):
        pool = make(rng, "bf16", Hkv, D, page, [3000] * B, junk=0.0)
        q = quantize(rng.standard_normal((T, H, D)), "bf16")
        sets.append(dict(pool=pool, q=q, dq=to_dev(q, "bf16"), k=to_dev(pool.k, "bf16"), v=to_dev(pool.v, "bf16"), table=i(pool.table), start=i([0] * B), ts=i([0] * (B + 1)),
                         out=torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda"), ws=ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, B, H, T, D, ec.EC_BF16),
                         stream=torch.cuda.Stream()))
    call = lambda s: ec.ec_paged_chunk_step(s["dq"], s["k"], s["v"], s["table"], s["start"], s["ts"], 0.1, s["out"], s["ws"])  # noqa: E731
    torch.cuda.synchronize()
    for s in sets:
        s["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["graph"]):
            call(s)
    for step in range(4):
        todo = []
        for s in sets:
            L, news = rng.integers(0, 2600, B), rng.integers(0, 75, B)
            L[step] = -1
            starts = np.concatenate([[0], np.cumsum(news)])
            s["start"].copy_(i(L)), s["ts"].copy_(i(starts))
            todo.append((s, L, starts))
        torch.cuda.synchronize()
        for s in sets:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay() if step % 2 else call(s)
        torch.cuda.synchronize()
        for s, L, starts in todo:
            want, tol, _, _ = ref.chunk(s["pool"], s["q"], L, starts, 0.1, "bf16")
            assert (np.abs(to_host(s["out"]) - want) <= tol)[:starts[-1]].all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("T,slots", [(40, 4096), (300, 1024)])
def test_tokens_that_overlap_stay_inside(dtype, D, T, slots):
    """What tokens of several sequences get is not specified, but nothing beside out, lse and the workspace's bytes is written, however many tiles that makes."""
    B, H, Hkv, page = 96, 4, 2, 32
    rng = np.random.default_rng(T)
    pool = make(rng, dtype, Hkv, D, page, [slots])
    code = ec.EC_BF16 if dtype == "bf16" else ec.EC_F32
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    size = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, B, H, T, D, code).numel()
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    out = torch.full((T + 8, H, D), 5.5, dtype=torch_dtype(dtype), device="cuda")
    lse = torch.full((T + 8, H), 6.5, device="cuda")
    q = to_dev(quantize(rng.standard_normal((T, H, D)), dtype), dtype)
    k, v = to_dev(pool.k, dtype), to_dev(pool.v, dtype)
    table = i(np.repeat(pool.table[:1], B, 0))
    for starts in ([0, T] * (B // 2) + [0], [2 ** 31 - 1, -5] * (B // 2) + [T], list(rng.integers(-T, 2 * T, B + 1))):
        for start in ([slots - T] * B, list(rng.integers(-2, slots + 2, B)), [2 ** 31 - 1] * B):
            assert ec.ec_paged_chunk_step(q, k, v, table, i(start), i(starts), 0.1, out[:T], ws[:size], lse[:T]) == ec.EC_OK
            torch.cuda.synchronize()
            assert (ws[size:] == 77).all() and (out[T:] == 5.5).all() and (lse[T:] == 6.5).all()


@pytest.mark.parametrize("dtype,D,H", [("bf16", 128, 1), ("bf16", 64, 40), ("f32", 64, 1)])
def test_the_longest_cache(dtype, D, H):
    """2^28 slots, the most there are, all on one page: every row of it counts equally often, so that the output is that of the page alone. A lane adds up to 2^28 / (256
    segments, 4 waves, 16 slots) = 16384 times 1 to 4 numbers of its own: within 2^16 roundings."""
    page, rng = 256, np.random.default_rng(4)
    pool = make(rng, dtype, 1, D, page, [page], spare=0)
    q = quantize(rng.standard_normal((1, H, D)), dtype)
    pool.table = np.zeros((1, 1), np.int32)
    want, tol, lse, lse_tol = ref.chunk(pool, q, [page - 1], [0, 1], D ** -0.5, dtype)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, got_lse = torch.empty(1, H, D, dtype=torch_dtype(dtype), device="cuda"), torch.empty(1, H, device="cuda")
    ws = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, 1, D, ec.EC_BF16 if dtype == "bf16" else ec.EC_F32)
    table = torch.zeros((1, 2 ** 28 // page), dtype=torch.int32, device="cuda")
    ec.ec_paged_chunk_step(to_dev(q, dtype), to_dev(pool.k, dtype), to_dev(pool.v, dtype), table, i([2 ** 28 - 1]), i([0, 1]), D ** -0.5, out, ws, got_lse)
    more = 2.0 ** 16 * ref.U
    w = np.abs(pool.v).max()
    assert (np.abs(to_host(out) - want) <= tol + 2 * more * w).all()
    assert (np.abs(to_host(got_lse) - (lse + 20 * np.log(2))) <= lse_tol + more + 64 * ref.U).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wide_tables(dtype):
    """A table with room for 2^28 slots gives what one that just holds the sequences does, bit for bit."""
    H, D, page, L, n = 16, 128, 256, 1500, 2048
    rng = np.random.default_rng(8)
    pool = make(rng, dtype, H, D, page, [L + n])
    q = to_dev(quantize(rng.standard_normal((n, H, D)), dtype), dtype)
    k, v = to_dev(pool.k, dtype), to_dev(pool.v, dtype)
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    wide = torch.full((1, 2 ** 28 // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :pool.table.shape[1]] = i(pool.table)
    ws = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, n, D, ec.EC_BF16 if dtype == "bf16" else ec.EC_F32)
    out = []
    for table in (i(pool.table), wide):
        out.append(torch.empty_like(q))
        ec.ec_paged_chunk_step(q, k, v, table, i([L]), i([0, n]), D ** -0.5, out[-1], ws)
    assert torch.equal(out[0], out[1]) and not torch.isnan(out[0]).any()
