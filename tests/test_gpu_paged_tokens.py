"""PagedTokens: the three calls together over steps of mixed batches, against the definitions step by step, eager and replayed."""
import numpy as np
import pytest
import torch

import paged_ref
import token_ref as ref
from paper_2407_18121_amd import binding as ec
from paper_2407_18121_amd.pipeline import LayerState, PagedTokens, rotary_frequencies
from util import quantize, to_dev, to_host, torch_dtype

pytestmark = pytest.mark.gpu
LAYERS, PLACES, PAGE, MAX_PAGES = 2, 5, 16, 24


def _batch(dtype, H, Hkv, D, rot, tokens, n_pages, interleaved=False):
    freq, mscale = rotary_frequencies(rot, factor=4.0, kind="parts", trained=64)
    return PagedTokens(LAYERS, PLACES, tokens, H, Hkv, D, PAGE, n_pages, MAX_PAGES, torch_dtype(dtype), freq, mscale, interleaved)


def _check_step(batch, host, dtype, news, T, H, Hkv, D, scale, x, out, before):
    """A step that has run: the plan bit for bit, the rows that the pools took, attention over what they hold."""
    want = host.plan(before[0], news, before[1], T)
    got = (batch.start_b, batch.len_b, batch.seen_b, batch.token_start, batch.rows, batch.pos)
    for a, b in zip(got, want):
        assert np.array_equal(a.cpu().numpy(), b)
    assert np.array_equal(batch.table.cpu().numpy(), host.table) and int(batch.n_free) == host.n_free
    start, token_start, rows, pos = want[0], want[3], want[4], want[5]
    live = rows >= 0
    p, o = rows[live] // PAGE, rows[live] % PAGE
    freq = batch.freq.cpu().numpy()
    for layer in range(LAYERS):
        q, k, v = x[layer]
        k_pages, v_pages = to_host(batch.k_pages[layer]), to_host(batch.v_pages[layer])
        k_want, k_tol = ref.turned(k, pos, freq, batch.mscale, batch.interleaved, dtype)
        assert (np.abs(k_pages[p, :, o] - k_want[live]) <= k_tol[live]).all()
        assert np.array_equal(v_pages[p, :, o], v[live].astype(np.float64))
        assert np.array_equal(batch.pos_pages[layer].cpu().numpy()[p, 0, o], pos[live])
        # (the last layer's turned queries are still there; the first layer's differ by their own rounding only)
        if layer == LAYERS - 1:
            turned = to_host(batch.turned)
            q_want, q_tol = ref.turned(q, pos, freq, batch.mscale, batch.interleaved, dtype)
            assert (np.abs(turned - q_want) <= q_tol)[live].all()
            pool = paged_ref.Pool(k_pages, v_pages, np.zeros((1, 1, 1)), np.zeros((1, 1, 1)), host.table)
            pool.n_pages, pool.page = k_pages.shape[0], PAGE
            want_out, tol, _, _ = ref.chunk(pool, turned, start, token_start, scale, dtype)
            n = int(token_start[-1])
            ok = ref.fits(to_host(out[layer])[:n], want_out[:n], tol[:n])
            assert ok.all(), np.argwhere(~ok)[:4]
    return want


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D,rot,interleaved", [("bf16", 8, 2, 128, 128, False), ("bf16", 6, 6, 64, 40, True), ("f32", 4, 1, 64, 22, False)])
def test_steps(dtype, H, Hkv, D, rot, interleaved, captured):
    """Chunks of prompts, drafted tokens, single ones, sequences that end and begin, a pool that runs out: every step against the definitions; the same with one
    graph replayed for all steps, with the program's own work between the replays."""
    rng = np.random.default_rng(H + D)
    T, N = 160, 40
    batch = _batch(dtype, H, Hkv, D, rot, T, N, interleaved)
    host = ref.Planned(PLACES, PAGE, N, MAX_PAGES, np.arange(N - 1, -1, -1))
    scale = D ** -0.5
    fused = [torch.zeros(T, (H + 2 * Hkv) * D, dtype=torch_dtype(dtype), device="cuda") for _ in range(LAYERS)]
    parts = [(f[:, :H * D].view(T, H, D), f[:, H * D:(H + Hkv) * D].view(T, Hkv, D), f[:, (H + Hkv) * D:].view(T, Hkv, D)) for f in fused]
    out = torch.zeros(LAYERS, T, H, D, dtype=torch_dtype(dtype), device="cuda")

    def step():
        batch.begin()
        for i in range(LAYERS):
            batch.attend(i, *parts[i], scale, out[i])
    graph = None
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    length, seen = np.full(PLACES, -1), np.zeros(PLACES, np.int64)
    plans = [([0, 1], [], [100, 7, 0, 0, 0]), ([], [], [5, 60, 0, 0, 0]), ([2, 4], [], [1, 1, 33, 0, 90]), ([], [0], [3, 1, 1, 0, 1]), ([0, 3], [4], [70, 1, 40, 20, 1]),
             ([], [], [150, 2, 3, 4, 0]), ([], [1], [1, 0, 1, 1, 0]), ([1], [], [60, 90, 1, 1, 0]), ([], [0, 2], [1, 1, 1, 1, 1])]
    for admit, release, news in plans:
        batch.admit(admit) if admit else None
        batch.release(release) if release else None
        length[admit], seen[admit], length[release], seen[release] = 0, 0, -1, 0
        x = []
        for i in range(LAYERS):
            y = quantize(rng.standard_normal((T, H + 2 * Hkv, D)), dtype)
            fused[i].copy_(to_dev(y.reshape(T, -1), dtype))
            x.append((y[:, :H], y[:, H:H + Hkv], y[:, H + Hkv:]))
        batch.new_b.copy_(torch.tensor(news, dtype=torch.int32))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        want = _check_step(batch, host, dtype, news, T, H, Hkv, D, scale, x, out, (length.copy(), seen.copy()))
        length, seen = want[1].astype(np.int64), want[2].astype(np.int64)
    assert (want[0] == -1).any()  # the pool has run out on the way, and places were free


def test_compressed_prompts_come_in_as_rows():
    """A prompt is compressed by LayerState, its rows are stored, and tokens attend to them."""
    B, H, D, T, n = 2, 4, 64, 200, 50
    rng = np.random.default_rng(3)
    host = [quantize(rng.standard_normal((B, H, T, D)), "bf16") for _ in range(3)]
    state = LayerState(B, H, D, T, n, n, torch.bfloat16, (1, 4))
    state.prefill(*(to_dev(x, "bf16") for x in host), D ** -0.5, ec.new_workspace(ec.EC_FN_PREFILL_SCORE, B, H, T, D, ec.EC_BF16))
    freq, mscale = rotary_frequencies(D)
    batch = PagedTokens(1, 4, 16, H, H, D, PAGE, 30, 8, torch.bfloat16, freq, mscale)
    batch.admit([3, 1], [n, n], [T, T])
    batch.begin()
    mass = torch.rand(B, 1, n, device="cuda")
    batch.store(0, [3, 1], state.k_cache, state.v_cache, state.pos, mass)
    batch.new_b.copy_(torch.tensor([0, 3, 0, 5], dtype=torch.int32))
    batch.begin()
    assert batch.start_b.tolist() == [-1, n, -1, n] and batch.len_b.tolist() == [-1, n + 3, -1, n + 5] and batch.seen_b.tolist() == [0, T + 3, 0, T + 5]
    assert batch.pos[:8].tolist() == [T, T + 1, T + 2, T, T + 1, T + 2, T + 3, T + 4]
    q, k, v = (to_dev(quantize(rng.standard_normal((16, H, D)), "bf16"), "bf16") for _ in range(3))
    out = torch.zeros_like(q)
    batch.attend(0, q, k, v, D ** -0.5, out)
    pool = paged_ref.Pool(to_host(batch.k_pages[0]), to_host(batch.v_pages[0]), np.zeros((1, 1, 1)), np.zeros((1, 1, 1)), batch.table.cpu().numpy())
    want, tol, _, _ = ref.chunk(pool, to_host(batch.turned), [-1, n, -1, n], [0, 0, 3, 3, 8], D ** -0.5, "bf16")
    assert (np.abs(to_host(out)[:8] - want[:8]) <= tol[:8]).all() and not out[8:].any()
    for b, place in enumerate((3, 1)):
        p, o = pool.table[place, np.arange(n) // PAGE], np.arange(n) % PAGE
        assert np.array_equal(pool.k[p, :, o], to_host(state.k_cache[b]).transpose(1, 0, 2)[:n])
    batch.release([3])
    batch.new_b.zero_()
    batch.begin()
    assert int(batch.n_free) == 30 - -(-(n + 3) // PAGE)


def test_sequences_do_not_come_and_go_in_a_capture():
    freq, mscale = rotary_frequencies(64)
    batch = PagedTokens(1, 2, 8, 2, 2, 64, PAGE, 8, 4, torch.float32, freq, mscale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="outside a capture"):
            batch.admit([0])
        batch.begin()
    for bad in ([0, 0], [2], [-1]):
        with pytest.raises(ValueError):
            batch.admit(bad)
    with pytest.raises(ValueError):
        batch.admit([0], [3, 4])
