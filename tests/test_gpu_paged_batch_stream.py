"""PagedBatch does not wait for the device: a token is prepared while those before it run, and still finds the lengths and pages of its own."""
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from paper_2407_18121_amd.pipeline import PagedBatch

pytestmark = pytest.mark.gpu
L, PLACES, H, HKV, D, PAGE = 2, 5, 4, 2, 64, 8
ROWS, SEEN = [30, 7, 64, 9], [90, 7, 70, 33]


def admitted(dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(1)
    batch = PagedBatch(L, PLACES, H, HKV, D, PAGE, 80, 16, dtype, recent=4)
    n = max(ROWS)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(dtype)  # noqa: E731
    batch.admit([3, 0, 4, 1], ROWS, SEEN)
    for i in range(L):
        batch.store(i, [3, 0, 4, 1], rand(4, HKV, n, D), rand(4, HKV, n, D), torch.arange(n, dtype=torch.int32, device="cuda").expand(4, 1, n).contiguous(),
                    torch.rand(4, 1, n, device="cuda", generator=g))
    return batch


def tokens(batch, count, inputs, out, between=lambda: None):
    for t in range(count):
        keep = None if t % 7 == 6 else 40 + t % 3
        batch.begin()
        between()
        for i in range(L):
            q, k, v = (x[t, i] for x in inputs)
            batch.decode(i, q, k, v, 0.125, out[t, i]) if keep is None else batch.decode_scored(i, q, k, v, 0.125, out[t, i], keep)
        between()
        batch.end(keep)
        between()
        if t == 20:
            batch.shrink(25)
            batch.release(0)
        if t == 24:
            batch.admit([0], [0], [0])


def made(count):
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda heads: torch.randn((count, L, PLACES, heads, D), device="cuda", generator=g).bfloat16()  # noqa: E731
    return (rand(H), rand(HKV), rand(HKV)), torch.zeros((count, L, PLACES, H, D), dtype=torch.bfloat16, device="cuda")


def test_tokens_do_not_wait():
    """Everything that would synchronize raises."""
    inputs, out = made(40)
    batch = admitted()
    ec.load()
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        tokens(batch, 40, inputs, out)
    finally:
        torch.cuda.set_sync_debug_mode("default")


def test_tokens_far_ahead_of_the_device():
    """Forty tokens queued behind long products, against the same ones waited for one call at a time."""
    inputs, want = made(40)
    got, batches = torch.zeros_like(want), [admitted(), admitted()]
    tokens(batches[0], 40, inputs, want, torch.cuda.synchronize)
    big = torch.randn(8192, 8192, device="cuda").bfloat16()
    torch.cuda.synchronize()
    for _ in range(150):
        big @ big
    end = torch.cuda.Event()
    end.record()
    tokens(batches[1], 40, inputs, got)
    assert not end.query()  # the products were still running when the last token was queued
    torch.cuda.synchronize()
    assert torch.equal(got, want) and batches[0].rows == batches[1].rows
    for name in ("k_pages", "v_pages", "pos_pages", "mass_pages", "table", "numbers"):
        assert torch.equal(getattr(batches[0], name), getattr(batches[1], name)), name


def test_layers_of_a_captured_token_share_the_budget():
    """After a token with that budget a graph takes its tensor, and keeps it while other budgets are used."""
    batch = admitted()
    eager = batch._budget(12)
    batch._budget(13)
    graph = torch.cuda.CUDAGraph()
    held = []
    with torch.cuda.graph(graph):
        held += [batch._budget(12), batch._budget(12), batch._budget(11), batch._budget(11)]
        copy = held[0] + held[2]
    assert held[0] is held[1] is eager and held[2] is not held[3] and 11 not in batch.budgets
    for keep in range(20, 60):
        batch._budget(keep)
    for _ in range(3):
        graph.replay()
        assert copy.eq(23).all() and batch._budget(12).eq(12).all()


def test_what_the_host_sends_is_not_captured():
    """Refused with everything as it was, and the graph of a token around it still works."""
    batch = admitted()
    inputs, out = made(1)
    x = [x[0, 0] for x in inputs]
    kv, pos = torch.zeros(1, HKV, 64, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 64, dtype=torch.int32, device="cuda")
    batch.begin()
    batch.decode(0, *x, 0.125, out[0, 0])
    state = lambda: (list(batch.rows), list(batch.seen), [list(h) for h in batch.held], list(batch.free), dict(batch.changes))  # noqa: E731
    before, graph = state(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: batch.admit([2], [3], [3]), lambda: batch.release(0), lambda: batch.store(0, [0], kv, kv, pos, pos.float()), batch.begin, batch.end,
                     lambda: batch.shrink(3)):
            with pytest.raises(RuntimeError, match="cannot be captured"):
                call()
        batch.decode(0, *x, 0.125, out[0, 1])
    graph.replay()
    assert state() == before and torch.equal(out[0, 0], out[0, 1])
    batch.end()
    assert batch.numbers[0].tolist() == [8, 10, -1, 31, 65]
