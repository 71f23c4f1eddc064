"""Pages and slots planned on the device against the same rules followed page by page on the host: every array, bit for bit."""
import numpy as np
import pytest
import torch

import token_ref as ref
from paper_2407_18121_amd import binding as ec

pytestmark = pytest.mark.gpu


class Device:
    """The arrays of a plan on the device, from a host plan's state."""

    def __init__(self, host):
        i = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.table, self.held, self.stack, self.n_free = i(host.table), i(host.held), i(host.stack), torch.tensor([host.n_free], dtype=torch.int32, device="cuda")
        self.page = host.page

    def plan(self, length, new, seen, T, maps=True, in_place=False):
        B = len(length)
        i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        blank = lambda n, dt=torch.int32: torch.full((n,), -77, dtype=dt, device="cuda")  # noqa: E731
        length, seen = i(length), None if seen is None else i(seen)
        self.len, self.new = length, i(new)
        self.start, self.token_start = blank(B), blank(B + 1)
        self.after, self.seen_after = (length, seen) if in_place else (blank(B), None if seen is None else blank(B))
        self.rows, self.pos = (blank(T, torch.int64), blank(T)) if maps else (None, None)
        assert ec.ec_paged_plan(length, self.new, self.table, self.held, self.stack, self.n_free, self.page, self.start, self.after, self.token_start, self.rows,
                                self.pos, seen_b=seen, seen_after_b=self.seen_after, T=T) == ec.EC_OK


def compare(host, dev, want):
    got = dict(table=dev.table, held=dev.held, stack=dev.stack, n_free=dev.n_free, start=dev.start, after=dev.after, seen_after=dev.seen_after,
               token_start=dev.token_start, rows=dev.rows, pos=dev.pos)
    want = dict(zip(("start", "after", "seen_after", "token_start", "rows", "pos"), want), table=host.table, held=host.held, stack=host.stack, n_free=[host.n_free])
    for name, x in got.items():
        if x is not None:
            assert np.array_equal(x.cpu().numpy(), want[name]), name


@pytest.mark.parametrize("B,page,most,share", [(1, 16, 8, 1.0), (2, 8, 40, 0.5), (16, 16, 70, 1.0), (63, 32, 9, 0.6), (64, 64, 5, 0.9), (65, 8, 33, 0.4), (257, 16, 12, 0.7),
                                               (1000, 256, 3, 0.8), (1025, 8, 6, 0.5), (8192, 128, 2, 0.6)])
def test_steps_of_a_batch(B, page, most, share):
    """Sequences come, grow, shrink and end over several steps, out of a pool that does not hold all of them: what one step leaves is where the next starts."""
    rng = np.random.default_rng(B + page)
    N = max(int(B * most * share), 1)
    host = ref.Planned(B, page, N, most, rng.permutation(N))
    dev = Device(host)
    length, seen = np.full(B, -1, np.int64), np.zeros(B, np.int64)
    for step in range(6):
        kind = rng.random(B)
        length = np.where(kind < 0.1, -1, np.where((kind < 0.3) | (length < 0), np.minimum(length, rng.integers(0, page * most, B)), length))
        length = np.where((length < 0) & (rng.random(B) < 0.5), 0, length)  # a new sequence
        new = np.where(rng.random(B) < 0.5, 1, rng.integers(-2, 3 * page, B))
        new[rng.integers(0, B)] = page * most + 1  # more than a table holds, or exactly
        total = int(np.maximum(new, 0).sum())
        T = max(total + (5 if step % 2 else -page), 1)  # the last tokens of every second step have no room
        T = 1 if step == 4 else T
        with_seen = step != 2
        want = host.plan(length, new, seen if with_seen else None, T)
        dev.plan(length, new, seen if with_seen else None, T, maps=step != 3, in_place=step == 1)
        compare(host, dev, want)
        length, seen = want[1].astype(np.int64), want[2].astype(np.int64) if with_seen else seen
        held = [p for b in range(B) for p in host.table[b, :host.held[b]]]
        assert sorted(held + list(host.stack[:host.n_free])) == list(range(N))  # every page is somewhere, once


def test_the_first_that_misses_pages_holds_up_the_others():
    host = ref.Planned(4, 8, 5, 8, [4, 3, 2, 1, 0])
    dev = Device(host)
    args = ([0, 0, 0, 0], [8, 40, 8, 0], [3, 4, 5, 6], 60)
    want = host.plan(*args)
    dev.plan(*args)
    compare(host, dev, want)
    assert list(want[0]) == [0, -1, -1, 0] and list(want[2]) == [11, 4, 5, 6] and host.n_free == 4
    assert list(want[4][:8]) == list(range(8)) and (want[4][8:] == -1).all()


def test_pages_that_are_given_back_are_taken_in_the_same_step():
    host = ref.Planned(3, 8, 6, 6, [0, 1, 2, 3, 4, 5])
    dev = Device(host)
    for args in (([0, 0, 0], [33, 8, 0], [0, 0, 0], 64), ([-1, 8, 0], [0, 24, 16], [9, 9, 9], 64), ([-1, 3, 0], [5, 0, 16], [1, 2, 3], 64)):
        want = host.plan(*args)
        dev.plan(*args)
        compare(host, dev, want)
    assert host.n_free == 3


def test_extreme_numbers():
    """Lengths and counts near 2^31 wrap round nowhere; table entries that name no page give rows of none."""
    big = 2 ** 31 - 1
    host = ref.Planned(6, 256, 40, 5, np.arange(40))
    host.table[5, :2], host.held[5] = [99, -5], 2
    dev = Device(host)
    args = ([0, big, 5, -big, 1, 300], [big, big, 3, 7, 1279, 5], [1, 2, big - 1, 4, 5, 6], 1 << 12)
    with np.errstate(over="ignore"):
        host_args = (args[0], [min(x, 1 << 13) for x in args[1]], [1, 2, 0, 4, 5, 6], args[3])  # (int32 wraps for the third's position: looked at below)
        want = list(host.plan(*host_args))
    dev.plan(*args)
    assert (dev.start.cpu().numpy() == -1).tolist() == [True] * 6  # no token lies before T, as the first sequence brings more than that
    assert np.array_equal(dev.token_start.cpu().numpy()[1:], [1 << 12] * 6) and np.array_equal(dev.start.cpu().numpy(), want[0])
    assert np.array_equal(dev.after.cpu().numpy(), [0, big, 5, -1, 1, 300])
    assert np.array_equal(dev.table.cpu().numpy(), host.table) and np.array_equal(dev.stack.cpu().numpy(), host.stack)
    host.table[5, :2], host.held[5] = [99, -5], 2
    dev = Device(host)
    args = ([0, big, 5, -big, 1, 300], [4, 9, 3, 7, 1279, 5], [1, 2, 3, 4, 5, 6], 2000)
    want = host.plan(*args)
    dev.plan(*args)
    compare(host, dev, want)
    assert (want[4][-(2000 - 1307):] == -1).all() and want[0].tolist() == [0, -1, 5, -1, 1, 300]


def test_a_state_that_is_none_stays_within_its_arrays():
    """More pages held and free than there are: unspecified pages, but nothing outside the arrays."""
    B, page, most, N = 40, 8, 9, 30
    rng = np.random.default_rng(3)
    guard = lambda n: torch.full((n + 128,), -123, dtype=torch.int32, device="cuda")  # noqa: E731
    table, stack, held, free = guard(B * most), guard(N), guard(B), guard(1)
    table[64:64 + B * most] = torch.from_numpy(rng.integers(-50, 50, B * most).astype(np.int32)).cuda()
    held[64:64 + B] = torch.from_numpy(rng.integers(-4, 30, B).astype(np.int32)).cuda()
    free[64] = 99
    inner = lambda x, n: x[64:64 + n]  # noqa: E731
    for _ in range(3):
        length, new = (torch.from_numpy(rng.integers(-3, 80, B).astype(np.int32)).cuda() for _ in range(2))
        out = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B, B, B + 1)]
        ec.ec_paged_plan(length, new, inner(table, B * most).view(B, most), inner(held, B), inner(stack, N), inner(free, 1), page, *out, T=500)
        for x, n in ((table, B * most), (stack, N), (held, B), (free, 1)):
            assert (x[:64] == -123).all() and (x[64 + n:] == -123).all()
        assert (inner(held, B) >= 0).all() and (inner(held, B) <= most).all() and 0 <= int(free[64]) <= N


def test_replayed_steps():
    """A captured step whose lengths stay on the device: replays follow what the rules give, with eager work of the program between them."""
    B, page, most, N, T = 9, 8, 20, 120, 40
    rng = np.random.default_rng(8)
    host = ref.Planned(B, page, N, most, rng.permutation(N))
    dev = Device(host)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    length, seen, new, start, token_start = i([0] * B), i([0] * B), i([1] * B), i([0] * B), i([0] * (B + 1))
    rows, pos = torch.zeros(T, dtype=torch.int64, device="cuda"), i([0] * T)
    call = lambda: ec.ec_paged_plan(length, new, dev.table, dev.held, dev.stack, dev.n_free, page, start, length, token_start, rows, pos, seen, seen)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    at, saw = np.zeros(B, np.int64), np.zeros(B, np.int64)
    for step in range(12):
        n = rng.integers(0, 5, B)
        if step == 6:
            at[2:5] = -1
            length[2:5] = -1
        new.copy_(torch.from_numpy(n.astype(np.int32)))
        want = host.plan(at, n, saw, T)
        graph.replay()
        dev.start, dev.after, dev.seen_after, dev.token_start, dev.rows, dev.pos = start, length, seen, token_start, rows, pos
        compare(host, dev, want)
        at, saw = want[1].astype(np.int64), want[2].astype(np.int64)
        if step % 3 == 0:
            torch.cuda.synchronize()
