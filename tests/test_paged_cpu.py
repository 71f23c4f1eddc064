"""Refusals of the calls on paged caches, and their workspace sizes: nothing is launched."""
import ctypes

import pytest
import torch

from paper_2407_18121_amd import binding as ec
from paper_2407_18121_amd.pipeline import PagedBatch

ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)  # never dereferenced: validation fails first


def _step(fn="ec_paged_decode_step", **other):
    a = dict(q=ONE, k_new=ONE, v_new=ONE, k_pages=ONE, v_pages=ONE, pos_pages=ONE, mass_pages=ONE, table=ONE, len_b=ONE, new_pos_b=ONE, B=2, H=8,
             Hkv=4, G=1, D=128, page=16, n_pages=9, max_pages=4, scale=0.5, dt=1, out=ONE, ws=ONE, ws_bytes=0, stream=None)
    if fn == "ec_paged_decode_step":
        del a["mass_pages"]
    a.update(other)
    return getattr(ec.load(), fn)(*a.values())


def _store(**other):
    a = dict(k=ONE, v=ONE, pos=ONE, mass=ONE, table=ONE, start_b=None, n_rows_b=None, B=2, Hkv=4, G=1, T=8, src_rows=8, D=128, page=16, n_pages=9,
             max_pages=4, dt=1, k_pages=ONE, v_pages=ONE, pos_pages=ONE, mass_pages=ONE, stream=None)
    a.update(other)
    return ec.load().ec_paged_store(*a.values())


def _evict(**other):
    a = dict(k_pages=ONE, v_pages=ONE, pos_pages=ONE, mass_pages=ONE, table=ONE, len_b=ONE, keep_b=ONE, seen_b=ONE, B=2, Hkv=4, G=1, D=128, page=16,
             n_pages=9, max_pages=4, max_evict=10, first=1, recent=5, dt=1, ws=ONE, ws_bytes=0, stream=None)
    a.update(other)
    return ec.load().ec_paged_evict_min(*a.values())


SHAPE = [(dict(B=0), ec.EC_EINVAL), (dict(Hkv=0), ec.EC_EINVAL), (dict(G=2), ec.EC_EINVAL), (dict(D=0), ec.EC_EINVAL), (dict(page=0), ec.EC_EINVAL),
         (dict(page=-16), ec.EC_EINVAL), (dict(n_pages=0), ec.EC_EINVAL), (dict(max_pages=0), ec.EC_EINVAL), (dict(table=None), ec.EC_EINVAL),
         (dict(page=24), ec.EC_EUNSUPPORTED), (dict(page=4), ec.EC_EUNSUPPORTED), (dict(page=512), ec.EC_EUNSUPPORTED),
         (dict(max_pages=1 << 27), ec.EC_EUNSUPPORTED), (dict(n_pages=1 << 28), ec.EC_EUNSUPPORTED), (dict(D=96), ec.EC_EUNSUPPORTED), (dict(dt=2), ec.EC_EUNSUPPORTED),
         (dict(B=20000), ec.EC_EUNSUPPORTED), (dict(B=1, Hkv=65535, H=65535, page=256, dt=0), ec.EC_EUNSUPPORTED), (dict(k_pages=ODD), ec.EC_EUNSUPPORTED), (dict(v_pages=ODD), ec.EC_EUNSUPPORTED)]


@pytest.mark.parametrize("other,status", SHAPE)
def test_shapes_are_refused(other, status):
    for fn in ("ec_paged_decode_step", "ec_paged_decode_score_step"):
        assert _step(fn, **other) == status
    other = {p: x for p, x in other.items() if p != "H"}
    assert _store(**other) == status
    assert _evict(**other) == status


@pytest.mark.parametrize("fn", ["ec_paged_decode_step", "ec_paged_decode_score_step"])
def test_step_refusals(fn):
    for p in ("q", "k_new", "v_new", "k_pages", "v_pages", "len_b", "out"):
        assert _step(fn, **{p: None}) == ec.EC_EINVAL, p
    assert _step(fn, new_pos_b=None) == ec.EC_EINVAL             # positions without the new ones
    assert _step(fn, pos_pages=None, new_pos_b=None) == ec.EC_EWORKSPACE
    assert _step(fn, H=0) == ec.EC_EINVAL
    assert _step(fn, H=6) == ec.EC_EINVAL                        # no multiple of Hkv
    assert _step(fn, H=40000) == ec.EC_EUNSUPPORTED
    for bad in (0.0, -0.5, float("inf"), float("nan")):
        assert _step(fn, scale=bad) == ec.EC_EINVAL
    for p in ("q", "k_new", "v_new", "out"):
        assert _step(fn, **{p: ODD}) == ec.EC_EUNSUPPORTED, p
    code = ec.EC_FN_PAGED_DECODE_STEP if fn == "ec_paged_decode_step" else ec.EC_FN_PAGED_DECODE_SCORE_STEP
    need = ec.ec_workspace_bytes(code, 2, 8, 64, 128, ec.EC_BF16)
    assert need > 0
    assert _step(fn, ws_bytes=need - 1) == ec.EC_EWORKSPACE
    assert _step(fn, ws=None, ws_bytes=need) == ec.EC_EWORKSPACE
    assert _step(fn, ws=ODD, ws_bytes=need) == ec.EC_EWORKSPACE
    if fn == "ec_paged_decode_score_step":
        assert _step(fn, mass_pages=None) == ec.EC_EINVAL


def test_store_refusals():
    assert _store(k=None) == ec.EC_EINVAL
    assert _store(v=None) == ec.EC_EINVAL
    assert _store(k=None, v=None, pos=None, mass=None) == ec.EC_EINVAL   # nothing to store
    assert _store(T=0) == ec.EC_EINVAL
    assert _store(T=9) == ec.EC_EINVAL                                   # more than the source has
    for p in ("k_pages", "v_pages", "pos_pages", "mass_pages"):
        assert _store(**{p: None}) == ec.EC_EINVAL, p
    for p in ("k", "v"):
        assert _store(**{p: ODD}) == ec.EC_EUNSUPPORTED, p


def test_evict_refusals():
    for p in ("k_pages", "v_pages", "mass_pages", "len_b", "keep_b", "pos_pages", "seen_b"):
        assert _evict(**{p: None}) == ec.EC_EINVAL, p
    assert _evict(max_evict=0) == ec.EC_EINVAL
    assert _evict(max_evict=65) == ec.EC_EINVAL                          # more than the slots of a sequence
    for p in ("pos_pages", "mass_pages"):
        assert _evict(**{p: ODD}) == ec.EC_EUNSUPPORTED, p
    assert _evict(first=-1) == ec.EC_EINVAL
    assert _evict(recent=-1) == ec.EC_EINVAL
    assert _evict(seen_b=None, recent=0) == ec.EC_EWORKSPACE
    assert _evict(pos_pages=None, first=0, recent=0) == ec.EC_EWORKSPACE
    need = ec.ec_workspace_bytes(ec.EC_FN_PAGED_EVICT_MIN, 2, 1, 10, 128, ec.EC_BF16)
    assert _evict(ws_bytes=need - 1) == ec.EC_EWORKSPACE
    assert _evict(ws=None, ws_bytes=need) == ec.EC_EWORKSPACE


def test_workspace_sizes():
    assert ec.ec_workspace_bytes(ec.EC_FN_PAGED_STORE, 2, 4, 64, 128, ec.EC_BF16) == 0
    # a step's scores and statistics grow with the slots, a step without scores does not need them
    few, many = (ec.ec_workspace_bytes(ec.EC_FN_PAGED_DECODE_SCORE_STEP, 2, 8, n, 128, ec.EC_BF16) for n in (64, 1 << 20))
    assert many - few >= 2 * 8 * 4 * ((1 << 20) - 64)
    assert (ec.ec_workspace_bytes(ec.EC_FN_PAGED_DECODE_STEP, 2, 8, 64, 128, ec.EC_BF16)
            == ec.ec_workspace_bytes(ec.EC_FN_PAGED_DECODE_STEP, 2, 8, 1 << 20, 128, ec.EC_BF16))
    assert ec.ec_workspace_bytes(ec.EC_FN_PAGED_EVICT_MIN, 3, 2, 100, 64, ec.EC_F32) >= 3 * 2 * 100 * 8
    with pytest.raises(ec.EcError):
        ec.ec_workspace_bytes(ec.EC_FN_PAGED_DECODE_STEP, 2, 8, 64, 96, ec.EC_BF16)


def test_binding_refuses_what_does_not_fit():
    B, H, Hkv, D, N, page, mp = 2, 8, 4, 64, 6, 8, 3
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    q, kn, kp = torch.zeros((B, H, D), dtype=bf), torch.zeros((B, Hkv, D), dtype=bf), torch.zeros((N, Hkv, page, D), dtype=bf)
    pos, mass, table, n = torch.zeros((N, 1, page), dtype=i32), torch.zeros((N, 1, page)), torch.zeros((B, mp), dtype=i32), torch.zeros(B, dtype=i32)
    step = lambda **o: ec.ec_paged_decode_score_step(**{**dict(q=q, k_new=kn, v_new=kn, k_pages=kp, v_pages=kp, pos_pages=pos, mass_pages=mass,  # noqa: E731
                                                               page_table=table, cache_len_b=n, new_pos_b=n, scale=0.1, out=q, ws=None), **o})
    plain = lambda **o: ec.ec_paged_decode_step(**{**dict(q=q, k_new=kn, v_new=kn, k_pages=kp, v_pages=kp, pos_pages=pos, page_table=table,  # noqa: E731
                                                          cache_len_b=n, new_pos_b=n, scale=0.1, out=q, ws=None), **o})
    evict = lambda **o: ec.ec_paged_evict_min(**{**dict(k_pages=kp, v_pages=kp, pos_pages=pos, mass_pages=mass, page_table=table, len_b=n,  # noqa: E731
                                                        keep_b=n, seen_b=n, max_evict=1, protect_first=1, protect_recent=1, ws=None), **o})
    store = lambda **o: ec.ec_paged_store(**{**dict(k=kn[:, :, None].expand(B, Hkv, 5, D).contiguous(), v=kn[:, :, None].expand(B, Hkv, 5, D).contiguous(),  # noqa: E731
                                                    pos=None, mass=None, page_table=table, k_pages=kp, v_pages=kp, pos_pages=None, mass_pages=None), **o})
    for call in (step, plain, evict, store):
        with pytest.raises(ValueError, match="device memory"):       # everything fits: only the device is wrong
            call()
        with pytest.raises(ValueError, match="page_table must be torch.int32"):
            call(page_table=table.long())
        with pytest.raises(ValueError, match="page_table must be"):
            call(page_table=n)
        with pytest.raises(ValueError, match="v_pages must have shape"):
            call(v_pages=kp[:-1])
    for call in (step, plain):
        with pytest.raises(ValueError, match="q must be torch.bfloat16"):
            call(q=q.float())
        with pytest.raises(ValueError, match="k_new must have shape"):
            call(k_new=q)
        with pytest.raises(ValueError, match="cache_len_b must be an int32 tensor"):
            call(cache_len_b=n.long())
        with pytest.raises(ValueError, match="new_pos_b is required"):
            call(new_pos_b=None)
        with pytest.raises(ValueError, match="pos_pages must have shape"):
            call(pos_pages=pos[..., 1:])
    with pytest.raises(ValueError, match="mass_pages is required"):
        step(mass_pages=None)
    with pytest.raises(ValueError, match="score groups"):
        step(mass_pages=torch.zeros((N, 2, page)))
    with pytest.raises(ValueError, match="keep_b must be an int32 tensor"):
        evict(keep_b=n[:1])
    with pytest.raises(ValueError, match="mass_pages must be torch.float32"):
        evict(mass_pages=mass.to(bf))
    with pytest.raises(ValueError, match="go together"):
        store(v=None)
    with pytest.raises(ValueError, match="nothing to store"):
        store(k=None, v=None)
    with pytest.raises(ValueError, match="mass must have shape"):
        store(mass=torch.zeros((B, 1, 4)), mass_pages=mass)
    with pytest.raises(ValueError, match="pos_pages is required"):
        store(pos=torch.zeros((B, 1, 5), dtype=i32))


def test_places_and_pages_of_a_batch():
    """What PagedBatch keeps on the host: pages taken and given back, and what it refuses without changing anything."""
    batch = PagedBatch(1, 3, 4, 2, 64, 16, 8, 3, torch.float32, device="cpu")
    batch.admit([2, 0], [17, 0], [40, 0])
    assert batch.rows == [0, -1, 17] and [len(h) for h in batch.held] == [0, 0, 2] and len(batch.free) == 6
    state = lambda: (list(batch.rows), list(batch.seen), [list(h) for h in batch.held], list(batch.free), batch.table.tolist())
    before = state()
    for places, rows, seen in (([1, 1], [5, 5], [5, 5]), ([-2], [5], [5]), ([3], [5], [5]), ([1], [5, 6], [5, 6]), ([1], [-1], [5]), ([1], [49], [49]),
                               ([2], [5], [5])):
        with pytest.raises(ValueError):
            batch.admit(places, rows, seen)
    x = torch.zeros(1, 2, 16, 64)
    for places in ([2], [-1], [3]):  # 17 rows, but 16 given; no such places
        with pytest.raises(ValueError):
            batch.store(0, places, x, x, torch.zeros(1, 1, 16, dtype=torch.int32), torch.zeros(1, 1, 16))
    for call in (lambda: batch.release(-1), lambda: batch.shrink(-1), batch.end):  # end(): no room has been made for a token
        with pytest.raises(ValueError):
            call()
    assert state() == before
    batch.admit([], [], [])
    batch.begin()
    assert [len(h) for h in batch.held] == [1, 0, 2] and state()[4][0][0] == batch.held[0][0]
    batch.end()
    assert batch.rows == [1, -1, 18] and batch.seen == [1, 0, 41] and batch.len_b.tolist() == [1, -1, 18] and batch.len_after.tolist() == [2, 0, 19]
    batch.release(2)
    assert batch.table[2].tolist() == [-1] * 3 and len(batch.free) == 7


@pytest.mark.parametrize("fn", ["ec_paged_decode_step", "ec_paged_decode_score_step"])
def test_outputs_over_inputs_are_refused(fn):
    code = ec.EC_FN_PAGED_DECODE_STEP if fn == "ec_paged_decode_step" else ec.EC_FN_PAGED_DECODE_SCORE_STEP
    need = ec.ec_workspace_bytes(code, 2, 8, 64, 128, ec.EC_BF16)
    at = {p: 1 << 20 << i for i, p in enumerate(("out", "q", "k_new", "v_new"))}
    for p, rows in (("q", 16), ("k_new", 8), ("v_new", 8)):  # out has 16 rows of 256 bytes
        for off in (0, 16, 15 * 256, -16, -(rows * 256 - 16)):
            x = {k: ctypes.c_void_p(v) for k, v in {**at, p: at["out"] + off}.items()}
            assert _step(fn, ws_bytes=need, **x) == ec.EC_EINVAL, (p, off)
