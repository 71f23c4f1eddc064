"""Refusals of the calls on several new tokens over paged caches, and their workspace sizes: nothing is launched."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from paper_2407_18121_amd.pipeline import rotary_frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
at = lambda n: ctypes.c_void_p(n << 32)  # noqa: E731  far apart, never dereferenced: validation fails first
ODD = ctypes.c_void_p((50 << 32) + 8)
INF, NAN = float("inf"), float("nan")


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "ec_tokens.h")).read()
    declared = set(re.findall(r"\bint (ec_[a-z_]+)\(", header))
    assert declared == set(ec.TOKEN_SYMBOLS)
    for name in declared:
        assert hasattr(ctypes.CDLL(ec.LIB_PATH), name), name


def _plan(**other):
    a = dict(len_b=at(1), new_b=at(2), seen_b=at(3), table=at(4), held_b=at(5), free=at(6), n_free=at(7), B=4, T=64, page=16, n_pages=9, max_pages=4,
             start_b=at(8), len_after=at(9), seen_after=at(10), token_start=at(11), rows=at(12), pos=at(13), stream=None)
    a.update(other)
    return ec.load().ec_paged_plan(*a.values())


def _rotary(**other):
    a = dict(q=at(1), k=at(2), v=at(3), q_step=512, k_step=256, v_step=256, pos=at(4), rows=at(5), freq=at(6), mscale=1.0, rot=128, pairing=0, T=8, H=4, Hkv=2,
             G=1, D=128, page=16, n_pages=9, dt=1, q_out=at(7), k_pages=at(8), v_pages=at(9), pos_pages=at(10), mass_pages=at(11), stream=None)
    a.update(other)
    return ec.load().ec_paged_rotary_store(*a.values())


def _chunk(**other):
    a = dict(q=at(1), k_pages=at(2), v_pages=at(3), table=at(4), start_b=at(5), token_start=at(6), B=2, T=8, H=4, Hkv=2, D=128, page=16, n_pages=9, max_pages=4,
             scale=0.5, dt=1, out=at(7), lse=at(8), ws=at(9), ws_bytes=0, stream=None)
    a.update(other)
    return ec.load().ec_paged_chunk_step(*a.values())


def test_plan_refusals():
    for p in ("len_b", "new_b", "table", "held_b", "free", "n_free", "start_b", "len_after", "token_start", "seen_b", "seen_after"):
        assert _plan(**{p: None}) == ec.EC_EINVAL, p
    for p in ("B", "T", "page", "n_pages", "max_pages"):
        assert _plan(**{p: 0}) == ec.EC_EINVAL, p
    for other in (dict(page=24), dict(page=4), dict(page=512), dict(max_pages=1 << 27), dict(n_pages=1 << 28), dict(B=8193), dict(T=(1 << 24) + 1)):
        assert _plan(**other) == ec.EC_EUNSUPPORTED, other
    # arrays that are one another's, or overlap by an entry
    near = lambda n, off: ctypes.c_void_p((n << 32) + off)  # noqa: E731
    for other in (dict(start_b=at(1)), dict(len_after=near(1, 12)), dict(len_after=at(2)), dict(seen_after=at(1)), dict(seen_after=near(3, 4)), dict(pos=near(12, 508)),
                  dict(token_start=near(8, 12)), dict(held_b=at(1)), dict(free=near(4, 60)), dict(n_free=near(6, 32)), dict(rows=at(2)), dict(table=at(2))):
        assert _plan(**other) == ec.EC_EINVAL, other


def test_rotary_refusals():
    for p in ("q", "k", "v", "pos", "rows", "freq", "q_out", "k_pages", "v_pages"):
        assert _rotary(**{p: None}) == ec.EC_EINVAL, p
    for other in (dict(T=0), dict(H=0), dict(Hkv=0), dict(G=3), dict(page=0), dict(n_pages=0), dict(rot=0), dict(rot=7), dict(rot=130), dict(rot=-2), dict(pairing=2),
                  dict(mscale=INF), dict(mscale=NAN), dict(q_step=511), dict(k_step=248), dict(v_step=0), dict(q_step=-512), dict(q_out=at(1)),
                  dict(q_out=ctypes.c_void_p((2 << 32) + 7 * 512)), dict(q_out=ctypes.c_void_p((3 << 32) - 16))):
        assert _rotary(**other) == ec.EC_EINVAL, other
    for other in (dict(D=96, rot=96), dict(dt=2), dict(page=24), dict(n_pages=1 << 28), dict(H=65536, q_step=1 << 23), dict(T=(1 << 24) + 1), dict(T=1 << 24, H=65, q_step=8320),
                  dict(q_step=516), dict(k_step=1 << 41), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(q_out=ODD), dict(k_pages=ODD), dict(v_pages=ODD)):
        assert _rotary(**other) == ec.EC_EUNSUPPORTED, other


def test_chunk_refusals():
    for p in ("q", "k_pages", "v_pages", "table", "start_b", "token_start", "out"):
        assert _chunk(**{p: None}) == ec.EC_EINVAL, p
    for other in (dict(B=0), dict(T=0), dict(H=0), dict(Hkv=0), dict(H=5), dict(page=0), dict(n_pages=0), dict(max_pages=0), dict(scale=0.0), dict(scale=-1.0),
                  dict(scale=INF), dict(scale=NAN)):
        assert _chunk(**other) == ec.EC_EINVAL, other
    for other in (dict(D=96), dict(dt=2), dict(page=24), dict(max_pages=1 << 27), dict(n_pages=1 << 28), dict(B=40000), dict(H=65538), dict(T=(1 << 24) + 1),
                  dict(T=1 << 24, H=66), dict(q=ODD), dict(out=ODD), dict(k_pages=ODD), dict(v_pages=ODD)):
        assert _chunk(**other) == ec.EC_EUNSUPPORTED, other
    need = ec.ec_workspace_bytes(ec.EC_FN_PAGED_CHUNK_STEP, 2, 4, 8, 128, ec.EC_BF16)
    assert need > 0
    assert _chunk(ws_bytes=need - 1) == ec.EC_EWORKSPACE
    assert _chunk(ws=None, ws_bytes=need) == ec.EC_EWORKSPACE
    assert _chunk(ws=ODD, ws_bytes=need) == ec.EC_EWORKSPACE
    for other in (dict(out=at(1)), dict(out=ctypes.c_void_p((1 << 32) + 8176)), dict(lse=at(1)), dict(lse=at(7))):
        assert _chunk(ws_bytes=need, **other) == ec.EC_EINVAL, other


def test_workspaces():
    for fn in (ec.EC_FN_PAGED_PLAN, ec.EC_FN_PAGED_ROTARY_STORE):
        assert ec.ec_workspace_bytes(fn, 4, 8, 100, 128, ec.EC_BF16) == 0
    size = lambda T, H, D=128: ec.ec_workspace_bytes(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, T, D, ec.EC_BF16)  # noqa: E731
    assert size(1, 8) <= size(100, 8) <= size(1 << 20, 8) == size(1 << 24, 64) and size(100, 8, 64) < size(100, 8)
    for D, dt, T, H in ((96, ec.EC_BF16, 1, 1), (64, 2, 1, 1), (64, ec.EC_F32, (1 << 24) + 1, 1), (64, ec.EC_F32, 1 << 24, 65)):
        with pytest.raises(ec.EcError):
            ec.ec_workspace_bytes(ec.EC_FN_PAGED_CHUNK_STEP, 1, H, T, D, dt)


def _calls():
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: t(*s, dtype=torch.int32)  # noqa: E731
    B, T, H, Hkv, D, N, page = 2, 6, 4, 2, 64, 5, 8
    pools = dict(k_pages=t(N, Hkv, page, D), v_pages=t(N, Hkv, page, D))
    return {
        "ec_paged_plan": dict(len_b=i(B), new_b=i(B), page_table=i(B, 3), held_b=i(B), free_pages=i(N), n_free=i(1), page=page, start_b=i(B), len_after_b=i(B),
                              token_start=i(B + 1), rows=t(T, dtype=torch.int64), pos=i(T), seen_b=i(B), seen_after_b=i(B)),
        "ec_paged_rotary_store": dict(q=t(T, H, D), k=t(T, Hkv, D), v=t(T, Hkv, D), pos=i(T), rows=t(T, dtype=torch.int64), freq=t(16), q_out=t(T, H, D), **pools,
                                      pos_pages=i(N, 1, page), mass_pages=t(N, 1, page)),
        "ec_paged_chunk_step": dict(q=t(T, H, D), **pools, page_table=i(B, 3), start_b=i(B), token_start=i(B + 1), scale=0.1, out=t(T, H, D), ws=None, lse=t(T, H)),
    }


@pytest.mark.parametrize("name", sorted(_calls()))
def test_python_refusals(name):
    """Fitting host tensors get as far as the check of where they live; each of a wrong type or shape is named."""
    good = _calls()[name]
    assert set(_calls()) == set(ec.TOKEN_SYMBOLS)
    with pytest.raises(ValueError, match="device memory"):
        getattr(ec, name)(**good)
    sizes = {"freq"} | ({"rows", "pos", "free_pages"} if name == "ec_paged_plan" else set())  # what they hold says how much there is
    for p, x in good.items():
        if not isinstance(x, torch.Tensor):
            continue
        with pytest.raises((ValueError, TypeError)):
            getattr(ec, name)(**dict(good, **{p: x.to(torch.float64)}))
        if p not in sizes:
            with pytest.raises(ValueError):
                getattr(ec, name)(**dict(good, **{p: torch.zeros([n + 1 for n in x.shape], dtype=x.dtype)}))


def test_python_refusals_of_layout():
    good = _calls()["ec_paged_rotary_store"]
    for p in ("q", "k", "v"):
        x = good[p]
        for bad in (x.transpose(1, 2).contiguous().transpose(1, 2), torch.zeros(x.shape[0], x.shape[1], 2 * x.shape[2])[..., ::2],
                    torch.zeros(x.shape[0], 2 * x.shape[1], x.shape[2])[:, ::2]):
            with pytest.raises(ValueError, match="dense"):
                ec.ec_paged_rotary_store(**dict(good, **{p: bad}))
    with pytest.raises(ValueError, match="T is needed"):
        ec.ec_paged_plan(**dict(_calls()["ec_paged_plan"], rows=None, pos=None))


@pytest.mark.parametrize("rot", [2, 22, 64, 128])
def test_frequencies(rot):
    """The three ways to stretch a context, pair by pair; an fp32 number is half a step off."""
    i = np.arange(rot // 2)
    plain = 10000.0 ** (-2.0 * i / rot)
    near = lambda got, want: np.all(np.abs(got[0].numpy() - want) <= np.abs(want) * 2.0 ** -24 * 1.0001)  # noqa: E731
    f = lambda *a, **k: rotary_frequencies(rot, *a, **k, device="cpu")  # noqa: E731
    assert near(f(), plain) and f()[1] == 1.0 and f()[0].dtype == torch.float32
    assert near(f(500000.0), 500000.0 ** (-2.0 * i / rot))
    assert near(f(factor=8.0), plain / 8)
    if rot > 2:
        raised = f(factor=8.0, kind="base")
        assert near(raised, (10000.0 * 8.0 ** (rot / (rot - 2))) ** (-2.0 * i / rot)) and raised[1] == 1.0
        assert raised[0][0] == 1.0 and abs(float(raised[0][-1]) * 8 / plain[-1] - 1) < 1e-6
    got, mscale = f(factor=8.0, kind="parts", trained=2048)
    turns = plain * 2048 / (2 * np.pi)
    want = [w if t > 32 else w / 8 if t < 1 else w * (t - 1) / 31 + w / 8 * (32 - t) / 31 for w, t in zip(plain, turns)]
    assert np.all(np.abs(got.numpy() - want) <= np.abs(want) * 2.0 ** -23) and abs(mscale - (0.1 * np.log(8) + 1)) < 1e-15


def test_frequency_refusals():
    for bad in (dict(rot=3), dict(rot=0), dict(rot=64, factor=0.5), dict(rot=64, kind="other"), dict(rot=2, kind="base", factor=2.0)):
        with pytest.raises(ValueError):
            rotary_frequencies(**bad, device="cpu")
