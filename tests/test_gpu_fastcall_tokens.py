"""The native half of the binding against its ctypes half for the calls on several new tokens at a time, in the manner of test_gpu_fastcall_paged.py: both are
bound to functions that note their arguments and launch nothing."""
import ctypes
import inspect
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from test_gpu_fastcall import _others

pytestmark = pytest.mark.gpu
B, T, H, HKV, D, N, PAGE, MP = 2, 6, 8, 4, 64, 5, 16, 3


def _calls(dt, G):
    t = lambda *s, dtype=dt: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    f, i = (lambda *s: t(*s, dtype=torch.float32)), (lambda *s: t(*s, dtype=torch.int32))
    pools = lambda: dict(k_pages=t(N, HKV, PAGE, D), v_pages=t(N, HKV, PAGE, D))  # noqa: E731
    part = t(T, (H + 2 * HKV) * D)
    return {
        "paged_plan": dict(len_b=i(B), new_b=i(B), page_table=i(B, MP), held_b=i(B), free_pages=i(N), n_free=i(1), page=PAGE, start_b=i(B), len_after_b=i(B),
                           token_start=i(B + 1), rows=t(T, dtype=torch.int64), pos=i(T), seen_b=i(B), seen_after_b=i(B), T=9),
        "paged_rotary_store": dict(q=part[:, :H * D].view(T, H, D), k=part[:, H * D:(H + HKV) * D].view(T, HKV, D), v=t(T, HKV, D), pos=i(T),
                                   rows=t(T, dtype=torch.int64), freq=f(10), q_out=t(T, H, D), **pools(), pos_pages=i(N, G, PAGE), mass_pages=f(N, G, PAGE),
                                   interleaved=False, mscale=1.5),
        "paged_chunk_step": dict(q=t(T, H, D), **pools(), page_table=i(B, MP), start_b=i(B), token_start=i(B + 1), scale=0.3, out=t(T, H, D), ws=f(40), lse=f(T, H)),
    }


@pytest.fixture
def noted(monkeypatch):
    lib, fast, seen, stubs = ec.load(), ec._fast, [], {}
    assert fast is not None
    for name in ec._FAST_TOKENS:
        fn = getattr(lib, "ec_" + name)
        stubs["ec_" + name] = ctypes.CFUNCTYPE(ctypes.c_int, *fn.argtypes)(lambda *a, name=name: seen.append((name, *a)) or 0)
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731

    def native(name, args):
        order = [p for p in inspect.signature(getattr(ec, "ec_" + name)).parameters if p != "check"]
        rc = getattr(fast, name)(*(args[p] for p in order))
        assert rc == (0 if seen else None)
        return seen.pop() if seen else None

    def through_ctypes(name, args):
        try:
            getattr(ec, "ec_" + name)(**args)
        except Exception as e:
            assert not seen
            return e
        return seen.pop()
    fast.bind_tokens(tuple(address(stubs["ec_" + n]) for n in ec._FAST_TOKENS))
    monkeypatch.setattr(ec, "_fast", None)
    monkeypatch.setattr(ec, "load", lambda: SimpleNamespace(**stubs))
    yield native, through_ctypes
    fast.bind_tokens(tuple(address(getattr(lib, "ec_" + n)) for n in ec._FAST_TOKENS))


@pytest.mark.parametrize("name", ec._FAST_TOKENS)
@pytest.mark.parametrize("dt,G", [(torch.bfloat16, 1), (torch.float32, HKV)])
def test_usual_calls(noted, name, dt, G):
    """Both halves hand the library the same; none of these calls is left to ctypes."""
    native, through_ctypes = noted
    good = _calls(dt, G)[name]
    usual = [good] + [dict(good, **{p: None}) for p in ("rows", "pos", "seen_b", "seen_after_b", "pos_pages", "mass_pages", "lse", "ws") if p in good
                      and not (name == "paged_rotary_store" and p in ("rows", "pos"))]
    if name == "paged_plan":
        usual += [dict(good, rows=None, pos=None), dict(good, T=None)]
    if name == "paged_rotary_store":
        usual += [dict(good, pos_pages=None, mass_pages=None), dict(good, interleaved=True), dict(good, q=good["q"].contiguous())]
        one = lambda x: x[:1]  # noqa: E731  a single token, whose distance to the next is nobody's
        usual += [dict(good, **{p: one(good[p]) for p in ("q", "k", "v", "pos", "rows", "q_out")})]
    for p in ("scale", "mscale"):
        if p in good:
            usual += [dict(good, **{p: s}) for s in (1.0 / np.sqrt(D), np.float64(0.125), 1, 1e30)]
    for args in usual:
        got = native(name, args)
        assert got is not None and got == through_ctypes(name, args)


@pytest.mark.parametrize("name", ec._FAST_TOKENS)
@pytest.mark.parametrize("dt,G", [(torch.bfloat16, 1), (torch.float32, HKV)])
def test_every_argument_replaced(noted, name, dt, G):
    """Whatever the ctypes half words an error about, the native half leaves to it; what it takes itself reaches the library alike."""
    native, through_ctypes = noted
    good = _calls(dt, G)[name]
    for p, x in good.items():
        refused = 0
        for other in _others(x):
            args = dict(good, **{p: other})
            got, want = native(name, args), through_ctypes(name, args)
            if isinstance(want, Exception):
                assert got is None, (p, other)
                refused += 1
            elif got is not None:
                assert repr(got) == repr(want), (p, other)  # a scale may be NaN
        assert refused >= (0 if p in ("T", "interleaved") else 3 if p in ("ws", "freq", "free_pages") else 5 if isinstance(x, torch.Tensor) else 1), (p, refused)


def test_number_of_arguments():
    ec.load()
    for name in ec._FAST_TOKENS:
        assert getattr(ec._fast, name)() is None
