"""The native half of the binding against its ctypes half for the calls on paged caches, in the manner of test_gpu_fastcall.py: both are bound to
functions that note their arguments and launch nothing."""
import ctypes
import inspect
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from test_gpu_fastcall import _others

pytestmark = pytest.mark.gpu
B, H, HKV, D, N, PAGE, MP, ROWS = 2, 8, 4, 64, 5, 16, 3, 7


def _calls(dt, G):
    t = lambda *s, dtype=dt: torch.zeros(s, dtype=dtype, device="cuda")
    f, i = (lambda *s: t(*s, dtype=torch.float32)), (lambda *s: t(*s, dtype=torch.int32))
    pools = lambda: dict(k_pages=t(N, HKV, PAGE, D), v_pages=t(N, HKV, PAGE, D), pos_pages=i(N, G, PAGE))
    step = lambda: dict(q=t(B, H, D), k_new=t(B, HKV, D), v_new=t(B, HKV, D), **pools(), page_table=i(B, MP), cache_len_b=i(B), new_pos_b=i(B), scale=0.3,
                        out=t(B, H, D), ws=f(40))
    return {
        "paged_store": dict(k=t(B, HKV, ROWS, D), v=t(B, HKV, ROWS, D), pos=i(B, G, ROWS), mass=f(B, G, ROWS), page_table=i(B, MP), **pools(),
                            mass_pages=f(N, G, PAGE), start_b=i(B), n_rows_b=i(B), T=5),
        "paged_decode_step": step(),
        "paged_decode_score_step": dict(step(), mass_pages=f(N, G, PAGE)),
        "paged_evict_min": dict(pools(), mass_pages=f(N, G, PAGE), page_table=i(B, MP), len_b=i(B), keep_b=i(B), seen_b=i(B), max_evict=9,
                                protect_first=1, protect_recent=2, ws=f(40)),
    }


@pytest.fixture
def noted(monkeypatch):
    lib, fast, seen, stubs = ec.load(), ec._fast, [], {}
    assert fast is not None
    for name in ec._FAST_PAGED:
        fn = getattr(lib, "ec_" + name)
        stubs["ec_" + name] = ctypes.CFUNCTYPE(ctypes.c_int, *fn.argtypes)(lambda *a, name=name: seen.append((name, *a)) or 0)
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value

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
    fast.bind_paged(tuple(address(stubs["ec_" + n]) for n in ec._FAST_PAGED))
    monkeypatch.setattr(ec, "_fast", None)
    monkeypatch.setattr(ec, "load", lambda: SimpleNamespace(**stubs))
    yield native, through_ctypes
    fast.bind_paged(tuple(address(getattr(lib, "ec_" + n)) for n in ec._FAST_PAGED))


@pytest.mark.parametrize("name", ec._FAST_PAGED)
@pytest.mark.parametrize("dt,G", [(torch.bfloat16, 1), (torch.float32, HKV)])
def test_usual_calls(noted, name, dt, G):
    """Both halves hand the library the same; none of these calls is left to ctypes."""
    native, through_ctypes = noted
    good = _calls(dt, G)[name]
    usual = [good]
    usual += [dict(good, **{p: None}) for p in ("start_b", "n_rows_b", "T", "seen_b", "ws", "mass") if p in good]
    if name == "paged_store":
        usual += [dict(good, k=None, v=None), dict(good, k=None, v=None, pos=None, k_pages=None, v_pages=None, pos_pages=None),
                  dict(good, pos=None, mass=None, pos_pages=None, mass_pages=None), dict(good, pos=None, pos_pages=None)]
    else:
        usual += [dict(good, pos_pages=None)] if name == "paged_evict_min" else [dict(good, pos_pages=None, new_pos_b=None), dict(good, pos_pages=None)]
    if "scale" in good:
        usual += [dict(good, scale=s) for s in (1.0 / np.sqrt(D), np.float64(0.125), 1, 1e30)]
    for args in usual:
        got = native(name, args)
        assert got is not None and got == through_ctypes(name, args)


@pytest.mark.parametrize("name", ec._FAST_PAGED)
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
        assert refused >= (3 if p == "ws" else 7 if isinstance(x, torch.Tensor) else 1), (p, refused)


def test_number_of_arguments():
    ec.load()
    for name in ec._FAST_PAGED:
        assert getattr(ec._fast, name)() is None
