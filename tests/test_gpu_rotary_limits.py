"""Rotary positions of as many tokens as a call takes."""
import numpy as np
import pytest
import torch

import token_ref as ref
from paper_2407_18121_amd import binding as ec
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu


def test_most_tokens():
    """2^24 tokens whose heads are too many for two tokens a workgroup: a workgroup each would be 2^32 threads. Nearly all of them are padding, of which nothing is read."""
    T, H, Hkv, D, page, N, at = 1 << 24, 1, 8, 128, 8, 2, [0, 1, 255, (1 << 23) + 1, (1 << 24) - 2, (1 << 24) - 1]
    if torch.cuda.mem_get_info()[0] < 96 << 30:
        pytest.skip("needs 96 GiB of device memory")
    rng = np.random.default_rng(1)
    q, q_out = (torch.empty((T, H, D), device="cuda") for _ in range(2))
    k = torch.empty((T, Hkv, D), device="cuda")
    rows = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    x = quantize(rng.standard_normal((len(at), H + Hkv, D)), "f32")
    q[at], k[at], q_out[at] = to_dev(x[:, :H], "f32"), to_dev(x[:, H:], "f32"), -7.0
    rows[at] = torch.arange(1, 1 + len(at), device="cuda")
    pools = [torch.full((N, Hkv, page, D), 5.0, device="cuda") for _ in range(2)]
    ec.ec_paged_rotary_store(q, k, k, pos, rows, torch.from_numpy(freq).cuda(), q_out, *pools)
    want, tol = ref.turned(x, np.array(at), freq, 1.0, False, "f32")
    assert (np.abs(to_host(q_out[at]) - want[:, :H]) <= tol[:, :H]).all()
    got_k, got_v = (to_host(p).transpose(0, 2, 1, 3).reshape(N * page, Hkv, D) for p in pools)
    assert (np.abs(got_k[1:1 + len(at)] - want[:, H:]) <= tol[:, H:]).all() and np.array_equal(got_v[1:1 + len(at)], x[:, H:].astype(np.float64))
    assert (got_k[1 + len(at):] == 5).all() and (got_v[1 + len(at):] == 5).all() and (got_k[0] == 5).all()
