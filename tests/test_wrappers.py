"""Every Python entry point can be called with fitting arguments: host tensors get as far as the check of where they live, and the one that has
no workspace gives on the device what its sister on a caller's workspace gives."""
import numpy as np
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from util import quantize, to_dev

B, H, HKV, T, D, N, CAP, L, P, PAGE, MP = 2, 4, 2, 6, 64, 5, 9, 7, 3, 8, 3
HOST_ONLY = {"ec_status_string", "ec_workspace_bytes", "ec_evict_index"}


def _calls():
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: t(*s, dtype=torch.int32)  # noqa: E731
    row, kv, cache = t(B, H, D), t(B, H, T, D), t(B, H, CAP, D)
    step = dict(q=row, k_new=row, v_new=row, k_cache=cache, v_cache=cache, pos=i(B, 1, CAP), scale=0.1, out=row)
    ints, freq = dict(cache_len=7, new_pos=11), t(B, 1, CAP)
    pools = dict(k_pages=t(N, HKV, PAGE, D), v_pages=t(N, HKV, PAGE, D), pos_pages=i(N, 1, PAGE))
    paged = dict(q=row, k_new=t(B, HKV, D), v_new=t(B, HKV, D), **pools, page_table=i(B, MP), cache_len_b=i(B), new_pos_b=i(B), scale=0.1, out=row, ws=None)
    prompt = dict(q=kv, k=kv, v=kv, out=kv, lse=t(B, H, T), score=t(B, 1, T), scale=0.1, ws=None)
    merged = dict(k=kv, v=kv, anchor_idx=i(B, 1, N), k_cache=cache, v_cache=cache)
    return {
        "ec_prefill_score": prompt,
        "ec_prefill_score_varlen": dict(prompt, seq_len=i(B)),
        "ec_chunk_score": dict(prompt, k=t(B, H, P + T, D), v=t(B, H, P + T, D), score=t(B, 1, P + T), P=P),
        "ec_select_anchors": dict(score=t(B, 1, T), n_anchor=N, protect_first=1, protect_last=1, anchor_idx=i(B, 1, N)),
        "ec_select_anchors_varlen": dict(score=t(B, 1, T), seq_len=i(B), n_anchor_b=i(B), protect_first=1, protect_last=1, anchor_idx=i(B, 1, N)),
        "ec_merge_compact": merged,
        "ec_merge_compact_varlen": dict(merged, seq_len=i(B), n_anchor_b=i(B)),
        "ec_remerge_compact": dict(merged, k=t(B, H, L + 1, D), v=t(B, H, L + 1, D), L=L),
        "ec_decode_step": dict(step, **ints, evict_idx=2, ws=None),
        "ec_decode_step_shaped": dict(step, **ints, evict_idx=2, ws=None),
        "ec_decode_step_varlen": dict(step, cache_len_b=i(B), evict_idx_b=i(B), new_pos_b=i(B)),
        "ec_decode_score_step": dict(step, **ints, freq=freq, ws=None),
        "ec_decode_score_step_static": dict(step, **ints, freq=freq),
        "ec_evict_min": dict(k_cache=cache, v_cache=cache, pos=None, freq=freq, length=8, protect_first=1, protect_recent=2, victim=i(B, 1)),
        "ec_importance_mean": dict(score=t(B, 1, T), T_new=T),
        "ec_retention_step_varlen": dict(n_seen_b=i(B), cache_len_b=i(B), evict_idx_b=i(B), new_pos_b=i(B), pending_b=i(B), gamma_num=1, gamma_den=2),
        "ec_paged_store": dict(k=t(B, HKV, T, D), v=t(B, HKV, T, D), pos=i(B, 1, T), mass=t(B, 1, T), page_table=i(B, MP), **pools,
                               mass_pages=t(N, 1, PAGE)),
        "ec_paged_decode_step": paged,
        "ec_paged_decode_score_step": dict(paged, mass_pages=t(N, 1, PAGE)),
        "ec_paged_evict_min": dict(pools, mass_pages=t(N, 1, PAGE), page_table=i(B, MP), len_b=i(B), keep_b=i(B), seen_b=i(B), max_evict=9,
                                   protect_first=1, protect_recent=2, ws=None),
    }


def test_every_entry_point_is_here():
    assert set(_calls()) == set(ec.SYMBOLS) - HOST_ONLY


@pytest.mark.parametrize("name", sorted(_calls()))
def test_fitting_host_tensors_are_refused_for_where_they_live(name):
    with pytest.raises(ValueError, match="device memory"):
        getattr(ec, name)(**_calls()[name])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,G", [("bf16", 1), ("f32", H)])
def test_the_call_without_a_workspace(dtype, G):
    rng = np.random.default_rng(5)
    cap, n = 90, 77
    host = [quantize(rng.standard_normal(s), dtype) for s in ((B, H, D),) * 3 + ((B, H, cap, D),) * 2]
    got = []
    for static in (False, True):
        q, kn, vn, kc, vc = (to_dev(x, dtype) for x in host)
        pos, freq, out = torch.zeros(B, G, cap, dtype=torch.int32, device="cuda"), torch.ones(B, G, cap, device="cuda"), torch.empty_like(q)
        if static:
            assert ec.ec_decode_score_step_static(q, kn, vn, kc, vc, pos, freq, n, 4242, 0.125, out) == ec.EC_OK
        else:
            ec.ec_decode_score_step(q, kn, vn, kc, vc, pos, freq, n, 4242, 0.125, out, ec.new_workspace(ec.EC_FN_DECODE_SCORE_STEP, B, H, cap, D, ec.dtype_code(q)))
        got.append((out, kc, vc, pos, freq))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and int(got[1][3][0, 0, n]) == 4242
