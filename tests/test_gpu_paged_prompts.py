"""PagedTokens: compressed prompts that come in as rows when pages are short. What is refused takes no part in any later step."""
import numpy as np
import pytest
import torch

import paged_ref
import token_ref as ref
from paper_2407_18121_amd.pipeline import PagedTokens, rotary_frequencies
from util import quantize, to_dev, to_host

pytestmark = pytest.mark.gpu
H, Hkv, D, PAGE, T = 4, 2, 64, 16, 40


def batch_of(n_pages, places=4, max_pages=4):
    freq, mscale = rotary_frequencies(D)
    return PagedTokens(1, places, T, H, Hkv, D, PAGE, n_pages, max_pages, torch.bfloat16, freq, mscale)


def step(batch, rng, news):
    """One step; what attention of it is defined to be, from the pools as they are, and what came out."""
    q, k, v = (to_dev(quantize(rng.standard_normal((T, n, D)), "bf16"), "bf16") for n in (H, Hkv, Hkv))
    batch.new_b.copy_(torch.tensor(news, dtype=torch.int32))
    batch.begin()
    out = torch.full_like(q, 5.5)
    batch.attend(0, q, k, v, D ** -0.5, out)
    pool = paged_ref.Pool(to_host(batch.k_pages[0]), to_host(batch.v_pages[0]), np.zeros((1, 1, 1)), np.zeros((1, 1, 1)), batch.table.cpu().numpy())
    n = sum(news)
    want, tol, _, _ = ref.chunk(pool, to_host(batch.turned), batch.start_b.tolist(), batch.token_start.tolist(), D ** -0.5, "bf16")
    got = to_host(out)[:n]
    assert (np.abs(got - want[:n]) <= tol[:n]).all()
    return got


def holds(batch, place, k):
    s = np.arange(k.shape[2])
    return np.array_equal(to_host(batch.k_pages[0])[batch.table[place].cpu().numpy()[s // PAGE], :, s % PAGE], to_host(k[0]).transpose(1, 0, 2))


def rows_of(rng, n, count=1):
    k, v = (to_dev(quantize(rng.standard_normal((count, Hkv, n, D)), "bf16"), "bf16") for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32, device="cuda").expand(count, 1, n).contiguous()
    return k, v, pos, torch.ones(count, 1, n, device="cuda")


def test_a_prompt_that_finds_no_pages_stays_out():
    """Its rows were never stored: when pages come free later nothing attends to what another sequence left in them."""
    rng = np.random.default_rng(1)
    batch = batch_of(6)
    batch.admit([0])
    step(batch, rng, [40, 0, 0, 0])       # three of six pages
    batch.admit([3])
    step(batch, rng, [0, 0, 0, 20])       # two more
    with pytest.raises(ValueError, match="too few free pages"):
        batch.admit([1], [33], [100])     # three, but one is free
    assert batch.len_b.tolist() == [40, -1, -1, 20] and int(batch.n_free) == 1
    with pytest.raises(ValueError, match="not admitted with rows"):
        batch.store(0, [1], *rows_of(rng, 33))
    batch.release([0])
    got = step(batch, rng, [0, 2, 0, 1])  # pages are there now
    assert batch.start_b.tolist() == [-1, -1, -1, 20] and not got[:2].any() and got[2].any()
    assert batch.rows[:2].tolist() == [-1, -1] and batch.len_b.tolist() == [-1, -1, -1, 21] and int(batch.n_free) == 4
    batch.admit([1], [33], [100])         # and the prompt comes in
    k, v, pos, mass = rows_of(rng, 33)
    batch.store(0, [1], k, v, pos, mass)
    got = step(batch, rng, [0, 2, 0, 1])
    assert batch.start_b.tolist() == [-1, 33, -1, 21] and batch.seen_b.tolist() == [0, 102, 0, 22] and got[:2].any()
    assert holds(batch, 1, k)


def test_all_prompts_of_a_call_come_in_or_none():
    rng = np.random.default_rng(2)
    batch = batch_of(5)
    with pytest.raises(ValueError, match=r"\[2\]"):
        batch.admit([0, 2], [16, 65], [1, 1])  # five pages, but a table has four
    with pytest.raises(ValueError, match=r"\[2\]"):
        batch.admit([0, 2], [33, 33], [1, 1])  # three and three of five
    assert batch.len_b.tolist() == [-1] * 4 and batch.seen_b.tolist() == [0] * 4
    step(batch, rng, [1, 0, 1, 0])
    assert batch.start_b.tolist() == [-1] * 4 and int(batch.n_free) == 5 and sorted(batch.free_pages.tolist()) == list(range(5))


def test_pages_released_before_serve_a_prompt_at_once():
    rng = np.random.default_rng(3)
    batch = batch_of(4)
    batch.admit([2])
    step(batch, rng, [0, 0, 40, 0])
    batch.release([2])
    batch.admit([1, 0], [33, 0], [50, 0])
    k, v, pos, mass = rows_of(rng, 33)
    batch.store(0, [1], k, v, pos, mass)
    assert holds(batch, 1, k)
    assert batch.start_b.tolist() == [-1, -1, 0, -1]  # of the step that has run: a new one is begun by begin()
    step(batch, rng, [3, 1, 0, 0])
    assert batch.start_b.tolist() == [0, 33, -1, -1] and batch.pos[:4].tolist() == [0, 1, 2, 50] and int(batch.n_free) == 0
