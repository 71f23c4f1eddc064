"""Sizes on the host: a workspace for many evictions serves fewer, and a batch that runs out of pages changes nothing."""
import pytest
import torch

from paper_2407_18121_amd import binding as ec
from paper_2407_18121_amd.pipeline import PagedBatch


@pytest.mark.parametrize("B,G", [(1, 1), (4, 8), (2, 40), (64, 1), (100, 1)])
def test_an_eviction_workspace_serves_every_smaller_eviction(B, G):
    sizes = [ec.ec_workspace_bytes(ec.EC_FN_PAGED_EVICT_MIN, B, G, n, 128, ec.EC_BF16) for n in (1, 2, 3, 40, 127, 128, 129, 130, 1000, 1 << 20)]
    assert sizes == sorted(sizes)


def test_a_batch_out_of_pages_is_left_as_it_was():
    batch = PagedBatch(1, 3, 4, 2, 64, 16, 5, 3, torch.float32, device="cpu")
    batch.admit([0, 1, 2], [16, 32, 5], [16, 32, 5])  # one page is free, two sequences need one
    state = lambda: (list(batch.rows), [list(h) for h in batch.held], list(batch.free), batch.table.tolist(), batch.numbers.tolist())  # noqa: E731
    before = state()
    with pytest.raises(ValueError, match="are free"):
        batch.begin()
    assert state() == before and batch.changes == {}
    batch.release(2)
    batch.begin()
    batch.end()
    assert batch.rows == [17, 33, -1] and batch.free == [] and batch.table.tolist() == [h + [-1] * (3 - len(h)) for h in batch.held]
    assert batch.numbers.tolist() == [[17, 33, -1], [18, 34, 0], [17, 33, 0], [18, 34, 1]]
