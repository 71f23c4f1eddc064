"""Sizes of paged calls that nothing is launched for: a workspace for many evictions serves fewer."""
import pytest

from paper_2407_18121_amd import binding as ec


@pytest.mark.parametrize("B,G", [(1, 1), (4, 8), (2, 40), (64, 1), (100, 1)])
def test_an_eviction_workspace_serves_every_smaller_eviction(B, G):
    sizes = [ec.ec_workspace_bytes(ec.EC_FN_PAGED_EVICT_MIN, B, G, n, 128, ec.EC_BF16) for n in (1, 2, 3, 40, 127, 128, 129, 130, 1000, 1 << 20)]
    assert sizes == sorted(sizes)
