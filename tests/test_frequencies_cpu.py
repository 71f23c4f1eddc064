"""Arguments of rotary_frequencies that give no frequencies are refused."""
import math

import pytest

from paper_2407_18121_amd.pipeline import rotary_frequencies

NAN = float("nan")


@pytest.mark.parametrize("bad", [dict(base=0.0), dict(base=-10.0), dict(base=NAN), dict(base=math.inf), dict(factor=NAN), dict(factor=math.inf),
                                 dict(kind="parts", low=4.0, high=4.0), dict(kind="parts", low=8.0, high=4.0), dict(kind="parts", low=NAN), dict(kind="parts", trained=0)])
def test_refusals(bad):
    with pytest.raises(ValueError):
        rotary_frequencies(64, device="cpu", **bad)


def test_every_frequency_is_a_number():
    for kind in ("linear", "base", "parts"):
        freq, mscale = rotary_frequencies(64, base=1e-3, factor=1e6, kind=kind, trained=1, low=0.0, high=1e-3, device="cpu")
        assert freq.isfinite().all() and math.isfinite(mscale)
