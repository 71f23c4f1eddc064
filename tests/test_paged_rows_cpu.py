"""The per-row bounds of paged_rows.py see a mistake planted in the oracle: a row's mass left out or added twice."""
import numpy as np
import pytest

import paged_rows as rows
import test_gpu_paged_masses as masses

LONG = [i for i, c in enumerate(masses.CASES) if max(c[-1]) > 250 and len(c[-1]) < 10]


@pytest.mark.parametrize("case", LONG)
def test_mistakes_are_out_of_bounds(case):
    pool, dtype, lens, q, kn, vn, scale = masses.inputs(case)
    _, _, add, tol = rows.step(pool, q.astype(np.float64), kn, vn, lens, [7000] * len(lens), scale, dtype)
    got, here = np.argwhere(add > 0), add > 0
    assert len(got) > 250
    fits = lambda x: rows.outputs_fit(x, pool.mass, tol)  # noqa: E731
    assert fits(pool.mass.astype(np.float32).astype(np.float64)).all()
    seen = ~fits(pool.mass - add) & here
    assert seen.sum() >= 0.99 * here.sum(), "a row left out goes unseen"
    seen = ~fits(pool.mass + add) & here
    assert seen.sum() >= 0.99 * here.sum(), "a row counted twice goes unseen"
