"""The 64-bit reference's distillation gradient against differences of its loss, where the record's
probabilities do not sum to 1 (CPU)."""
import numpy as np
import pytest

import ops_reference as R

RECORDS = {
    "no entries": ([-1, 23, -1, -2, 40], [0.3, 0.2, 0.1, 0.9, 0.15]),
    "entries of probability 0": ([4, 19, 0, 7, 2], [0.0, 0.0, 0.0, 0.0, 0.0]),
    "one entry": ([4, -1, 4, -1, 4], [0.3, 0.2, 0.1, 0.9, 0.15]),
    "more than the whole mass": ([4, 19, -1, 4, 7], [0.8, 0.4, 0.1, 0.9, 0.3]),
    "the whole mass and more in one": ([4, 19, 2, 1, 7], [1.2, 0.1, 0.1, 0.05, 0.05]),
}


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
@pytest.mark.parametrize("record", RECORDS)
def test_gradient_of_a_record_of_any_mass_is_the_derivative(record, tail, T):
    rng = np.random.default_rng(3)
    V, step = 23, 1e-5
    z = rng.normal(size=V) * 2
    ids = np.array(RECORDS[record][0])
    with np.errstate(divide="ignore"):
        lp = np.log(np.array(RECORDS[record][1]))
    g = R.distill_row(z, T, ids, lp, tail)[1]
    for v in range(V):
        hi, lo = z.copy(), z.copy()
        hi[v] += step
        lo[v] -= step
        d = (R.distill_row(hi, T, ids, lp, tail)[0] - R.distill_row(lo, T, ids, lp, tail)[0]) / (2 * step)
        # a central difference: third derivatives (at most 2 here) times step^2, rounding / step
        assert abs(d - g[v]) < 2e-9, v
