"""The formulas of the worker's operators against differences (CPU): the gradients of the
64-bit reference are the derivatives of its own losses.  And the calls that fail without a
device."""
import ctypes as C

import numpy as np
import pytest

import ops_reference as R
from paper_1805_08469_amd import gem as G


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
def test_distill_gradient_is_the_derivative(tail, T):
    rng = np.random.default_rng(3)
    V, k = 23, 5
    z = rng.normal(size=V) * 2
    ids = np.array([4, 19, -1, 4, 7])
    lp = np.log(np.array([0.3, 0.2, 0.1, 0.9, 0.15]))
    g = R.distill_row(z, T, ids, lp, tail)[1]
    step = 1e-5
    for v in range(V):
        hi, lo = z.copy(), z.copy()
        hi[v] += step
        lo[v] -= step
        d = (R.distill_row(hi, T, ids, lp, tail)[0] - R.distill_row(lo, T, ids, lp, tail)[0]) / (2 * step)
        # a central difference: third derivatives (at most 1 here) times step^2, rounding / step
        assert abs(d - g[v]) < 1e-9, v


def test_scan_gradients_are_the_derivatives():
    rng = np.random.default_rng(4)
    T, D = 9, 3
    x, g, dy = rng.normal(size=(3, T, D))
    h0, dl = rng.normal(size=(2, D))
    out = R.scan(x, g, h0, dy, dl)

    def value(x, g, h0):
        o = R.scan(x, g, h0, None, None)
        return (o["y"] * dy).sum() + (o["h_last"] * dl).sum()

    step = 1e-5
    for which, grad in ((0, out["dx"]), (1, out["dg"]), (2, out["dh0"])):
        for i in np.ndindex(grad.shape):
            hi, lo = [x.copy(), g.copy(), h0.copy()], [x.copy(), g.copy(), h0.copy()]
            hi[which][i] += step
            lo[which][i] -= step
            assert abs((value(*hi) - value(*lo)) / (2 * step) - grad[i]) < 1e-8


def test_calls_without_a_handle_fail_cleanly():
    L = G.lib()
    assert L.gem_ops_destroy(None) == G.GEM_EINVAL
    assert L.gem_ops_create(0, None, None) == G.GEM_EINVAL
    out = C.c_void_p()
    assert L.gem_ops_create(-1, None, C.byref(out)) == G.GEM_EINVAL
    assert L.gem_token_scores(None, None, None, 0, 0, None) == G.GEM_EINVAL
    assert L.gem_distill_loss(None, None, None, None, None) == G.GEM_EINVAL
    assert L.gem_distill_grad(None, None, None, None, None, None, 0) == G.GEM_EINVAL
    assert L.gem_scan_forward(None, None, None, 0, None, None) == G.GEM_EINVAL
    assert L.gem_scan_backward(None, None, None, None, 0, None, None, 0, None, 0, None) == G.GEM_EINVAL


def test_sizes_of_scratch_and_states():
    L = G.lib()
    n = C.c_int64()
    assert L.gem_scan_scratch(10, 10, None) == G.GEM_EINVAL
    assert L.gem_scan_scratch(-1, 10, C.byref(n)) == G.GEM_EINVAL
    assert L.gem_scan_scratch(10, 0, C.byref(n)) == G.GEM_EINVAL
    assert L.gem_scan_scratch(2**31, 1, C.byref(n)) == G.GEM_EINVAL
    assert L.gem_scan_state_rows(-1, C.byref(n)) == G.GEM_EINVAL
    assert G.gem_scan_scratch(0, 1) == 0
    assert G.gem_scan_state_rows(0) == 0 and G.gem_scan_state_rows(1) == 1
    rows = [G.gem_scan_state_rows(t) for t in (1, 1000, 100000)]
    assert rows == sorted(rows) and rows[-1] <= 100000


def test_limits_match_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gem.h")).read()
    assert int(re.search(r"#define GEM_TOP_MAX (\d+)", text).group(1)) == G.GEM_TOP_MAX
    assert 1 << int(re.search(r"#define GEM_VOCAB_MAX \(1 << (\d+)\)", text).group(1)) == G.GEM_VOCAB_MAX
