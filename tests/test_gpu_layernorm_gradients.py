"""Gradients of norms whose rows lie far from zero or are tiny: what cancels in the formula cancels before it is rounded, and no
intermediate leaves the range of fp32 where the result does not.  Tolerances: those of tests/test_gpu_layernorm.py, which count the formula's own
roundings and nothing of the rows' mean."""

import numpy as np
import pytest

from oracle import step as O
from tests.test_gpu_layernorm import case, check_bwd, host, run_bwd, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [100.0, 1000.0, 8000.0])
@pytest.mark.parametrize("d,T", [(64, 9), (1365, 300), (4096, 3), (4096, 400), (8192, 30), (16384, 20), (20000, 5)])
def test_gradients_of_rows_far_from_zero(d, T, offset):
    """dy partly along the normalised row, so that its part along the row is of the gradient's size."""
    rng = np.random.default_rng(d)
    c = case(d + T, T, d, O.LAYER, False, False, False, bias=False)
    z = rng.standard_normal((T, d))
    c["x"] = up((z + offset).astype(np.float32))
    dy = up((1e-2 * (z + rng.standard_normal((T, d)))).astype(np.float32))
    for dh in (None, up((1e-2 * rng.standard_normal((T, d))).astype(np.float32))):
        check_bwd(c, run_bwd(c, dy, dh), dy, dh)


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("d", [63, 96, 2730, 4096, 18000])
def test_gradients_of_tiny_rows(d, kind):
    """rstd up to 1e19: dx is a number of fp32, the square of rstd times a gradient is not."""
    for x16 in (False, True):
        c = case(d, 6, d, kind, x16, x16, False, bias=False)
        rng = np.random.default_rng(d)
        z = rng.standard_normal((6, d))
        c["x"] = up((1e-19 * z).astype(np.float32), x16)
        dy = up((300.0 * (z + rng.standard_normal((6, d)))).astype(np.float32))
        mean, rstd = up(np.zeros(6, np.float32)), up(np.full(6, 9e18, np.float32))
        got = run_bwd(c, dy, None, mean=mean, rstd=rstd)
        check_bwd(c, got, dy, None)
        assert np.isfinite(host(got["dx"])).all()
