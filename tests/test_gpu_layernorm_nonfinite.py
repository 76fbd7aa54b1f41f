"""Rows that hold infinities or NaN, or whose squares leave fp32, come out of every form of the norm as the formula has them: mean, rstd and y."""

import numpy as np
import pytest

from oracle import step as O
from tests.test_gpu_layernorm import case, host, run_fwd, up

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("x16", [False, True])
@pytest.mark.parametrize("d", [7, 64, 120, 250, 256, 300, 1000, 1024, 2730, 4096, 5001, 8192, 16384, 20000])
def test_rows_that_are_not_finite(d, x16, kind):
    from paper_2509_13232_b200 import binding as B
    for T, residual in ((9, False), (9, True), (170, False)):
        c = case(d, T, d, kind, x16, False, False, residual=residual)
        x = host(c["x"]).astype(np.float32)
        x[1, 0], x[2, d - 1], x[3, d // 2], x[4, d // 3] = INF, -INF, NAN, INF
        x[5, 0], x[5, d - 1] = INF, -INF
        x[6], x[7] = 1e25, INF
        c["x"] = up(x, x16)
        got = run_fwd(c)
        assert got["status"] == B.DEV_NONFINITE
        h = host(got["h"] if residual else c["x"])
        with np.errstate(invalid="ignore", over="ignore"):
            mean = h.mean(axis=1) if kind == O.LAYER else np.zeros(T)
            m2 = ((h - mean[:, None])**2).mean(axis=1)
            if kind == O.RMS:
                m2[6] = INF                                       # (1e50 is no number of fp32)
            rstd = 1.0 / np.sqrt(m2 + 1e-6)
            y = (h - mean[:, None]) * rstd[:, None] * host(c["weight"]) + host(c["bias"])
        if kind == O.LAYER:
            np.testing.assert_allclose(host(got["mean"]), mean, rtol=1e-4, atol=1e-4)
        live = [i for i in range(T) if kind == O.RMS or i != 6]   # a constant row of 1e25: what its mean is rounded by is all of its deviations
        np.testing.assert_allclose(host(got["rstd"])[live], rstd[live], rtol=1e-4)
        np.testing.assert_allclose(host(got["y"])[live], y[live], rtol=1e-3, atol=1e-3)


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("x16", [False, True])
@pytest.mark.parametrize("d", [64, 250, 1000, 2730, 4096, 8192, 16384, 20000])
def test_rows_whose_squares_leave_fp32(d, x16, kind):
    """The mean square of fp32 is infinite: rstd is 0, and y the bias."""
    from paper_2509_13232_b200 import binding as B
    for scale in (1e21, 1e25, 1e30):
        for T in (3, 200):
            c = case(d, T, d, kind, x16, False, False)
            rng = np.random.default_rng(d)
            x = (scale * (rng.standard_normal((T, d)) + np.where(np.arange(d) < d // 2, 2.0, -2.0))).astype(np.float32)
            c["x"] = up(x, x16)
            got = run_fwd(c)
            assert got["status"] == B.DEV_NONFINITE
            assert not got["rstd"].any() and np.array_equal(host(got["y"]), np.broadcast_to(host(c["bias"]), (T, d)))
            if kind == O.LAYER:
                h = host(c["x"])
                assert np.all(np.abs(host(got["mean"]) - h.mean(axis=1)) <= 72 * 2.0**-24 * np.abs(h).mean(axis=1))
