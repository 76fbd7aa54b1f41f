"""Norms of rows whose mean is far from zero and whose columns lie on levels of their own: squares are those about the mean.

Tolerances, derived before any run; u = 2^-24.  A row of up to 16384 columns: a thread adds at most 16 terms of a kind, then five shuffles, then at
most 32 warps.
  Squares about the mean m that the call returns (no slip of m's own is in them): with c_w the distance of a warp's point from m and S_w the
  squares about that point, the terms S_w, 2 c_w E_w and n_w c_w^2 take at most 16 + 5 + 3 roundings each, E_w as many of sum |deviation|, and
  2 |c e| <= c^2 + e^2, so at most 56 u of S_w + n_w c_w^2; joining 32 warps, the division and eps 36 u more.  rstd: half of that, and four roundings of its
  own: 50 u.  (For points near the warps' means.  The kernel's may be up to sqrt(3) deviations off them, which the bound is not widened for.)
  mean: as in the tests of ordinary rows, K u mean|h| with K = 72.
  y (fp32) from the returned mean and rstd: (x - m) r w + b takes four roundings.
"""

import numpy as np
import pytest

from oracle import step as O
from tests.test_gpu_layernorm import U, case, host, run_fwd, up

pytestmark = pytest.mark.gpu


def levels(rng, pattern, T, d):
    """Levels of the columns, of size one."""
    j = np.arange(d)
    if pattern == "halves":
        one = np.where(j < d // 2, 1.0, -1.0)
    elif pattern == "blocks":
        one = np.where(j // 128 % 2 == 0, 1.0, -1.0)
    elif pattern == "slope":
        one = 2.0 * j / d - 1.0
    else:
        one = rng.standard_normal(-(-d // 256))[j // 256]
    return np.broadcast_to(one, (T, d))


@pytest.mark.parametrize("offset", [0.0, 100.0, 1000.0, 20000.0])
@pytest.mark.parametrize("pattern", ["halves", "blocks", "slope", "random"])
@pytest.mark.parametrize("d,T", [(256, 3), (1365, 5), (3000, 20), (3000, 400), (4096, 3), (4096, 400), (4103, 300), (16384, 4), (16384, 200)])
def test_squares_of_columns_on_levels(d, T, pattern, offset):
    for x16 in (False, True):
        for residual in (False, True):
            rng = np.random.default_rng(d + T)
            c = case(d, T, d, O.LAYER, x16, False, False, residual=residual)
            x = levels(rng, pattern, T, d) + 0.05 * rng.standard_normal((T, d)) + offset * rng.uniform(0.9, 1.1, (T, 1))
            c["x"] = up(x.astype(np.float32), x16)
            got = run_fwd(c, eps=1e-6)
            h = host(got["h"]) if residual else host(c["x"])
            mean, rstd = host(got["mean"])[:, None], host(got["rstd"])[:, None]
            assert np.all(np.abs(mean - h.mean(axis=1, keepdims=True)) <= 72 * U * np.abs(h).mean(axis=1, keepdims=True))
            want = 1.0 / np.sqrt(((h - mean)**2).mean(axis=1, keepdims=True) + 1e-6)
            worst = float((np.abs(rstd - want) / (U * want)).max())
            assert worst <= 50, worst
            xw = (h - mean) * rstd * host(c["weight"])
            y = xw + host(c["bias"])
            assert np.all(np.abs(host(got["y"]) - y) <= 4 * U * (np.abs(xw) + np.abs(y)))
