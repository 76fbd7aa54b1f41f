"""Newton-Schulz updates at the ends of the range: zero matrices and the smallest epsilons, entries near the ends of fp32, and
coefficients under which the iteration has no bound."""

import numpy as np
import pytest

from oracle import operators as O
from tests.test_gpu_muon import gradient, orthogonalize, workspace

pytestmark = pytest.mark.gpu

TINY = 2.0**-126                          # the smallest normal fp32 number
LEAST = 2.0**-149                         # the smallest of all


@pytest.mark.parametrize("eps", [TINY, LEAST, 1e-37])
@pytest.mark.parametrize("m,n", [(40, 70), (300, 64), (64, 2000)])
def test_a_zero_update_is_zero_whatever_eps(m, n, eps):
    import torch
    from paper_2509_13232_b200 import binding as B
    g = np.zeros((2, m, n), np.float32)
    g[1] = gradient(np.random.default_rng(m), 1, m, n)[0]
    got, st = orthogonalize(g, eps=eps)
    assert st == 0 and np.all(got[0] == 0) and np.all(np.isfinite(got[1]))
    W = torch.ones(2, m, n, device="cuda").bfloat16()
    M, G = torch.zeros(2, m, n, device="cuda"), torch.from_numpy(g).cuda()
    ws, k = workspace(m, n, 2)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_muon_update(W, M, G, ws[:k], B.default_muon_params(eps=eps), status)
    torch.cuda.synchronize()
    assert int(status[0]) == 0 and bool((W[0] == 1).all()) and bool(torch.isfinite(W[1].float()).all())


# The factor scale / (norm + eps) is past fp32's range or among its subnormal numbers, with few bits left.
@pytest.mark.parametrize("m,n,size,eps", [(64, 64, 1e-37, LEAST), (300, 130, 2e-39, LEAST), (40, 900, 1e-36, TINY),
                                          (64, 64, 1e40, 1e-7), (300, 530, 3e40, 1e-7), (130, 200, 1e-8, 1e-7)])
def test_the_ends_of_the_range(m, n, size, eps):
    """Tolerance as in test_gpu_muon: twice what the fp16 roundings do to this input, and 2^-19 for the fp32 sums."""
    g = (gradient(np.random.default_rng(n), 1, m, n).astype(np.float64) * size).astype(np.float32)
    assert np.all(np.isfinite(g)) and np.any(g != 0)
    eps32 = float(np.float32(eps))
    got, st = orthogonalize(g, eps=eps)
    assert st == 0
    want, rounded = O.newton_schulz(g[0], eps=eps32), O.newton_schulz_rounded(g[0], eps=eps32)
    norm = np.linalg.norm(want)
    assert np.linalg.norm(got[0] - want) <= 2 * np.linalg.norm(rounded - want) + 2.0**-19 * norm


@pytest.mark.parametrize("m,n", [(60, 90), (500, 300), (1, 1)])
@pytest.mark.parametrize("bf16", [False, True])
def test_an_iteration_without_bound_is_reported(m, n, bf16):
    import torch
    from paper_2509_13232_b200 import binding as B
    g = gradient(np.random.default_rng(n), 1, m, n)
    got, st = orthogonalize(g, out_bf16=bf16, coef_a=90.0, coef_b=50.0, coef_c=50.0, steps=12)
    assert not np.all(np.isfinite(got)) and st == B.DEV_NONFINITE
    W = torch.zeros(m, n, device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    ws, k = workspace(m, n, 1)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    p = B.default_muon_params(coef_a=90.0, coef_b=50.0, coef_c=50.0, steps=12)
    B.spo_muon_update(W, torch.zeros(m, n, device="cuda"), torch.from_numpy(g[0]).cuda(), ws[:k], p, status)
    torch.cuda.synchronize()
    assert int(status[0]) == B.DEV_NONFINITE


def test_a_large_but_finite_result_is_not_reported():
    g = gradient(np.random.default_rng(0), 1, 60, 90)
    got, st = orthogonalize(g, coef_a=90.0, coef_b=0.0, coef_c=0.0, steps=2)        # X = 8100 U / |U|: no other term
    assert st == 0
    want = 8100.0 * g[0] / (np.linalg.norm(g[0].astype(np.float64)) + float(np.float32(1e-7)))
    np.testing.assert_allclose(got[0], want, rtol=2.0**-20)                          # six roundings to 32 bits
