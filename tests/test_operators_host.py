"""Host-only checks of the operators around the loss: the float64 definitions against closed forms and finite
differences, and the library's refusals, which come before any device work."""

import ctypes

import numpy as np
import pytest

from oracle import operators as O
from oracle import spo_oracle as S
from paper_2509_13232_b200 import binding as B
from paper_2509_13232_b200 import build as spo_build


@pytest.fixture(scope="module")
def lib():
    spo_build.build()
    return B.lib()


# ------------------------------------------------------------------------------------------------ definitions
def test_uniform_logits():
    out = O.logprobs(np.ones((3, 4)), np.zeros((10, 4)), np.array([0, 9, 10]), top_k=3)
    np.testing.assert_allclose(out["logp"], [-np.log(10), -np.log(10), -np.inf])
    np.testing.assert_allclose(out["entropy"], np.log(10))
    np.testing.assert_array_equal(out["top_ids"], [[0, 1, 2]] * 3)          # equal logits: ascending ids


def test_logprobs_against_the_loss_oracle_and_brute_force():
    rng = np.random.default_rng(0)
    h, w, y = rng.standard_normal((7, 5)), rng.standard_normal((11, 5)), rng.integers(0, 11, 7)
    out = O.logprobs(h, w, y, top_k=11)
    p = np.exp(h @ w.T)
    p /= p.sum(axis=1, keepdims=True)
    np.testing.assert_allclose(out["logp"], np.log(p[np.arange(7), y]))
    np.testing.assert_allclose(out["entropy"], -(p * np.log(p)).sum(axis=1))
    np.testing.assert_allclose(np.exp(out["top_logp"]).sum(axis=1), 1.0)
    assert np.all(np.diff(out["top_logp"], axis=1) <= 0)
    fwd = S.loss_forward(h, w, y, out["logp"], None, np.array([0, 7]), np.array([1.0]))
    np.testing.assert_allclose(fwd["logp"], out["logp"])
    np.testing.assert_allclose(fwd["loss"], -1.0)                            # every ratio is one
    half = O.logprobs(h, w, y, inv_t=0.5)
    np.testing.assert_allclose(half["logp"], O.logprobs(0.5 * h, w, y)["logp"])


def test_logprobs_gradients_against_differences():
    rng = np.random.default_rng(1)
    h, w, y = rng.standard_normal((4, 3)), rng.standard_normal((6, 3)), np.array([0, 5, 2, -100])
    mask, it = np.array([1, 1, 0, 1]), 0.7
    gl, gs, ge = rng.standard_normal((3, 4))
    gl[3] = 0.0                                                              # no target in that row

    def value(hh, ww):
        o = O.logprobs(hh, ww, y, None, it)
        keep = mask != 0
        return (np.where(y >= 0, gl, 0) * np.where(y >= 0, o["logp"], 0) + gs * o["lse"] + ge * o["entropy"])[keep].sum()

    o = O.logprobs(h, w, y, None, it)
    dh, dw, _ = O.logprobs_backward(h, w, y, mask, o["lse"], o["entropy"], gl, gs, ge, it)
    for x, dx, f in ((h, dh, lambda z: value(z, w)), (w, dw, lambda z: value(h, z))):
        for i in np.ndindex(*x.shape):
            step = np.zeros_like(x)
            step[i] = 1e-5
            assert abs((f(x + step) - f(x - step)) / 2e-5 - dx[i]) < 1e-8
    assert np.all(dh[2] == 0)


def test_the_loss_gradient_is_the_log_prob_gradient_with_coef():
    rng = np.random.default_rng(2)
    h, w, y, coef = rng.standard_normal((5, 3)), rng.standard_normal((7, 3)), rng.integers(0, 7, 5), rng.standard_normal(5)
    lse = O.logprobs(h, w, y)["lse"]
    dh, dw = S.loss_backward(h, w, y, lse, coef)
    dh2, dw2, _ = O.logprobs_backward(h, w, y, None, lse, None, coef, None, None)
    np.testing.assert_allclose(dh, dh2)
    np.testing.assert_allclose(dw, dw2)


def test_newton_schulz_acts_on_singular_values():
    rng = np.random.default_rng(3)
    u, _ = np.linalg.qr(rng.standard_normal((6, 4)))
    v, _ = np.linalg.qr(rng.standard_normal((9, 4)))
    sv = np.array([3.0, 1.0, 0.5, 0.2])
    a, b, c = O.NS_COEFFICIENTS
    x = sv / np.linalg.norm(sv)
    for _ in range(5):
        x = a * x + b * x**3 + c * x**5
    np.testing.assert_allclose(O.newton_schulz((u * sv) @ v.T), (u * x) @ v.T, atol=1e-6)    # eps = 1e-7 in the norm
    g = rng.standard_normal((6, 9))
    np.testing.assert_allclose(O.newton_schulz(g), O.newton_schulz(g.T).T, atol=1e-12)
    np.testing.assert_allclose(O.newton_schulz(g), O.newton_schulz(1e6 * g), atol=1e-6)
    assert np.all(O.newton_schulz(np.zeros((3, 4))) == 0)
    assert np.linalg.norm(O.newton_schulz_rounded(g) - O.newton_schulz(g)) < 5e-3 * np.linalg.norm(O.newton_schulz(g))


def test_muon_step_by_hand():
    """A rank-one gradient, one step of the map from sigma = 1: a + b + c times u v^T."""
    g = np.outer([3.0, 4.0], [0.0, 2.0])
    w, m, o = O.muon_update(np.ones((2, 2)), np.zeros((2, 2)), g, lr=0.1, mu=0.5, weight_decay=0.2, nesterov=True, mode=0, steps=1)
    np.testing.assert_allclose(m, g)
    k = sum(O.NS_COEFFICIENTS)
    np.testing.assert_allclose(o, k * np.outer([0.6, 0.8], [0.0, 1.0]), atol=1e-6)
    np.testing.assert_allclose(w, 0.98 - 0.1 * o)
    assert O.muon_scale(400, 100, 1) == 2.0 and O.muon_scale(100, 400, 1) == 1.0 and O.muon_scale(100, 400, 2) == 4.0


# ------------------------------------------------------------------------------------------------ refusals
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)       # never dereferenced on the host
BIG = 1 << 40


def lp(lib, H=FAKE, ldH=64, W=FAKE, dtype=1, y=FAKE, mask=None, T=8, d=64, V=100, it=1.0, K=2, logp=FAKE, lse=FAKE, ent=None,
       ids=FAKE, tlp=FAKE, ws=FAKE, n=BIG):
    return lib.spo_logprobs(H, ldH, W, dtype, y, mask, T, d, V, it, K, logp, lse, ent, ids, tlp, ws, n, None, None)


@pytest.mark.parametrize("bad,want", [
    (dict(dtype=7), B.ERR_UNSUPPORTED_DTYPE), (dict(T=-1), B.ERR_INVALID_ARG), (dict(d=0), B.ERR_INVALID_ARG),
    (dict(V=0), B.ERR_INVALID_ARG), (dict(ldH=32), B.ERR_INVALID_ARG), (dict(ldH=68), B.ERR_BAD_SHAPE),
    (dict(d=72, ldH=72), B.ERR_BAD_SHAPE), (dict(dtype=0, d=66, ldH=68), B.ERR_BAD_SHAPE), (dict(V=1 << 29), B.ERR_BAD_SHAPE),
    (dict(T=1 << 31), B.ERR_BAD_SHAPE), (dict(it=0.0), B.ERR_INVALID_ARG), (dict(it=-1.0), B.ERR_INVALID_ARG),
    (dict(it=float("nan")), B.ERR_INVALID_ARG), (dict(it=float("inf")), B.ERR_INVALID_ARG), (dict(K=21), B.ERR_INVALID_ARG),
    (dict(K=-1), B.ERR_INVALID_ARG), (dict(V=1), B.ERR_INVALID_ARG), (dict(y=None), B.ERR_INVALID_ARG),
    (dict(logp=None), B.ERR_INVALID_ARG), (dict(lse=None), B.ERR_INVALID_ARG), (dict(ids=None), B.ERR_INVALID_ARG),
    (dict(tlp=None), B.ERR_INVALID_ARG), (dict(H=None), B.ERR_INVALID_ARG), (dict(ws=None), B.ERR_INVALID_ARG),
    (dict(H=ODD), B.ERR_BAD_ALIGNMENT), (dict(W=ODD), B.ERR_BAD_ALIGNMENT), (dict(ent=ODD), B.ERR_BAD_ALIGNMENT)])
def test_logprobs_refuses(lib, bad, want):
    assert lp(lib, **bad) == want


def lpb(lib, H=FAKE, ldH=64, W=FAKE, dtype=1, y=FAKE, mask=None, lse=FAKE, ent=FAKE, gl=FAKE, gs=None, ge=FAKE, T=8, d=64, V=100,
        it=1.0, dH=FAKE, dHt=1, dW=FAKE, dWt=1, ws=FAKE):
    return lib.spo_logprobs_bwd(H, ldH, W, dtype, y, mask, lse, ent, gl, gs, ge, T, d, V, it, dH, dHt, dW, dWt, 0, ws, BIG, None, None)


@pytest.mark.parametrize("bad,want", [
    (dict(dtype=3), B.ERR_UNSUPPORTED_DTYPE), (dict(dHt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(dWt=-1), B.ERR_UNSUPPORTED_DTYPE),
    (dict(dtype=0, dHt=0, dWt=1), B.ERR_UNSUPPORTED_DTYPE), (dict(dtype=0, dHt=1, dWt=0), B.ERR_UNSUPPORTED_DTYPE),
    (dict(d=96, ldH=96), B.ERR_BAD_SHAPE), (dict(y=None), B.ERR_INVALID_ARG), (dict(ent=None), B.ERR_INVALID_ARG),
    (dict(lse=None), B.ERR_INVALID_ARG), (dict(dH=None), B.ERR_INVALID_ARG), (dict(dW=None), B.ERR_INVALID_ARG),
    (dict(ws=None), B.ERR_INVALID_ARG), (dict(dW=ODD), B.ERR_BAD_ALIGNMENT), (dict(gl=ODD), B.ERR_BAD_ALIGNMENT),
    (dict(it=0.0), B.ERR_INVALID_ARG), (dict(ldH=60), B.ERR_INVALID_ARG)])
def test_logprobs_bwd_refuses(lib, bad, want):
    assert lpb(lib, **bad) == want


def mu(lib, W=FAKE, Wt=1, M=FAKE, G=FAKE, Gt=0, b=1, m=8, n=8, ws=FAKE, **params):
    return lib.spo_muon_update(W, Wt, M, G, Gt, b, m, n, ws, BIG, ctypes.byref(B.default_muon_params(**params)), None, None)


@pytest.mark.parametrize("bad,want", [
    (dict(Wt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(Gt=5), B.ERR_UNSUPPORTED_DTYPE), (dict(b=-1), B.ERR_INVALID_ARG),
    (dict(m=0), B.ERR_INVALID_ARG), (dict(n=-3), B.ERR_INVALID_ARG), (dict(m=1 << 24), B.ERR_BAD_SHAPE),
    (dict(m=70000, n=70000), B.ERR_BAD_SHAPE), (dict(b=70000), B.ERR_BAD_SHAPE), (dict(W=None), B.ERR_INVALID_ARG),
    (dict(M=None), B.ERR_INVALID_ARG), (dict(G=None), B.ERR_INVALID_ARG), (dict(ws=None), B.ERR_INVALID_ARG),
    (dict(W=ODD), B.ERR_BAD_ALIGNMENT), (dict(M=ODD), B.ERR_BAD_ALIGNMENT), (dict(steps=0), B.ERR_INVALID_ARG),
    (dict(steps=17), B.ERR_INVALID_ARG), (dict(momentum=1.0), B.ERR_INVALID_ARG), (dict(eps=0.0), B.ERR_INVALID_ARG),
    (dict(lr=float("nan")), B.ERR_INVALID_ARG), (dict(coef_a=1e3), B.ERR_INVALID_ARG), (dict(nesterov=2), B.ERR_INVALID_ARG),
    (dict(scale_mode=3), B.ERR_INVALID_ARG)])
def test_muon_refuses(lib, bad, want):
    assert mu(lib, **bad) == want


def test_orthogonalize_refuses(lib):
    p = ctypes.byref(B.default_muon_params())
    assert lib.spo_orthogonalize(FAKE, 0, 1, 8, 8, None, 0, FAKE, BIG, p, None, None) == B.ERR_INVALID_ARG
    assert lib.spo_orthogonalize(FAKE, 0, 1, 8, 8, ODD, 0, FAKE, BIG, p, None, None) == B.ERR_BAD_ALIGNMENT
    assert lib.spo_orthogonalize(FAKE, 0, 1, 8, 8, FAKE, 4, FAKE, BIG, p, None, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.spo_orthogonalize(FAKE, 0, 1, 8, 8, FAKE, 0, FAKE, BIG, None, None, None) == B.ERR_INVALID_ARG
    assert lib.spo_default_muon_params(None) == B.ERR_INVALID_ARG


def test_scratch_sizes(lib):
    size = B.spo_workspace_bytes
    assert size(B.WS_LOGPROBS, T=0, d=64, V=10, B=0) >= 0
    assert size(B.WS_LOGPROBS, T=5, d=64, V=10, B=21) == 0                   # more alternatives than there may be
    assert size(B.WS_LOGPROBS, T=100000, d=4096, V=151936, B=20) < 3 << 30   # bounded, whatever T is
    assert size(B.WS_LOGPROBS, T=10**6, d=4096, V=151936, B=20) < 3 << 30
    assert size(B.WS_LOGPROBS_BWD, T=10**6, d=4096, V=151936) == size(B.WS_LOGPROBS_BWD, T=9472 * 100, d=4096, V=151936)
    assert size(B.WS_MUON, T=0, d=5, B=1) == 0 and size(B.WS_MUON, T=70000, d=70000, B=1) == 0
    assert 0 < size(B.WS_MUON, T=100, d=200, B=1) < size(B.WS_MUON, T=100, d=200, B=3)
