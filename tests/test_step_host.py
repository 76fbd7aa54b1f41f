"""Without a GPU: the float64 definitions of oracle/step.py (closed forms, finite differences), and what spo_layernorm_*, spo_grad_norm and
spo_adamw_* refuse before anything is launched."""

import ctypes
import math

import numpy as np
import pytest

from oracle import step as O
from paper_2509_13232_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    return B.lib()


# ------------------------------------------------------------------------------------------------ definitions
def test_layer_norm_by_hand():
    x = np.array([[1.0, 3.0, 5.0, 7.0], [2.0, 2.0, 2.0, 2.0]])
    o = O.layernorm(x, weight=[1, 2, 1, 1], bias=[0, 0, 10, 0], eps=1e-12)
    s = 1 / math.sqrt(5.0)
    np.testing.assert_allclose(o["y"][0], [-3 * s, -2 * s, 10 + s, 3 * s], rtol=1e-9)
    np.testing.assert_allclose(o["y"][1], [0, 0, 10, 0])
    np.testing.assert_allclose(o["mean"], [4, 2])
    r = O.layernorm(x, kind=O.RMS, eps=1e-12)
    np.testing.assert_allclose(r["y"][0], x[0] / math.sqrt(21.0), rtol=1e-9)
    np.testing.assert_allclose(r["rstd"], [21.0**-0.5, 0.5], rtol=1e-9)
    m = O.layernorm(np.where([[True], [False]], x, np.nan), mask=[1, 0])
    assert np.all(m["y"][1] == 0) and m["rstd"][1] == 0 and np.isfinite(m["y"]).all()


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
def test_layer_norm_gradients_by_differences(kind):
    rng = np.random.default_rng(0)
    x, w, b, dy, dh = rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal(5), *rng.standard_normal((2, 3, 5))
    mask = [1, 0, 1]

    def value(x, w, b):
        return float((O.layernorm(x, w, b, mask=mask, eps=1e-3, kind=kind)["y"] * dy).sum() + (x * dh)[[0, 2]].sum())

    f = O.layernorm(x, w, b, mask=mask, eps=1e-3, kind=kind)
    g = O.layernorm_backward(dy, x, f["mean"], f["rstd"], w, dh, mask, kind)
    for name, at in (("dx", 0), ("dw", 1), ("db", 2)):
        args = [x, w, b]
        for i in np.ndindex(*args[at].shape):
            step = np.zeros_like(args[at])
            step[i] = 1e-5
            up, down = list(args), list(args)
            up[at], down[at] = args[at] + step, args[at] - step
            assert abs((value(*up) - value(*down)) / 2e-5 - g[name][i]) < 1e-8


def test_gradient_norm_by_hand():
    assert O.grad_norm([[3.0], [[0.0, 4.0]]]) == (5.0, 1.0)
    assert O.grad_norm([[3.0], [4.0]], max_norm=1.0, scale=0.5) == (2.5, 0.2)
    assert O.grad_norm([[3.0], [4.0]], max_norm=3.0, scale=-0.5) == (2.5, -0.5)
    assert O.grad_norm([]) == (0.0, 1.0)


def test_adamw_by_hand():
    """From zero moments the first step is lr sign(g) (up to eps), whatever the betas."""
    w, m, v, first = O.adamw([1.0, 1.0, 2.0], [0.5, -2.0, 0.0], np.zeros(3), np.zeros(3), 1, lr=0.25, decay=0.5)
    np.testing.assert_allclose(w, [1 - 0.25 - 0.125, 1 + 0.25 - 0.125, 2 - 0.25], rtol=1e-6)
    np.testing.assert_allclose(m, [0.05, -0.2, 0], rtol=1e-6)
    np.testing.assert_allclose(v, [0.00025, 0.004, 0], rtol=1e-4)
    # a gradient that is not usable changes nothing
    w, m, v, _ = O.adamw([1.0] * 3, [np.nan, np.inf, 2.0**61], [3.0] * 3, [4.0] * 3, 7, lr=0.25, decay=0.5)
    assert np.all(w == 1) and np.all(m == 3) and np.all(v == 4)
    # the moments of a constant gradient approach it, its step the rate
    w, m, v = np.zeros(1), np.zeros(1), np.zeros(1)
    for t in range(1, 2000):
        w, m, v, first = O.adamw(w, [0.01], m, v, t, lr=2.0**-10, beta2=0.99)
    np.testing.assert_allclose([m[0], v[0], first[0]], [0.01, 1e-4, 2.0**-10], rtol=1e-4)


def test_codes_of_8_bit_states():
    rng = np.random.default_rng(1)
    # every code of a block whose scale is its largest magnitude comes back as it was
    for sign in (1, -1):
        m = np.concatenate([np.arange(128), np.full(128, 127)]).astype(np.int8) * np.int8(sign)
        v = np.arange(256).astype(np.uint8)
        for scale in (1.0, 3e-7, 5e4):
            s = np.array([scale], np.float32)
            fm, fv = O.decode(m, s, v, s)
            np.testing.assert_allclose(fm, sign * scale * (np.abs(m.astype(float)) / 127)**2, rtol=1e-6)
            np.testing.assert_allclose(fv, scale * (v / 255.0)**4, rtol=1e-6)
            cm, sm, cv, sv = O.encode(fm, fv)
            assert np.array_equal(cm, m) and np.array_equal(cv, v)
    # a code is never further than half a step of the root from its value
    m, v = (rng.standard_normal(1000) * 1e-3).astype(np.float32), (rng.standard_normal(1000)**4 * 1e-6).astype(np.float32)
    cm, sm, cv, sv = O.encode(m, v)
    fm, fv = O.decode(cm, sm, cv, sv)
    top = np.repeat(sm, 256)[:1000].astype(float)
    assert np.all(np.abs(np.sqrt(np.abs(fm) / top) - np.sqrt(np.abs(m) / top)) <= 0.5 / 127 + 1e-6) and np.all(fm * m >= 0)
    top = np.repeat(sv, 256)[:1000].astype(float)
    far = np.abs((fv / top)**0.25 - (v / top)**0.25)
    assert np.all(far <= np.where(cv == 1, 1.0, 0.5) / 255 + 1e-6)
    # zeros, the floors, and a positive v that would round to zero
    cm, sm, cv, sv = O.encode(np.zeros(3, np.float32), np.array([1.0, 1e-30, 0.0], np.float32))
    assert list(cm) == [0, 0, 0] and sm[0] == 2.0**-100 and list(cv) == [255, 1, 0]


# ------------------------------------------------------------------------------------------------ refusals
BIG = 1 << 40


def at(k, odd=0):
    """Addresses far apart; never dereferenced on the host."""
    return ctypes.c_void_p((k + 1 << 44) + odd)


NAN, INF = float("nan"), float("inf")
X, R, W_, BIAS, MASK, Y, H, MEAN, RSTD, DY, DH, DX, DW, DB, WS = range(15)


def fwd(lib, x=at(X), ldx=64, r=None, dt=1, w=at(W_), b=at(BIAS), wt=1, mask=at(MASK), T=8, d=64, eps=1e-6, kind=0, y=at(Y), yt=1,
        h=None, mean=at(MEAN), rstd=at(RSTD)):
    return lib.spo_layernorm_fwd(x, ldx, r, dt, w, b, wt, mask, T, d, eps, kind, y, yt, h, mean, rstd, None, None)


@pytest.fixture
def no_gpu():
    """Calls that pass every check, with addresses of nothing: only where there is no device that could run them."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    return lambda rc: rc == B.ERR_UNSUPPORTED_ARCH


@pytest.mark.parametrize("bad,want", [
    (dict(dt=3), B.ERR_UNSUPPORTED_DTYPE), (dict(wt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(yt=-1), B.ERR_UNSUPPORTED_DTYPE),
    (dict(T=-1), B.ERR_INVALID_ARG), (dict(d=0), B.ERR_INVALID_ARG), (dict(ldx=63), B.ERR_INVALID_ARG), (dict(kind=2), B.ERR_INVALID_ARG),
    (dict(T=1 << 31), B.ERR_BAD_SHAPE), (dict(d=(1 << 20) + 1, ldx=1 << 21), B.ERR_BAD_SHAPE), (dict(eps=0.0), B.ERR_INVALID_ARG),
    (dict(eps=NAN), B.ERR_INVALID_ARG), (dict(eps=INF), B.ERR_INVALID_ARG), (dict(r=at(R)), B.ERR_INVALID_ARG),
    (dict(h=at(H)), B.ERR_INVALID_ARG), (dict(kind=1), B.ERR_INVALID_ARG), (dict(x=None), B.ERR_INVALID_ARG),
    (dict(y=None), B.ERR_INVALID_ARG), (dict(x=at(X, 8)), B.ERR_BAD_ALIGNMENT), (dict(w=at(W_, 2)), B.ERR_BAD_ALIGNMENT),
    (dict(rstd=at(RSTD, 4)), B.ERR_BAD_ALIGNMENT),
    # outputs on top of inputs: y on x only element for element
    (dict(y=at(X, 16)), B.ERR_INVALID_ARG), (dict(y=at(X), ldx=72), B.ERR_INVALID_ARG), (dict(y=at(X), yt=0), B.ERR_INVALID_ARG),
    (dict(y=at(X), r=at(R), h=at(H)), B.ERR_INVALID_ARG), (dict(y=at(R), r=at(R), h=at(H)), B.ERR_INVALID_ARG),
    (dict(y=at(H), r=at(R), h=at(H)), B.ERR_INVALID_ARG), (dict(h=at(X), r=at(R), ldx=72), B.ERR_INVALID_ARG),
    (dict(h=at(R, 32), r=at(R)), B.ERR_INVALID_ARG), (dict(y=at(W_)), B.ERR_INVALID_ARG), (dict(mean=at(X)), B.ERR_INVALID_ARG),
    (dict(mean=at(RSTD)), B.ERR_INVALID_ARG), (dict(rstd=at(Y)), B.ERR_INVALID_ARG)])
def test_layernorm_fwd_refuses(lib, bad, want):
    assert fwd(lib, **bad) == want


@pytest.mark.parametrize("good", [
    dict(), dict(T=0, x=None, y=None), dict(w=None, b=None, mean=None, rstd=None, mask=None), dict(kind=1, mean=None), dict(y=at(X)),
    dict(h=at(X), r=at(R)), dict(h=at(R), r=at(R)), dict(d=63, ldx=65), dict(yt=0), dict(dt=0, wt=0, yt=1), dict(T=1, ldx=999, y=at(X)),
    dict(d=1 << 20, ldx=1 << 20)])
def test_layernorm_fwd_takes(lib, no_gpu, good):
    assert no_gpu(fwd(lib, **good))


def bwd(lib, dy=at(DY), dyt=1, x=at(X), ldx=64, dt=1, w=at(W_), wt=1, mask=at(MASK), mean=at(MEAN), rstd=at(RSTD), dh=at(DH), T=8, d=64,
        kind=0, dx=at(DX), dw=at(DW), db=at(DB), dwt=0, ws=at(WS), n=BIG):
    return lib.spo_layernorm_bwd(dy, dyt, x, ldx, dt, w, wt, mask, mean, rstd, dh, T, d, kind, dx, dw, db, dwt, 0, ws, n, None, None)


@pytest.mark.parametrize("bad,want", [
    (dict(dt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(dyt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(dwt=9), B.ERR_UNSUPPORTED_DTYPE),
    (dict(wt=-2), B.ERR_UNSUPPORTED_DTYPE), (dict(T=-5), B.ERR_INVALID_ARG), (dict(d=-1), B.ERR_INVALID_ARG), (dict(kind=7), B.ERR_INVALID_ARG),
    (dict(ldx=10), B.ERR_INVALID_ARG), (dict(T=1 << 31), B.ERR_BAD_SHAPE), (dict(mean=None), B.ERR_INVALID_ARG),
    (dict(kind=1), B.ERR_INVALID_ARG), (dict(rstd=None), B.ERR_INVALID_ARG), (dict(dy=None), B.ERR_INVALID_ARG),
    (dict(x=None), B.ERR_INVALID_ARG), (dict(dx=None), B.ERR_INVALID_ARG), (dict(ws=None), B.ERR_INVALID_ARG),
    (dict(dw=at(DW, 4)), B.ERR_BAD_ALIGNMENT), (dict(dy=at(DY, 2)), B.ERR_BAD_ALIGNMENT), (dict(dw=at(DB)), B.ERR_INVALID_ARG),
    (dict(dx=at(DY), dyt=0), B.ERR_INVALID_ARG), (dict(dx=at(DY, 16)), B.ERR_INVALID_ARG), (dict(dx=at(DH, 32)), B.ERR_INVALID_ARG),
    (dict(dx=at(X), ldx=80), B.ERR_INVALID_ARG), (dict(dx=at(W_)), B.ERR_INVALID_ARG), (dict(dw=at(X)), B.ERR_INVALID_ARG),
    (dict(db=at(DX, 64)), B.ERR_INVALID_ARG), (dict(dw=at(RSTD)), B.ERR_INVALID_ARG)])
def test_layernorm_bwd_refuses(lib, bad, want):
    assert bwd(lib, **bad) == want


@pytest.mark.parametrize("good", [
    dict(), dict(T=0, dy=None, x=None, dx=None, rstd=None, ws=None, mean=None), dict(dw=None, db=None, ws=None, n=0), dict(kind=1, mean=None),
    dict(dx=at(DY)), dict(dx=at(DH)), dict(dx=at(X)), dict(dyt=0), dict(w=None, mask=None, dh=None, db=None), dict(d=61, ldx=61)])
def test_layernorm_bwd_takes(lib, no_gpu, good):
    assert no_gpu(bwd(lib, **good))


def norm(lib, g=at(0), n=100, dt=1, k=1, mx=1.0, s=1.0, out=at(1), ws=at(2), nb=BIG, table=True):
    t = (B.SpoGradTensor * 2)()
    t[0].g, t[0].n, t[0].dtype = g, n, dt
    return lib.spo_grad_norm(t if table else None, k, mx, s, out, ws, nb, None, None)


@pytest.mark.parametrize("bad,want", [
    (dict(k=-1), B.ERR_INVALID_ARG), (dict(table=False), B.ERR_INVALID_ARG), (dict(out=None), B.ERR_INVALID_ARG),
    (dict(ws=None), B.ERR_INVALID_ARG), (dict(dt=2), B.ERR_UNSUPPORTED_DTYPE), (dict(n=-1), B.ERR_INVALID_ARG), (dict(g=None), B.ERR_INVALID_ARG),
    (dict(n=1 << 40), B.ERR_BAD_SHAPE), (dict(g=at(0, 1)), B.ERR_BAD_ALIGNMENT), (dict(g=at(0, 2), dt=0), B.ERR_BAD_ALIGNMENT),
    (dict(mx=NAN), B.ERR_INVALID_ARG), (dict(mx=INF), B.ERR_INVALID_ARG), (dict(s=NAN), B.ERR_INVALID_ARG), (dict(s=-INF), B.ERR_INVALID_ARG),
    (dict(ws=at(2, 8)), B.ERR_BAD_ALIGNMENT), (dict(out=at(1, 4)), B.ERR_BAD_ALIGNMENT)])
def test_grad_norm_refuses(lib, bad, want):
    assert norm(lib, **bad) == want


def test_grad_norm_takes(lib, no_gpu):
    for good in (dict(), dict(k=0, table=False), dict(n=0, g=None), dict(g=at(0, 2)), dict(mx=-1.0), dict(s=-0.5)):
        assert no_gpu(norm(lib, **good))


def adam(lib, k=1, table=True, params=True, f=None, rate=None, count=None, tensor={}, **overrides):
    t = (B.SpoAdamwTensor * 2)()
    q = t[0]
    q.w, q.g, q.m, q.v, q.n, q.state_bits, q.lr_scale, q.decay_scale = at(0), at(1), at(2), at(3), 100, 32, 1.0, 1.0
    for name, x in tensor.items():
        setattr(q, name, x)
    p = ctypes.byref(B.default_adamw_params(**overrides)) if params else None
    return lib.spo_adamw_update(t if table else None, k, f, rate, count, p, None, None)


EIGHT = dict(state_bits=8, m_scale=at(4), v_scale=at(5))


@pytest.mark.parametrize("bad,want", [
    (dict(k=-1), B.ERR_INVALID_ARG), (dict(table=False), B.ERR_INVALID_ARG), (dict(params=False), B.ERR_INVALID_ARG),
    (dict(lr=NAN), B.ERR_INVALID_ARG), (dict(lr=INF), B.ERR_INVALID_ARG), (dict(beta1=1.0), B.ERR_INVALID_ARG), (dict(beta2=-0.1), B.ERR_INVALID_ARG),
    (dict(beta1=NAN), B.ERR_INVALID_ARG), (dict(eps=0.0), B.ERR_INVALID_ARG), (dict(eps=-1.0), B.ERR_INVALID_ARG), (dict(eps=INF), B.ERR_INVALID_ARG),
    (dict(weight_decay=NAN), B.ERR_INVALID_ARG), (dict(step=0), B.ERR_INVALID_ARG), (dict(f=at(8, 2)), B.ERR_BAD_ALIGNMENT),
    (dict(rate=at(8, 1)), B.ERR_BAD_ALIGNMENT)] + [(dict(tensor=t), want) for t, want in (
        (dict(w_dtype=2), B.ERR_UNSUPPORTED_DTYPE), (dict(g_dtype=3), B.ERR_UNSUPPORTED_DTYPE), (dict(state_bits=16), B.ERR_UNSUPPORTED_DTYPE),
        (dict(n=-1), B.ERR_INVALID_ARG), (dict(n=1 << 34), B.ERR_BAD_SHAPE), (dict(w=None), B.ERR_INVALID_ARG), (dict(g=None), B.ERR_INVALID_ARG),
        (dict(m=None), B.ERR_INVALID_ARG), (dict(v=None), B.ERR_INVALID_ARG), (dict(m_scale=at(4)), B.ERR_INVALID_ARG),
        (dict(state_bits=8), B.ERR_INVALID_ARG), (dict(EIGHT, v_scale=None), B.ERR_INVALID_ARG), (dict(lr_scale=NAN), B.ERR_INVALID_ARG),
        (dict(decay_scale=INF), B.ERR_INVALID_ARG), (dict(w=at(0, 2)), B.ERR_BAD_ALIGNMENT), (dict(g=at(1, 1), g_dtype=1), B.ERR_BAD_ALIGNMENT),
        (dict(m=at(2, 1)), B.ERR_BAD_ALIGNMENT), (dict(copy=at(6, 1)), B.ERR_BAD_ALIGNMENT), (dict(EIGHT, m_scale=at(4, 2)), B.ERR_BAD_ALIGNMENT))])
def test_adamw_refuses(lib, bad, want):
    assert adam(lib, **bad) == want


def test_adamw_takes(lib, no_gpu):
    for good in (dict(), dict(k=0, table=False), dict(tensor=dict(n=0, w=None, g=None, m=None, v=None)), dict(tensor=EIGHT), dict(beta1=0.0, beta2=0.0),
                 dict(tensor=dict(EIGHT, m=at(2, 1), v=at(3, 3), w=at(0, 2), w_dtype=1, g=at(1, 4), copy=at(6, 2))), dict(lr=-1.0),
                 dict(f=at(8, 4), rate=at(9, 4), count=at(10, 4))):
        assert no_gpu(adam(lib, **good))
    assert lib.spo_default_adamw_params(None) == B.ERR_INVALID_ARG


def test_decode_refuses(lib, no_gpu):
    d = lambda m=at(0), ms=at(1), v=at(2), vs=at(3), n=10, mo=at(4), vo=at(5): lib.spo_adamw_decode(m, ms, v, vs, n, mo, vo, None)  # noqa: E731
    for bad in (dict(n=-1), dict(m=None), dict(mo=None), dict(v=None), dict(vo=None), dict(ms=None), dict(vs=None)):
        assert d(**bad) == B.ERR_INVALID_ARG
    assert d(ms=at(1, 2)) == B.ERR_BAD_ALIGNMENT and d(vo=at(5, 1)) == B.ERR_BAD_ALIGNMENT
    for good in (dict(), dict(m=None, mo=None), dict(v=None, vo=None, vs=None), dict(m=at(0, 1)), dict(n=0, m=None)):
        assert no_gpu(d(**good))


def test_results_share_memory_with_nothing(lib, no_gpu):
    assert norm(lib, out=at(0, 192)) == B.ERR_INVALID_ARG and norm(lib, ws=at(0, 192)) == B.ERR_INVALID_ARG
    assert norm(lib, ws=at(1)) == B.ERR_INVALID_ARG
    assert no_gpu(norm(lib, out=at(0, 208), ws=at(3))) and no_gpu(norm(lib, n=0, out=at(0)))
    d = lambda m=at(0), ms=at(1), v=at(2), vs=at(3), n=300, mo=at(4), vo=at(5): lib.spo_adamw_decode(m, ms, v, vs, n, mo, vo, None)  # noqa: E731
    for bad in (dict(mo=at(0)), dict(mo=at(0, 296)), dict(mo=at(2)), dict(vo=at(1, 4)), dict(vo=at(3)), dict(vo=at(4, 1196)), dict(vo=at(0, 196))):
        assert d(**bad) == B.ERR_INVALID_ARG
    assert no_gpu(d(mo=at(0, 300))) and no_gpu(d(vo=at(4, 1200))) and no_gpu(d(n=0, mo=at(0)))


def test_scratch_sizes_of_the_step():
    size = B.spo_workspace_bytes
    for d in (1, 7, 64, 1000, 4096, 8192, 8200, 16384, 20000, 1 << 20):
        sizes = [size(B.WS_LAYERNORM_BWD, T=T, d=d) for T in (0, 1, 2, 17, 200, 5000, 10**6)]
        assert sizes == sorted(sizes) and sizes[0] > 0              # a buffer serves shorter calls
    assert size(B.WS_LAYERNORM_BWD, T=10**6, d=4096) < 64 << 20
    assert size(B.WS_LAYERNORM_BWD, T=5, d=(1 << 20) + 1) == 0 and size(B.WS_LAYERNORM_BWD, T=-1, d=5) == 0
    assert 0 < size(B.WS_GRAD_NORM) == size(B.WS_GRAD_NORM, N=10**12) < 1 << 16


# ------------------------------------------------------------------------------------------------ tables
def test_the_tables_refuse_on_the_host():
    import torch
    x = torch.zeros(8)
    with pytest.raises(ValueError):
        B.grad_list([x])                            # not on a GPU
    with pytest.raises(TypeError):
        B.grad_list([[1.0]])
    with pytest.raises(ValueError):
        B.adamw_list([x], [], [x], [x])             # a list is too short
    assert B.grad_list([]).count == 0
