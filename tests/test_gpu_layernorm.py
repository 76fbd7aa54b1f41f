"""GPU parity of spo_layernorm_fwd / spo_layernorm_bwd with the float64 definitions.

Tolerances, derived before any run; u = 2^-24 is half a step of fp32.  A sum of n terms over a row is taken by at most 1024 threads of
at most 32 terms each (longer rows: d / 1024 terms), five shuffles and at most 32 warps, so each of its terms takes at most
K = max(32, d / 1024) + 40 roundings: |error of a sum| <= K u sum |terms|.
  mean:  K u mean|h|.   rstd: half the relative error of the mean square, (K + 4) u / 2, and three roundings of its own, plus what the
  mean's error moves the squares by (second order).   y: (|xh| (K u + 4 u) + rstd (K u mean|h| + u |h|)) |w| + 2 u |y| + output rounding.
  dx: with c1 = mean(a xh), c2 = mean(a): rstd (4 u |a| + |xh| (K + 4) u mean|a xh| + 4 u |xh c1| + K u mean|a| + 2 u |c2|) + u |dx| +
  output rounding.   dw, db: a column's terms are added up by at most T / 64 + 100 roundings each: that times u sum |terms|, twice
  (the terms themselves have four roundings), plus output rounding.
The output's rounding is 2^-8 of the value for bf16 (half a step is at most 2^-9 of the largest value of a binade, 2^-8 of the smallest).
"""

import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu

U = 2.0**-24


def rows(rng, t, d):
    x = rng.standard_normal((t, d)) * np.exp(0.5 * rng.standard_normal((t, 1))) + rng.standard_normal((t, 1))
    return x.astype(np.float32)


def up(x, bf16=False):
    import torch
    if x is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.bfloat16() if bf16 else t


def host(t):
    return t.double().cpu().numpy()


def half_step(bf16):
    return 2.0**-8 if bf16 else U


def case(seed, T, d, kind, x16, y16, w16, weight=True, bias=True, residual=False, masked=False, pad=0, offset=0.0):
    import torch
    rng = np.random.default_rng(seed)
    c = dict(T=T, d=d, kind=kind, x16=x16, y16=y16, w16=w16)
    wide = up(rows(rng, T, d + pad) + np.float32(offset), x16)
    c["x"] = wide[:, :d]
    c["residual"] = up(rows(rng, T, d), x16) if residual else None
    c["weight"] = up((1 + 0.3 * rng.standard_normal(d)).astype(np.float32), w16) if weight else None
    c["bias"] = up(rng.standard_normal(d).astype(np.float32), w16) if bias else None
    c["mask"] = None
    if masked:
        keep = rng.random(T) < 0.6
        keep[0] = False
        c["mask"] = up(keep.astype(np.uint8))
        poison = torch.from_numpy(~keep).cuda()
        wide[poison, ::3] = float("nan")
        wide[poison, 1::3] = float("inf")
        if residual:
            c["residual"][poison] = float("nan")
    return c


def run_fwd(c, eps=1e-6, x=None, y=None, h=None, mean=True):
    import torch
    from paper_2509_13232_b200 import binding as B
    T, d = c["T"], c["d"]
    x = c["x"] if x is None else x
    nan = float("nan")
    y = torch.full((T, d), nan, dtype=torch.bfloat16 if c["y16"] else torch.float32, device="cuda") if y is None else y
    if c["residual"] is not None and h is None:
        h = torch.full((T, d), nan, dtype=x.dtype, device="cuda")
    mu = torch.full((T,), nan, device="cuda") if c["kind"] == O.LAYER and mean else None
    rstd = torch.full((T,), nan, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_layernorm_fwd(x, c["residual"], c["weight"], c["bias"], c["mask"], y, h, mu, rstd, st, eps=eps, kind=c["kind"])
    torch.cuda.synchronize()
    return dict(y=y, h=h, mean=mu, rstd=rstd, status=int(st[0]))


def check_fwd(c, got, eps=1e-6):
    d = c["d"]
    f = lambda t: None if t is None else host(t)  # noqa: E731
    with np.errstate(invalid="ignore"):
        want = O.layernorm(f(c["x"]), f(c["weight"]), f(c["bias"]), f(c["residual"]), None if c["mask"] is None else c["mask"].cpu().numpy(),
                           eps, c["kind"], c["x16"])
    K = max(32, -(-d // 1024)) + 40
    live = np.ones(c["T"], bool) if c["mask"] is None else c["mask"].cpu().numpy() != 0
    size = np.abs(want["h"]).mean(axis=1, keepdims=True)
    if c["residual"] is not None:
        assert np.array_equal(host(got["h"]), want["h"])
    slip = K * U * size if c["kind"] == O.LAYER else 0.0
    if got["mean"] is not None:
        assert np.all(np.abs(host(got["mean"]) - want["mean"]) <= slip[:, 0] + U * np.abs(want["mean"]))
    r = want["rstd"][:, None]
    assert np.all(np.abs(host(got["rstd"])[:, None] - r) <= r * ((K + 4) / 2 + 3) * U + r**3 * slip**2)
    xh = (want["h"] - want["mean"][:, None]) * r
    w = 1.0 if c["weight"] is None else np.abs(f(c["weight"]))
    tol = (np.abs(xh) * (K + 4) * U + r * (slip + U * np.abs(want["h"])) + np.abs(xh) * (r * slip)**2) * w
    tol = tol + 2 * U * np.abs(want["y"]) + (half_step(True) * (np.abs(want["y"]) + tol) if c["y16"] else 0.0)
    err = np.abs(host(got["y"]) - want["y"])
    assert np.all(err <= tol), float((err / np.maximum(tol, 1e-300)).max())
    assert got["status"] == 0
    assert np.all(host(got["y"])[~live] == 0) and np.all(host(got["rstd"])[~live] == 0)


WIDTHS = [1, 2, 7, 8, 31, 32, 64, 100, 255, 256, 264, 777, 1000, 1024, 1365, 2048, 2056, 2730, 4096, 4100, 8192, 8200, 10000, 16384, 16392, 20001,
          32768, 32772, 40000]


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("x16", [True, False])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward_of_every_width(d, x16, kind):
    for T in (1, 5, 37):
        for extra in (dict(), dict(residual=True, masked=True, pad=8), dict(pad=3, bias=False, weight=False, y16=not x16)):
            c = case(d + T, T, d, kind, x16, **{"y16": x16, "w16": x16, **extra})
            check_fwd(c, run_fwd(c))


@pytest.mark.parametrize("T", [1, 2, 149, 1000, 70000])
@pytest.mark.parametrize("d", [16, 129])
def test_forward_of_many_rows(T, d):
    c = case(T, T, d, O.LAYER, True, True, False, masked=True, residual=True)
    check_fwd(c, run_fwd(c))


@pytest.mark.parametrize("eps", [1e-12, 1e-5, 0.5])
@pytest.mark.parametrize("d", [40, 3000])
def test_forward_of_rows_far_from_zero(d, eps):
    """The mean is a thousand times the deviations: squares are taken about it, not subtracted from one another."""
    c = case(d, 20, d, O.LAYER, False, False, False, offset=1000.0)
    check_fwd(c, run_fwd(c, eps), eps)


def test_forward_in_place():
    import torch
    for x16 in (True, False):
        for d in (100, 512, 40000):
            c = case(d, 9, d, O.LAYER, x16, x16, True)
            ref = run_fwd(c)
            x = c["x"].clone()
            got = run_fwd(c, x=x, y=x)
            assert torch.equal(got["y"], ref["y"])
            c = case(d, 9, d, O.RMS, x16, x16, True, residual=True, masked=True)
            ref = run_fwd(c)
            x = c["x"].clone()
            got = run_fwd(c, x=x, h=x)
            assert torch.equal(got["h"], ref["h"]) and torch.equal(got["y"], ref["y"])
            c["residual"] = r = c["residual"].clone()
            got = run_fwd(c, h=r)
            assert torch.equal(got["h"], ref["h"]) and torch.equal(got["y"], ref["y"])


def test_rows_without_an_answer():
    import torch
    from paper_2509_13232_b200 import binding as B
    for d in (64, 50, 33000):
        c = case(3, 6, d, O.LAYER, False, False, False)
        c["x"][1, 3], c["x"][4, d - 1], c["x"][5] = float("nan"), float("inf"), 3.25
        got = run_fwd(c)
        assert got["status"] == B.DEV_NONFINITE
        assert bool(torch.isnan(got["y"][1]).all()) and bool(torch.isnan(got["y"][4]).any())
        # a constant row: deviations are zero, y the bias
        np.testing.assert_allclose(host(got["y"])[5], host(c["bias"]), rtol=0, atol=3.25 * 80 * U / np.sqrt(1e-6) * np.abs(host(c["weight"])).max())
        for i in (0, 2, 3):
            assert bool(torch.isfinite(got["y"][i]).all())


def test_no_rows():
    from paper_2509_13232_b200 import binding as B
    import torch
    e = torch.empty(0, 64, device="cuda")
    B.spo_layernorm_fwd(e, None, None, None, None, e.clone(), None, None, None, None)
    dw, db = torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    B.spo_layernorm_bwd(e, e, None, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), None, e.clone(), dw, db, 1, None, None)
    assert float(dw[0]) == 7.0
    B.spo_layernorm_bwd(e, e, None, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), None, e.clone(), dw, db, 0, None, None)
    assert float(dw.abs().sum() + db.abs().sum()) == 0.0


# ------------------------------------------------------------------------------------------------ backward
def run_bwd(c, dy, dh, dw16=False, start=None, dx=None, want=(True, True), x=None, mean=None, rstd=None):
    import torch
    from paper_2509_13232_b200 import binding as B
    T, d = c["T"], c["d"]
    x = c["x"] if x is None else x
    if rstd is None:
        f = {k: None if c[k] is None else host(c[k]) for k in ("x", "weight")}
        with np.errstate(invalid="ignore"):
            s = O.layernorm(f["x"], mask=None if c["mask"] is None else c["mask"].cpu().numpy(), kind=c["kind"])
        mean, rstd = up(s["mean"].astype(np.float32)), up(s["rstd"].astype(np.float32))
    if c["kind"] == O.RMS:
        mean = None
    dx = torch.full((T, d), float("nan"), dtype=x.dtype, device="cuda") if dx is None else dx
    wt = torch.bfloat16 if dw16 else torch.float32
    dw, db = ((torch.full((d,), float("nan"), dtype=wt, device="cuda") if start is None else start[i].clone()) if want[i] else None for i in (0, 1))
    n = B.spo_workspace_bytes(B.WS_LAYERNORM_BWD, T=T, d=d)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    B.spo_layernorm_bwd(dy, x, c["weight"], c["mask"], mean, rstd, dh, dx, dw, db, int(start is not None), ws[:n], None, kind=c["kind"])
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    return dict(dx=dx, dw=dw, db=db, mean=mean, rstd=rstd)


def check_bwd(c, got, dy, dh, dw16=False, start=None):
    T, d = c["T"], c["d"]
    f = lambda t: None if t is None else host(t)  # noqa: E731
    mask = None if c["mask"] is None else c["mask"].cpu().numpy()
    want = O.layernorm_backward(f(dy), f(c["x"]), f(got["mean"]), f(got["rstd"]), f(c["weight"]), f(dh), mask, c["kind"])
    K = max(32, -(-d // 1024)) + 40
    a, xh = want["a"], want["xh"]
    r = np.where(np.ones(T) if mask is None else mask != 0, f(got["rstd"]), 0.0)[:, None]
    part = np.abs(a * xh).mean(axis=1, keepdims=True)
    tol = 4 * U * np.abs(a) + np.abs(xh) * ((K + 4) * U * part + 4 * U * part)
    if c["kind"] == O.LAYER:
        tol = tol + (K + 2) * U * np.abs(a).mean(axis=1, keepdims=True)
    tol = r * tol + 2 * U * np.abs(want["dx"]) + (2 * U * np.abs(np.nan_to_num(f(dh))) if dh is not None else 0.0)
    tol = tol + half_step(c["x16"]) * (np.abs(want["dx"]) + tol)
    err = np.abs(host(got["dx"]) - want["dx"])
    assert np.all(err <= tol), float((err / np.maximum(tol, 1e-300)).max())
    live = np.ones(T, bool) if mask is None else mask != 0
    assert np.all(host(got["dx"])[~live] == 0)
    g = np.where(live[:, None], f(dy), 0.0)
    for name, terms, i in (("dw", g * xh, 0), ("db", g, 1)):
        if got[name] is None:
            continue
        exact = want[name] + (f(start[i]) if start is not None else 0.0)
        tol = 2 * (T / 64 + 100) * U * np.abs(terms).sum(axis=0) + 2 * U * np.abs(exact)
        tol = tol + (half_step(True) * (np.abs(exact) + tol) if dw16 else 0.0)
        err = np.abs(host(got[name]) - exact)
        assert np.all(err <= tol), (name, float((err / np.maximum(tol, 1e-300)).max()))


def grads(seed, c, dy16, with_dh):
    rng = np.random.default_rng(seed)
    dy = up((1e-2 * rng.standard_normal((c["T"], c["d"]))).astype(np.float32), dy16)
    dh = up((1e-2 * rng.standard_normal((c["T"], c["d"]))).astype(np.float32), c["x16"]) if with_dh else None
    if c["mask"] is not None:
        off = c["mask"] == 0
        dy[off] = float("nan")
        if dh is not None:
            dh[off] = float("inf")
    return dy, dh


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("x16", [True, False])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward_of_every_width(d, x16, kind):
    for T in (1, 5, 37):
        for dy16, dh, dw16, extra in ((x16, False, False, {}), (not x16, True, True, dict(masked=True, pad=8)), (False, True, False, dict(weight=False, pad=3))):
            c = case(d + T, T, d, kind, x16, x16, x16, bias=False, **extra)
            dy, dh = grads(d, c, dy16, dh)
            check_bwd(c, run_bwd(c, dy, dh, dw16), dy, dh, dw16)


@pytest.mark.parametrize("T", [2, 149, 1500, 70000])
@pytest.mark.parametrize("d", [16, 200, 1031])
def test_backward_of_many_rows(T, d):
    if T * d > 2 * 10**7:
        T = 20000
    c = case(T, T, d, O.LAYER, True, True, False, masked=True)
    dy, dh = grads(T, c, False, True)
    check_bwd(c, run_bwd(c, dy, dh), dy, dh)


@pytest.mark.parametrize("dw16", [False, True])
@pytest.mark.parametrize("d", [72, 4096, 20000])
def test_backward_adds_to_gradients(d, dw16):
    rng = np.random.default_rng(d)
    c = case(d, 50, d, O.LAYER, True, True, True)
    dy, dh = grads(1, c, True, False)
    start = [up(rng.standard_normal(d).astype(np.float32), dw16) for _ in range(2)]
    check_bwd(c, run_bwd(c, dy, dh, dw16, start), dy, dh, dw16, start)


@pytest.mark.parametrize("d", [100, 512, 20000])
def test_backward_outputs_left_out_and_in_place(d):
    import torch
    c = case(d, 33, d, O.LAYER, True, True, True)
    dy, dh = grads(2, c, True, True)
    ref = run_bwd(c, dy, dh)
    for want in ((True, False), (False, True), (False, False)):
        got = run_bwd(c, dy, dh, want=want)
        assert torch.equal(got["dx"], ref["dx"])
        assert all(got[k] is None or torch.equal(got[k], ref[k]) for k in ("dw", "db"))
    for place in ("dy", "dh", "x"):
        t = dict(dy=dy.clone(), dh=dh.clone(), x=c["x"].clone())
        got = run_bwd(c, t["dy"], t["dh"], dx=t[place], x=t["x"], mean=ref["mean"], rstd=ref["rstd"])
        assert torch.equal(got["dx"], ref["dx"]) and torch.equal(got["dw"], ref["dw"]) and torch.equal(got["db"], ref["db"])


def test_everything_masked():
    import torch
    for d in (96, 20000):
        c = case(1, 12, d, O.RMS, True, True, True, masked=True)
        c["mask"].zero_()
        c["x"].fill_(float("nan"))
        got = run_fwd(c)
        assert got["status"] == 0 and float(got["y"].abs().sum()) == 0
        dy, dh = grads(2, c, True, True)
        back = run_bwd(c, dy, dh, mean=None, rstd=torch.full((12,), float("nan"), device="cuda"))
        assert all(float(back[k].float().abs().sum()) == 0 for k in ("dx", "dw", "db"))


def test_gradients_by_differences():
    """dx, dw and db of the kernels against differences of the float64 forward pass."""
    rng = np.random.default_rng(5)
    T, d = 4, 24
    c = case(9, T, d, O.LAYER, False, False, False)
    f = run_fwd(c, eps=1e-2)
    dy, dh = grads(3, c, False, True)
    got = run_bwd(c, dy, dh, mean=f["mean"], rstd=f["rstd"])
    x, w, b, g, gh = (host(t) for t in (c["x"], c["weight"], c["bias"], dy, dh))

    def value(x, w, b):
        return float((O.layernorm(x, w, b, eps=1e-2)["y"] * g).sum() + (x * gh).sum())

    for name, at in (("dx", 0), ("dw", 1), ("db", 2)):
        args = [x, w, b]
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in args[at].shape)
            s = np.zeros_like(args[at])
            s[i] = 1e-4
            hi, lo = list(args), list(args)
            hi[at], lo[at] = args[at] + s, args[at] - s
            assert abs((value(*hi) - value(*lo)) / 2e-4 - host(got[name])[i]) < 1e-6


def test_results_repeat_and_do_not_depend_on_the_stream():
    import torch
    c = case(1, 3000, 520, O.LAYER, True, True, True, masked=True)
    dy, dh = grads(1, c, True, True)
    ref = run_bwd(c, dy, dh)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = run_bwd(c, dy, dh, mean=ref["mean"], rstd=ref["rstd"])
        assert all(torch.equal(got[k], ref[k]) for k in ("dx", "dw", "db"))


def test_captured_and_replayed_with_other_rows():
    import torch
    from paper_2509_13232_b200 import binding as B
    T, d = 300, 1000
    c = [case(s, T, d, O.LAYER, True, True, True) for s in (1, 2)]
    x, dy = c[0]["x"].contiguous(), grads(1, c[0], True, False)[0]
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(B.spo_workspace_bytes(B.WS_LAYERNORM_BWD, T=T, d=d), dtype=torch.uint8, device="cuda")
    w, b = c[0]["weight"], c[0]["bias"]

    def both():
        B.spo_layernorm_fwd(x, None, w, b, None, y, None, mean, rstd, None)
        B.spo_layernorm_bwd(dy, x, w, None, mean, rstd, None, dx, dw, db, 0, ws, None)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.copy_(c[1]["x"])
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (y, dx, dw, db)]
    both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw, db)))


def test_the_binding_refuses():
    import torch
    from paper_2509_13232_b200 import binding as B
    x, y = torch.zeros(4, 32, device="cuda"), torch.zeros(4, 32, device="cuda")
    v, r = torch.zeros(32, device="cuda"), torch.zeros(4, device="cuda")
    ok = dict(x=x, residual=None, weight=v, bias=v.clone(), mask=None, y=y, h=None, mean=r, rstd=r.clone(), d_status=None)
    B.spo_layernorm_fwd(**ok)
    for bad, err in ((dict(x=x.cpu()), ValueError), (dict(x=x.half()), TypeError), (dict(x=x.t()), ValueError), (dict(x=v), ValueError),
                     (dict(weight=v[:16]), ValueError), (dict(weight=v.bfloat16()), TypeError), (dict(weight=v.half(), bias=None), TypeError),
                     (dict(y=y.t()), ValueError), (dict(y=torch.zeros(4, 64, device="cuda")[:, ::2]), ValueError), (dict(mean=r.double()), TypeError),
                     (dict(mask=torch.ones(4, dtype=torch.bool, device="cuda")), TypeError), (dict(residual=y.clone()), B.SpoError),
                     (dict(residual=y.clone(), h=y.bfloat16()), TypeError), (dict(x=torch.zeros(1, 32, device="cuda").expand(4, 32)), ValueError),
                     (dict(eps=0.0), B.SpoError), (dict(kind=2), B.SpoError), (dict(kind=B.NORM_RMS), B.SpoError)):
        with pytest.raises(err):
            B.spo_layernorm_fwd(**{**ok, **bad})
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    back = dict(dy=y, x=x, weight=v, mask=None, mean=r, rstd=r.clone(), dh=None, dx=torch.zeros_like(x), dw=v.clone(), db=v.clone(), dw_accumulate=0, ws=ws,
                d_status=None)
    B.spo_layernorm_bwd(**back)
    for bad, err in ((dict(ws=ws[:64]), B.SpoError), (dict(ws=None), B.SpoError), (dict(dw=v.bfloat16()), TypeError), (dict(dx=y.bfloat16()), TypeError),
                     (dict(dy=y[:3]), ValueError), (dict(rstd=None), TypeError), (dict(mean=None), B.SpoError), (dict(dw=v), B.SpoError),
                     (dict(db=back["dw"]), B.SpoError)):
        with pytest.raises(err):
            B.spo_layernorm_bwd(**{**back, **bad})
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,pad", [(4096, 0), (1000, 0), (2730, 0), (1365, 3), (8192, 0)])
def test_masked_rows_between_others(d, pad):
    """A masked row takes no part in its block's exchange of partial sums; the rows around it come out as in a batch without it, bit
    for bit, however the masked ones lie."""
    import torch
    from paper_2509_13232_b200 import binding as B
    T = 6000
    c = case(d, T, d, O.LAYER, True, True, True, pad=pad)
    dy, dh = grads(1, c, False, True)
    whole, back = run_fwd(c), run_bwd(c, dy, dh)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    for pattern in (torch.arange(T, device="cuda") % 2, torch.arange(T, device="cuda") // 4 % 2, torch.rand(T, generator=g, device="cuda") < 0.5):
        c["mask"] = pattern.to(torch.uint8)
        on = c["mask"] != 0
        for _ in range(3):
            got = run_fwd(c)
            assert torch.equal(got["y"][on], whole["y"][on]) and torch.equal(got["rstd"][on], whole["rstd"][on]) and got["status"] == 0
            assert float(got["y"][~on].abs().sum()) == 0
            b = run_bwd(c, dy, dh, mean=back["mean"], rstd=back["rstd"])
            assert torch.equal(b["dx"][on], back["dx"][on]) and float(b["dx"][~on].abs().sum()) == 0
