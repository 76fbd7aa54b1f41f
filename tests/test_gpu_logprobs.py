"""GPU parity of spo_logprobs / spo_logprobs_bwd with the float64 definitions.

Tolerances, derived before any run.  A logit is a sum of d products of exact inputs in fp32: its error is at most
eps_z = (d/16 + 2) 2^-23 max_tv sum_k |h_tk w_vk| (one rounding or truncation per 16 products).  lse and logp add the
rounding of the exponentials and of their sum, relative (V/32 + 64) 2^-24 + 2^-21 (chains of at most V/32 + 64 additions,
ex2.approx within 2^-22, twice), and a few roundings of numbers of lse's size.  The entropy weights such errors with |z|.
A stored gradient of a logit is off by 2^-8 (half a bf16 step, relative) plus its exponential's relative error, so an
entry of dH by that times sum_v |dz_tv| |w_vk|, and a bf16 result by another 2^-8 of itself.
"""

import numpy as np
import pytest

from oracle import operators as O
from paper_2509_13232_b200 import inputs

pytestmark = pytest.mark.gpu


def make(seed, T, d, V, bf16=True, grid=False, w_std=0.08):
    rng = np.random.default_rng(seed)
    h = rng.standard_normal((T, d)).astype(np.float32)
    w = (rng.standard_normal((V, d)) * w_std).astype(np.float32)
    if grid:           # every logit an exact fp32 sum whatever its order: the alternatives are the definition's
        h = np.clip(np.round(h * 32) / 32, -7.75, 7.75).astype(np.float32)
        w = (np.round(w * 256) / 256).astype(np.float32)
    if bf16:
        h, w = inputs.round_to_bf16(h), inputs.round_to_bf16(w)
    y = rng.integers(0, V, T).astype(np.int32)
    return h, w, y, rng


def tolerances(h, w, inv_t, want):
    d, V = h.shape[1], w.shape[0]
    if h.shape[0] == 0:
        return 0.0, 0.0, 0.0
    eps_z = (d / 16 + 2) * 2.0**-23 * float((np.abs(h).astype(np.float64) @ np.abs(w).astype(np.float64).T).max())
    size = max(float(np.abs(want["lse"]).max()), inv_t * float(np.abs(want["z"]).max()))
    rel = (V / 32 + 64) * 2.0**-24 + 2.0**-21
    tol = 2 * inv_t * eps_z + rel + 8 * 2.0**-24 * size
    return eps_z, tol, tol + 2 * (inv_t * eps_z + rel) * (size + 1)


def call_fwd(h, w, y, mask, K, inv_t, bf16=True, entropy=True, ld_pad=0, stream=None):
    import torch
    from paper_2509_13232_b200 import binding as B
    dt = torch.bfloat16 if bf16 else torch.float32
    T, d = h.shape
    wide = torch.full((max(T, 1), d + ld_pad), float("nan"), dtype=dt, device="cuda")
    wide[:T, :d] = torch.from_numpy(h).cuda().to(dt)
    H, W = wide[:T, :d], torch.from_numpy(w).cuda().to(dt)
    V = w.shape[0]
    yt = None if y is None else torch.from_numpy(y).cuda()
    mt = None if mask is None else torch.from_numpy(mask).cuda()
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    logp, lse, ent = nan(T) if y is not None else None, nan(T), nan(T) if entropy else None
    ids = torch.full((T, K), -7, dtype=torch.int32, device="cuda") if K else None
    tl = nan(T, K) if K else None
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    n = B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=d, V=V, B=K)
    ws = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")      # scratch holds anything
    torch.cuda.synchronize()
    B.spo_logprobs(H, W, yt, mt, logp, lse, ent, ids, tl, ws[:n] if n else ws, st, inv_temperature=inv_t)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xA5).all())
    get = lambda x: None if x is None else x.cpu().numpy()  # noqa: E731
    return dict(logp=get(logp), lse=get(lse), entropy=get(ent), top_ids=get(ids), top_logp=get(tl), status=int(st[0]))


def check_fwd(got, want, h, w, inv_t, K, exact_ids):
    _, tol, tol_ent = tolerances(h, w, inv_t, want)
    np.testing.assert_allclose(got["lse"], want["lse"], rtol=0, atol=tol)
    if got["logp"] is not None:
        np.testing.assert_allclose(got["logp"], want["logp"], rtol=0, atol=tol)
    if got["entropy"] is not None:
        np.testing.assert_allclose(got["entropy"], want["entropy"], rtol=0, atol=tol_ent)
    if K:
        np.testing.assert_allclose(got["top_logp"], want["top_logp"], rtol=0, atol=tol)
        if exact_ids:
            np.testing.assert_array_equal(got["top_ids"], want["top_ids"])


FWD = [
    # T, d, V, top_k, temperature, masked, row padding
    (1, 64, 1, 1, 1.0, False, 0),
    (1, 64, 7, 3, 1.0, False, 8),
    (1, 4096, 3001, 20, 1.0, False, 0),
    (2, 128, 512, 8, 0.7, False, 64),
    (16, 192, 1000, 9, 1.0, True, 0),
    (17, 64, 513, 5, 1.3, False, 0),
    (33, 128, 20000, 20, 1.0, False, 0),
    (64, 64, 31, 20, 1.0, True, 8),
    (100, 320, 2049, 1, 1.0, False, 0),
    (128, 128, 5000, 8, 0.9, False, 0),
    (129, 64, 20, 20, 1.0, False, 0),
    (129, 128, 5000, 8, 0.9, True, 16),
    (257, 192, 513, 20, 1.0, False, 0),
    (300, 64, 12345, 9, 1.0, False, 0),
    (700, 256, 3000, 0, 1.0, True, 0),
    (1300, 64, 1, 1, 1.0, False, 0),
    (19001, 64, 300, 4, 1.0, False, 0),
]


@pytest.mark.parametrize("T,d,V,K,temp,masked,pad", FWD)
def test_bf16_forward(T, d, V, K, temp, masked, pad):
    h, w, y, rng = make(T * 7 + d + V, T, d, V, grid=True)
    mask = (rng.random(T) < 0.7).astype(np.uint8) if masked else None
    inv_t = float(np.float32(1.0 / temp))
    want = O.logprobs(h, w, y, mask, inv_t, K)
    got = call_fwd(h, w, y, mask, K, inv_t, ld_pad=pad)
    assert got["status"] == 0
    check_fwd(got, want, h, w, inv_t, K, True)


@pytest.mark.parametrize("T,d,V,K,temp,masked,pad", [c for c in FWD if c[0] < 1000] + [(5, 4, 33, 2, 1.0, False, 4),
                                                                                   (70, 100, 4099, 20, 2.0, True, 0)])
def test_fp32_forward(T, d, V, K, temp, masked, pad):
    h, w, y, rng = make(T * 5 + d + V, T, d, V, bf16=False, grid=True)
    mask = (rng.random(T) < 0.7).astype(np.uint8) if masked else None
    inv_t = float(np.float32(1.0 / temp))
    want = O.logprobs(h, w, y, mask, inv_t, K)
    got = call_fwd(h, w, y, mask, K, inv_t, bf16=False, ld_pad=pad)
    assert got["status"] == 0
    check_fwd(got, want, h, w, inv_t, K, True)


@pytest.mark.parametrize("T,bf16", [(3, True), (200, True), (40, False)])
def test_random_inputs_without_a_grid(T, bf16):
    h, w, y, _ = make(99 + T, T, 512, 4000, bf16=bf16)
    want = O.logprobs(h, w, y, None, 1.0, 8)
    got = call_fwd(h, w, y, None, 8, 1.0, bf16=bf16)
    check_fwd(got, want, h, w, 1.0, 8, False)
    # the listed tokens are the ones their log-probs say
    logq = want["z"] - want["lse"][:, None]
    _, tol, _ = tolerances(h, w, 1.0, want)
    np.testing.assert_allclose(np.take_along_axis(logq, got["top_ids"].astype(np.int64), 1), got["top_logp"], rtol=0, atol=tol)


@pytest.mark.parametrize("T,bf16", [(4, True), (150, True), (9, False)])
def test_equal_logits_are_listed_by_ascending_id(T, bf16):
    d, V, K = 64, 3000, 20
    rng = np.random.default_rng(T)
    h = np.ones((T, d), np.float32)
    w = np.repeat(rng.integers(-3, 4, (V, 1)), d, axis=1).astype(np.float32) / 64      # seven distinct logits
    w[1000:1300] = w[0:300]
    got = call_fwd(h, w, np.zeros(T, np.int32), None, K, 1.0, bf16=bf16)
    want = O.logprobs(h, w, np.zeros(T, np.int32), None, 1.0, K)
    np.testing.assert_array_equal(got["top_ids"], want["top_ids"])
    for order in (1, -1):                       # all groups enter every list, in ascending logits; then none after the first
        w2 = np.sort(w[:, :1], axis=0)[::order].repeat(d, axis=1).copy()
        got = call_fwd(h, w2, None, None, K, 1.0, bf16=bf16)
        np.testing.assert_array_equal(got["top_ids"], O.logprobs(h, w2, None, None, 1.0, K)["top_ids"])


@pytest.mark.parametrize("T,bf16", [(6, True), (180, True), (50, False)])
def test_masked_rows_may_hold_anything(T, bf16):
    import torch  # noqa: F401
    h, w, y, rng = make(5 + T, T, 64, 700, bf16=bf16, grid=True)
    mask = np.ones(T, np.uint8)
    mask[::3] = 0
    h[::3] = np.nan
    h[3::6] = np.inf
    y[::3] = -100
    clean = np.where(mask[:, None] != 0, h, 0.0)
    want = O.logprobs(clean, w, y, mask, 1.0, 5)
    got = call_fwd(h, w, y, mask, 5, 1.0, bf16=bf16)
    assert got["status"] == 0
    check_fwd(got, want, clean, w, 1.0, 5, True)
    mask[:] = 0                                 # nothing left at all
    got = call_fwd(h, w, y, mask, 5, 1.0, bf16=bf16)
    assert got["status"] == 0 and np.all(got["lse"] == 0) and np.all(got["logp"] == 0) and np.all(got["top_ids"] == -1)


@pytest.mark.parametrize("T,bf16", [(6, True), (180, True), (50, False)])
def test_bad_targets_and_bad_rows_are_reported(T, bf16):
    from paper_2509_13232_b200 import binding as B
    h, w, y, _ = make(6 + T, T, 64, 700, bf16=bf16, grid=True)
    y[1], y[2] = 700, -1
    got = call_fwd(h, w, y, None, 3, 1.0, bf16=bf16)
    assert got["status"] == B.DEV_ID_OUT_OF_RANGE
    assert np.all(np.isneginf(got["logp"][1:3])) and np.all(np.isfinite(got["logp"][3:]))
    y[1:3] = 0
    h[4] = np.nan
    got = call_fwd(h, w, y, None, 3, 1.0, bf16=bf16)
    assert got["status"] == B.DEV_NONFINITE
    assert np.isnan(got["lse"][4]) and np.all(got["top_ids"][4] == -1)
    keep = np.arange(T) != 4
    want = O.logprobs(h[keep], w, y[keep], None, 1.0, 3)
    np.testing.assert_array_equal(got["top_ids"][keep], want["top_ids"])
    np.testing.assert_allclose(got["logp"][keep], want["logp"], rtol=0, atol=1e-4)


def test_no_rows():
    got = call_fwd(np.zeros((0, 64), np.float32), np.zeros((5, 64), np.float32), np.zeros(0, np.int32), None, 2, 1.0)
    assert got["status"] == 0 and got["lse"].shape == (0,)


# ------------------------------------------------------------------------------------------------ backward
def call_bwd(h, w, y, mask, lse, ent, gl, gs, ge, inv_t, bf16=True, dh32=False, dw32=False, dw_init=None, ld_pad=0):
    import torch
    from paper_2509_13232_b200 import binding as B
    dt = torch.bfloat16 if bf16 else torch.float32
    T, d = h.shape
    V = w.shape[0]
    wide = torch.full((max(T, 1), d + ld_pad), float("nan"), dtype=dt, device="cuda")
    wide[:T, :d] = torch.from_numpy(h).cuda().to(dt)
    H, W = wide[:T, :d], torch.from_numpy(w).cuda().to(dt)
    up = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()  # noqa: E731
    yt = None if y is None else torch.from_numpy(y).cuda()
    mt = None if mask is None else torch.from_numpy(mask).cuda()
    dH = torch.full((T, d), float("nan"), dtype=torch.float32 if dh32 or not bf16 else dt, device="cuda")
    wdt = torch.float32 if dw32 or not bf16 else dt
    dW = torch.full((V, d), float("nan"), dtype=wdt, device="cuda") if dw_init is None else up(dw_init).to(wdt)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    n = B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=T, d=d, V=V)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    B.spo_logprobs_bwd(H, W, yt, mt, up(lse), up(ent), up(gl), up(gs), up(ge), dH, dW, int(dw_init is not None), ws[:n], st,
                       inv_temperature=inv_t)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    return dH.float().cpu().numpy(), dW.float().cpu().numpy(), int(st[0])


def check_bwd(got_dh, got_dw, want, h, w, mask, inv_t, fwd, bf16, dh32, dw32, dw_init=None):
    dh, dw, size = want
    _, tol, _ = tolerances(h, w, inv_t, fwd)
    slip = (2.0**-8 if bf16 else 0.0) + 2 * tol + 2.0**-20     # relative error of a stored dz, against its terms
    on = np.ones(len(h)) if mask is None else (mask != 0).astype(np.float64)
    hh = np.abs(np.where(on[:, None] > 0, h, 0.0)).astype(np.float64)
    sums_v, sums_t = (w.shape[0] + 64) * 2.0**-24, (h.shape[0] + 64) * 2.0**-24      # fp32 accumulation
    bound_h = (slip + sums_v) * (size @ np.abs(w).astype(np.float64)) + (0 if dh32 or not bf16 else 2.0**-8) * np.abs(dh) + 1e-30
    bound_w = (slip + sums_t) * (size.T @ hh) + (0 if dw32 or not bf16 else 2.0**-8) * (np.abs(dw)) + 1e-30
    if dw_init is not None:
        dw = dw + dw_init
        bound_w = bound_w + (2.0**-8 if bf16 and not dw32 else 2.0**-23) * (np.abs(dw) + np.abs(dw_init))
    assert np.all(np.abs(got_dh - dh) <= bound_h)
    assert np.all(np.abs(got_dw - dw) <= bound_w)


BWD = [
    # T, d, V, temperature, masked, (logp, lse, entropy) gradients, dH fp32, dW fp32, accumulate, padding
    (1, 64, 1, 1.0, False, (1, 1, 1), False, False, False, 0),
    (1, 64, 300, 1.0, False, (1, 0, 0), False, True, False, 8),
    (40, 128, 513, 0.7, True, (1, 1, 1), False, False, False, 64),
    (200, 192, 1000, 1.0, False, (0, 0, 1), True, False, True, 0),
    (257, 64, 2049, 1.2, True, (1, 0, 1), False, True, True, 8),
    (700, 320, 700, 1.0, False, (0, 1, 0), False, False, False, 0),
    (9700, 64, 300, 1.0, True, (1, 1, 1), False, False, False, 0),      # more rows than one chunk
    (9700, 64, 260, 1.0, False, (1, 0, 1), True, True, True, 0),
    (9700, 64, 260, 1.0, False, (1, 0, 1), False, False, True, 0),
]


def upstream(rng, T, which):
    g = rng.standard_normal((3, T)).astype(np.float32)
    return [g[i] if which[i] else None for i in range(3)]


@pytest.mark.parametrize("T,d,V,temp,masked,which,dh32,dw32,acc,pad", BWD)
def test_bf16_backward(T, d, V, temp, masked, which, dh32, dw32, acc, pad):
    h, w, y, rng = make(T + d + V, T, d, V)
    mask = (rng.random(T) < 0.6).astype(np.uint8) if masked else None
    inv_t = float(np.float32(1.0 / temp))
    fwd = O.logprobs(h, w, y, None, inv_t)
    gl, gs, ge = upstream(rng, T, which)
    init = inputs.round_to_bf16(rng.standard_normal((V, d)).astype(np.float32)) if acc else None
    want = O.logprobs_backward(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge, inv_t)
    if mask is not None:
        h = np.where(mask[:, None] != 0, h, np.nan).astype(np.float32)
    dh, dw, st = call_bwd(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge, inv_t, dh32=dh32, dw32=dw32, dw_init=init,
                          ld_pad=pad)
    assert st == 0
    h = np.nan_to_num(h)
    check_bwd(dh, dw, want, h, w, mask, inv_t, fwd, True, dh32, dw32, init)


@pytest.mark.parametrize("T,d,V,temp,masked,which,dh32,dw32,acc,pad",
                         [c for c in BWD if c[0] < 1000] + [(33, 100, 77, 1.0, True, (1, 1, 1), 0, 0, False, 4),
                                                            (90, 64, 9001, 1.0, False, (1, 0, 1), 0, 0, True, 0)])
def test_fp32_backward(T, d, V, temp, masked, which, dh32, dw32, acc, pad):
    h, w, y, rng = make(T + d + V + 1, T, d, V, bf16=False)
    mask = (rng.random(T) < 0.6).astype(np.uint8) if masked else None
    inv_t = float(np.float32(1.0 / temp))
    fwd = O.logprobs(h, w, y, None, inv_t)
    gl, gs, ge = upstream(rng, T, which)
    init = rng.standard_normal((V, d)).astype(np.float32) if acc else None
    want = O.logprobs_backward(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge, inv_t)
    if mask is not None:
        h = np.where(mask[:, None] != 0, h, np.nan).astype(np.float32)
    dh, dw, st = call_bwd(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge, inv_t, bf16=False, dw_init=init, ld_pad=pad)
    assert st == 0
    check_bwd(dh, dw, want, np.nan_to_num(h), w, mask, inv_t, fwd, False, True, True, init)


@pytest.mark.parametrize("bf16", [True, False])
def test_backward_of_bad_targets_and_of_no_rows(bf16):
    from paper_2509_13232_b200 import binding as B
    h, w, y, rng = make(3, 20, 64, 90, bf16=bf16)
    y[0], y[1] = 90, -100
    mask = np.ones(20, np.uint8)
    mask[1] = 0
    fwd = O.logprobs(h, w, y, None, 1.0)
    gl, gs, ge = upstream(rng, 20, (1, 1, 1))
    want = O.logprobs_backward(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge)
    dh, dw, st = call_bwd(h, w, y, mask, fwd["lse"], fwd["entropy"], gl, gs, ge, 1.0, bf16=bf16)
    assert st == B.DEV_ID_OUT_OF_RANGE and np.all(dh[1] == 0)
    check_bwd(dh, dw, want, h, w, mask, 1.0, fwd, bf16, False, False)
    none = np.zeros(0, np.float32)
    for init in (None, np.ones((90, 64), np.float32)):
        _, dw, st = call_bwd(h[:0], w, y[:0], None, none, None, none, None, None, 1.0, bf16=bf16, dw_init=init)
        assert st == 0 and np.all(dw == (0 if init is None else 1))


@pytest.mark.parametrize("T,d,V,targets,masked,dh32,dw32,acc", [
    (1, 64, 1000, 1, False, False, False, False),
    (1, 2112, 600, 1, False, True, True, False),
    (5, 128, 3000, 2, False, True, False, True),
    (40, 64, 900, 7, True, False, True, True),
    (300, 192, 520, 1, False, True, True, False),          # one target for all
    (2500, 64, 300, 40, True, True, False, False),
    (9700, 64, 260, 3, True, True, True, False),           # more rows than one chunk
    (9700, 64, 260, 260, False, False, False, True),
])
def test_the_targets_entry_is_not_rounded(T, d, V, targets, masked, dh32, dw32, acc):
    """Upstream gradients that put every target's entry half way between two bf16 numbers: its term keeps 32 bits, so only
    the other entries' roundings are left, whose terms carry p."""
    h, w, y, rng = make(T + V, T, d, V, w_std=0.02)
    y = rng.integers(0, targets, T).astype(np.int32) * (V // targets)
    mask = (rng.random(T) < 0.7).astype(np.uint8) if masked else None
    if masked:
        mask[0] = 1
    fwd = O.logprobs(h, w, y, None, 1.0)
    gl = ((1 + 2.0**-8) / -np.expm1(fwd["logp"])).astype(np.float32)
    on = np.ones(T) if mask is None else (mask != 0).astype(np.float64)
    init = rng.standard_normal((V, d)).astype(np.float32) if acc else None
    if acc and not dw32:
        init = np.round(init * 16) / 16                    # exact in bf16
    dh, dw, _ = O.logprobs_backward(h, w, y, mask, fwd["lse"], None, gl, None, None, 1.0)
    got_dh, got_dw, st = call_bwd(h, w, y, mask, fwd["lse"], None, gl, None, None, 1.0, dh32=dh32, dw32=dw32, dw_init=init)
    assert st == 0
    _, tol, _ = tolerances(h, w, 1.0, fwd)
    p = np.exp(h.astype(np.float64) @ w.T.astype(np.float64) - fwd["lse"].astype(np.float64)[:, None]) * (gl * on)[:, None]
    slack = (2 * tol + 2.0**-20) * p                       # of a term in p, as elsewhere, and its rounding to bf16
    slack = slack + 2.0**-8 * p * (np.arange(V)[None, :] != y[:, None])
    slack[np.arange(T), y] += 2.0**-22 * gl * on           # the target's entry: rounded to 32 bits twice
    size = p.copy()
    size[np.arange(T), y] += gl * on
    aw, ah = np.abs(w).astype(np.float64), np.abs(h).astype(np.float64)
    bound_h = slack @ aw + (V + 64) * 2.0**-24 * (size @ aw) + (0 if dh32 else 2.0**-8) * np.abs(dh)
    bound_w = slack.T @ ah + (T + 64) * 2.0**-24 * (size.T @ ah)
    if not dw32:                                           # the rest of the target's term (2^-8 of it) goes through bf16
        bound_w = bound_w + 2.0**-16 * (size.T @ ah)
    if acc:
        dw = dw + init
        bound_w = bound_w + 2.0**-23 * (np.abs(dw) + np.abs(init))
    bound_w = bound_w + (0 if dw32 else 2.0**-8) * np.abs(dw)
    assert np.all(np.abs(got_dh - dh) <= bound_h)
    assert np.all(np.abs(got_dw - dw) <= bound_w)


def test_gradients_match_differences_of_the_forward():
    """Central differences of the library's own fp32 forward along a random direction of H and of W."""
    T, d, V, inv_t = 12, 32, 50, 0.8
    h, w, y, rng = make(11, T, d, V, bf16=False, w_std=0.3)
    gl, gs, ge = upstream(rng, T, (1, 1, 1))
    fwd = call_fwd(h, w, y, None, 0, inv_t, bf16=False)
    dh, dw, _ = call_bwd(h, w, y, None, fwd["lse"], fwd["entropy"], gl, gs, ge, inv_t, bf16=False)

    def value(hh, ww):
        o = call_fwd(hh.astype(np.float32), ww.astype(np.float32), y, None, 0, inv_t, bf16=False)
        return float((gl * o["logp"].astype(np.float64) + gs * o["lse"] + ge * o["entropy"]).sum())

    step = 2.0**-6
    for x, dx, which in ((h, dh, 0), (w, dw, 1)):
        v = np.round(rng.standard_normal(x.shape) * 8).astype(np.float32) / 8
        hi, lo = (value(h + s * v, w) if which == 0 else value(h, w + s * v) for s in (step, -step))
        slope = float((dx.astype(np.float64) * v).sum())
        # the third-order term of the difference, and the forward's rounding over the step
        mid = [value(h + s * v, w) if which == 0 else value(h, w + s * v) for s in (2 * step, -2 * step)]
        third = abs((mid[0] - mid[1]) / (4 * step) - (hi - lo) / (2 * step))
        assert abs((hi - lo) / (2 * step) - slope) <= third + T * 4e-6 / step


# ------------------------------------------------------------------------------------------------ how it is called
def test_other_stream_graph_replay_and_two_calls_at_once():
    import torch
    from paper_2509_13232_b200 import binding as B
    T, d, V, K = 37, 128, 3000, 5
    h, w, y, _ = make(21, T, d, V, grid=True)
    big = make(22, 300, d, V, grid=True)
    W = torch.from_numpy(w).cuda().bfloat16()

    def buffers(T):
        n = B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=d, V=V, B=K)
        f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
        return (f(T), f(T), f(T), torch.zeros(T, K, dtype=torch.int32, device="cuda"), f(T, K),
                torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"))

    H1, y1, o1 = torch.from_numpy(h).cuda().bfloat16(), torch.from_numpy(y).cuda(), buffers(T)
    H2, y2, o2 = torch.from_numpy(big[0]).cuda().bfloat16(), torch.from_numpy(big[2]).cuda(), buffers(300)
    B.spo_logprobs(H1, W, y1, None, *o1)
    B.spo_logprobs(H2, W, y2, None, *o2)
    torch.cuda.synchronize()
    ref1, ref2 = [x.clone() for x in o1[:5]], [x.clone() for x in o2[:5]]
    # two calls at once on two streams
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for x in o1[:5] + o2[:5]:
        x.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            B.spo_logprobs(H1, W, y1, None, *o1)
        with torch.cuda.stream(s2):
            B.spo_logprobs(H2, W, y2, None, *o2)
    torch.cuda.synchronize()
    for got, ref in zip(o1[:5] + o2[:5], ref1 + ref2):
        assert torch.equal(got, ref)
    # captured, then replayed on other values
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.spo_logprobs(H1, W, y1, None, *o1)
        B.spo_logprobs(H2, W, y2, None, *o2)
    H1.copy_(H2[:T])
    y1.copy_(y2[:T])
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o1[3], ref2[3][:T])
    np.testing.assert_allclose(o1[0].cpu(), ref2[0][:T].cpu(), rtol=0, atol=1e-5)
    for got, ref in zip(o2[:5], ref2):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("T", [37, 300])
def test_captured_backward_with_other_targets_at_each_replay(T):
    """What a call keeps in its scratch by target (rows, slots) is its own: replays with new targets, masks and gradients
    give the bits of fresh calls on scratch full of ones."""
    import torch
    from paper_2509_13232_b200 import binding as B
    d, V = 128, 700
    h, w, y, rng = make(31, T, d, V)
    H, W = torch.from_numpy(h).cuda().bfloat16(), torch.from_numpy(w).cuda().bfloat16()
    lse = torch.from_numpy(O.logprobs(h, w, y, None, 1.0)["lse"].astype(np.float32)).cuda()
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    n = B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=T, d=d, V=V)
    ws, fresh = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda")
    Y, M = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.ones(T, dtype=torch.uint8, device="cuda")
    gl = torch.ones(T, device="cuda")
    dH, dW, dH1, dW1 = (torch.empty_like(x) for x in (H, W, H, W))
    call = lambda a, b, s: B.spo_logprobs_bwd(H, W, Y, M, lse, None, gl, None, None, a, b, 0, s, st)  # noqa: E731
    call(dH, dW, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(dH, dW, ws)
    for k, targets in enumerate((V, 5, 1, V)):
        Y.copy_(torch.from_numpy(rng.integers(0, targets, T).astype(np.int32)))
        M.copy_(torch.from_numpy((rng.random(T) < 0.6 + 0.1 * k).astype(np.uint8)))
        gl.copy_(torch.from_numpy(rng.standard_normal(T).astype(np.float32)))
        dH.fill_(float("nan")), dW.fill_(float("nan"))
        g.replay()
        fresh.fill_(0xFF)
        call(dH1, dW1, fresh)
        torch.cuda.synchronize()
        assert torch.equal(dH, dH1) and torch.equal(dW, dW1) and int(st[0]) == 0


def test_old_log_probs_agree_with_the_loss_calls():
    """spo_logprobs feeds logp_old of the loss: with the same weights every ratio is one."""
    import torch
    from paper_2509_13232_b200 import binding as B
    from tests.helpers import run_loss
    lb = inputs.loss_batch(40, [300, 90, 57], 128, 1500, 0.05, True, 0.3, target="softmax")
    got = call_fwd(lb.h, lb.w, lb.y, None, 0, 1.0)
    lb.logp_old = got["logp"]
    out = run_loss(lb, one_pass=True, want_entropy=True)
    np.testing.assert_allclose(out["logp"], got["logp"], rtol=0, atol=2e-5)
    np.testing.assert_allclose(out["entropy"], got["entropy"], rtol=0, atol=2e-4)
    a = np.repeat(lb.a_norm, np.diff(lb.cu_seqlens))
    assert abs(out["loss"] + float(a.mean())) < 1e-4
    # and its backward with g_logp = coef gives the loss's gradients
    dh, dw, _ = call_bwd(lb.h, lb.w, lb.y, None, out["lse"], None, out["coef"], None, None, 1.0, dw32=True)
    for x, z in ((dh, out["dH"]), (dw, out["dW"])):
        assert np.linalg.norm(x - z) <= 2 * 2.0**-8 * np.linalg.norm(z)
    assert torch.cuda.is_available() and B.MAX_TOP_K == 20
