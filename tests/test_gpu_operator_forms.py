"""The forms that the operators around the loss take at the sizes of a large configuration: wide tiles (more than 1024 features), the
rungs of the streaming kernel, vocabularies of 20 000 and more, fp32 batches of several chunks, tall weight matrices.  The definitions
are evaluated in 64 bits on the GPU, elementary operation by elementary operation; tolerances are those of test_gpu_logprobs."""

import numpy as np
import pytest

from paper_2509_13232_b200 import inputs

pytestmark = pytest.mark.gpu


def data(seed, T, d, V, bf16, w_std, grid):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    h = torch.randn(T, d, generator=g, device="cuda")
    w = torch.randn(V, d, generator=g, device="cuda") * w_std
    if grid:           # every logit an exact fp32 sum whatever its order: the alternatives are the definition's
        h, w = (h * 32).round().div(32).clamp(-7.75, 7.75), (w * 256).round() / 256
    dt = torch.bfloat16 if bf16 else torch.float32
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    return h.to(dt), w.to(dt), y, g


def slack(H, W, inv_t, lse):
    """(tol of a log-prob, of an entropy): see test_gpu_logprobs.tolerances."""
    d, V = W.shape[1], W.shape[0]
    a = H.double().abs() @ W.double().abs().T
    eps_z = (d / 16 + 2) * 2.0**-23 * float(a.max())
    size = max(float(lse.abs().max()), inv_t * float((H.double() @ W.double().T).abs().max()))
    rel = (V / 32 + 64) * 2.0**-24 + 2.0**-21
    tol = 2 * inv_t * eps_z + rel + 8 * 2.0**-24 * size
    return tol, tol + 2 * (inv_t * eps_z + rel) * (size + 1)


def forward64(H, W, y, inv_t, K):
    import torch
    raw = H.double() @ W.double().T
    lse = torch.logsumexp(raw * inv_t, 1)
    lp = raw * inv_t - lse[:, None]
    ids = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :K]
    return dict(lse=lse, logp=lp.gather(1, y.long()[:, None])[:, 0], entropy=-(lp.exp() * lp).sum(1), top_ids=ids.int(),
                top_logp=lp.gather(1, ids))


def forward(H, W, y, K, entropy, inv_t):
    import torch
    from paper_2509_13232_b200 import binding as B
    (T, d), V = H.shape, W.shape[0]
    f = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    out = dict(logp=f(T), lse=f(T), entropy=f(T) if entropy else None)
    if K:
        out["top_ids"], out["top_logp"] = torch.full((T, K), -7, dtype=torch.int32, device="cuda"), f(T, K)
    n = B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=d, V=V, B=K)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_logprobs(H, W, y, None, out["logp"], out["lse"], out["entropy"], out.get("top_ids"), out.get("top_logp"), ws[:n], st,
                   inv_temperature=inv_t)
    torch.cuda.synchronize()
    assert int(st[0]) == 0 and bool((ws[n:] == 0xFF).all())
    return out


def check_forward(T, d, V, bf16, K, entropy, inv_t=1.0, w_std=0.03):
    import torch
    H, W, y, _ = data(T + d + V + K, T, d, V, bf16, w_std, True)
    want, got = forward64(H, W, y, inv_t, K), forward(H, W, y, K, entropy, inv_t)
    tol, tol_ent = slack(H, W, inv_t, want["lse"])
    for k in ("lse", "logp") + (("top_logp",) if K else ()):
        assert float((got[k].double() - want[k]).abs().max()) <= tol, k
    if entropy:
        assert float((got["entropy"].double() - want["entropy"]).abs().max()) <= tol_ent
    if K:
        assert torch.equal(got["top_ids"], want["top_ids"])


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("T,d,V,K", [(129, 1088, 20011, 0), (300, 1088, 5003, 8), (300, 1088, 5003, 20), (777, 2048, 3000, 5),
                                     (1300, 1152, 513, 13), (200, 4096, 32000, 0)])
def test_forward_on_wide_tiles(T, d, V, K, entropy):
    check_forward(T, d, V, True, K, entropy)


@pytest.mark.parametrize("T,K", [(65, 0), (81, 20), (96, 8), (97, 3), (49, 20), (128, 20)])
def test_forward_rungs_of_the_streaming_kernel(T, K):
    check_forward(T, 320, 40009, True, K, True, float(np.float32(1 / 0.7)))


@pytest.mark.parametrize("T,K", [(1, 20), (48, 8), (130, 20), (1100, 8)])
def test_forward_over_a_large_vocabulary(T, K):
    check_forward(T, 4096 if T < 200 else 256, 151936, True, K, True)


@pytest.mark.parametrize("T,d,V,K", [(200, 16, 500009, 20), (330, 8, 400000, 0), (2200, 64, 60001, 5)])
def test_fp32_forward_in_several_chunks(T, d, V, K):
    check_forward(T, d, V, False, K, True, w_std=0.3)


# ------------------------------------------------------------------------------------------------ backward
def check_backward(T, d, V, bf16, masked, dh32, dw32, accumulate, inv_t=1.0, targets=None, w_std=0.03):
    import torch
    from paper_2509_13232_b200 import binding as B
    H, W, y, g = data(T + d + V, T, d, V, bf16, w_std, False)
    if targets:
        y = y % targets
    mask = (torch.rand(T, generator=g, device="cuda") < 0.7).to(torch.uint8) if masked else None
    raw = H.double() @ W.double().T * inv_t
    lse = torch.logsumexp(raw, 1).float()
    lp = raw - lse.double()[:, None]
    ent = -(lp.exp() * lp).sum(1).float()
    gl, gs, ge = (torch.randn(T, generator=g, device="cuda") for _ in range(3))
    tol, _ = slack(H, W, inv_t, lse)
    on = torch.ones(T, device="cuda", dtype=torch.float64) if mask is None else mask.double()
    p = lp.exp() * on[:, None]
    a, b = (gs - gl).double()[:, None], ge.double()[:, None]
    dz = p * (a - b * (lp + ent.double()[:, None]))
    size = p * (a.abs() + b.abs() * (lp.abs() + ent.double().abs()[:, None]))
    at = torch.arange(T, device="cuda")
    dz[at, y.long()] += gl.double() * on
    size[at, y.long()] += gl.double().abs() * on
    dz, size = inv_t * dz, inv_t * size
    dt = H.dtype
    dH = torch.full((T, d), float("nan"), device="cuda", dtype=torch.float32 if dh32 else dt)
    wdt = torch.float32 if dw32 else dt
    start = torch.randn(V, d, generator=g, device="cuda").to(wdt) if accumulate else torch.zeros(V, d, device="cuda", dtype=wdt)
    dW = start.clone() if accumulate else torch.full((V, d), float("nan"), device="cuda", dtype=wdt)
    n = B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=T, d=d, V=V)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    dirty = H if mask is None else torch.where(mask[:, None] != 0, H, torch.full_like(H, float("nan")))
    B.spo_logprobs_bwd(dirty, W, y, mask, lse, ent, gl, gs, ge, dH, dW, int(accumulate), ws[:n], st, inv_temperature=inv_t)
    torch.cuda.synchronize()
    assert int(st[0]) == 0 and bool((ws[n:] == 0xFF).all())
    slip = (2.0**-8 if bf16 else 0.0) + 2 * tol + 2.0**-20
    dh = dz @ W.double()
    bound = (slip + (V + 64) * 2.0**-24) * (size @ W.double().abs()) + (0.0 if dH.dtype == torch.float32 else 2.0**-8) * dh.abs() + 1e-30
    assert bool(((dH.double() - dh).abs() <= bound).all())
    dw = dz.T @ H.double()
    bound = (slip + (T + 64) * 2.0**-24) * (size.T @ (H.double().abs() * on[:, None])) + 1e-30
    bound += (2.0**-8 if dW.dtype == torch.bfloat16 else 2.0**-23) * ((dw + start.double()).abs() + start.double().abs())
    dw += start.double()
    assert bool(((dW.double() - dw).abs() <= bound).all())


@pytest.mark.parametrize("T,d,V,masked,dh32,dw32,acc,targets", [
    (300, 1088, 20003, True, False, False, False, None),
    (700, 2048, 5000, False, True, True, True, 30),
    (1300, 1152, 3001, True, False, False, True, None),
    (203, 1024, 32000, True, False, False, False, 3),
    (130, 4096, 32000, False, False, True, False, None),
    (50, 256, 151936, False, False, False, False, None),
])
def test_bf16_backward_of_large_configurations(T, d, V, masked, dh32, dw32, acc, targets):
    check_backward(T, d, V, True, masked, dh32, dw32, acc, float(np.float32(1 / 0.9)), targets)


@pytest.mark.parametrize("T,d,V,masked,acc", [
    (200, 16, 500009, True, False),        # several chunks of rows
    (330, 8, 400000, False, True),
    (2000, 1300, 300, False, False),       # 128-wide tiles for dH,
    (300, 1000, 3001, True, True),         # for dW,
    (700, 64, 9001, False, False),         # and for the gradient of the logits
])
def test_fp32_backward_of_large_batches(T, d, V, masked, acc):
    check_backward(T, d, V, False, masked, True, True, acc, 1.0, None, 0.1)


# ------------------------------------------------------------------------------------------------ updates
@pytest.mark.parametrize("m,n,w_bf16", [(32000, 512, True), (20011, 256, False), (256, 30000, True)])
def test_update_of_a_matrix_with_a_row_or_column_per_token(m, n, w_bf16):
    import torch
    from paper_2509_13232_b200 import binding as B
    from tests.test_gpu_muon import gradient, iterate64, workspace
    rng = np.random.default_rng(m)
    g = gradient(rng, 1, m, n, 64) + 3e-4 * rng.standard_normal((1, m, n)).astype(np.float32)
    w = inputs.round_to_bf16((0.02 * rng.standard_normal((m, n))).astype(np.float32))
    W = torch.from_numpy(w).cuda().to(torch.bfloat16 if w_bf16 else torch.float32)
    M, G = torch.zeros(m, n, device="cuda"), torch.from_numpy(g[0]).cuda()
    ws, k = workspace(m, n, 1)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    lr = float(np.float32(0.05))
    B.spo_muon_update(W, M, G, ws[:k], B.default_muon_params(lr=lr, momentum=0.0, nesterov=0, scale_mode=B.MUON_SCALE_NONE), st)
    torch.cuda.synchronize()
    assert int(st[0]) == 0 and bool((ws[k:] == 0xFF).all()) and torch.equal(M, G)
    x, rounded = iterate64(g, False)[0], iterate64(g, True)[0]
    want = torch.from_numpy(w).cuda().double() - lr * x
    norm = torch.linalg.vector_norm
    allowed = lr * (2 * norm(rounded - x) + 2.0**-19 * norm(x)) + (2.0**-8 if w_bf16 else 2.0**-23) * norm(want)
    assert float(norm(W.double() - want)) <= float(allowed)
