"""GPU parity of spo_orthogonalize / spo_muon_update with the float64 definitions.

Tolerance, derived before any run.  The library rounds the iterate, its Gram matrix and the polynomial to fp16; what
those roundings do to a given input is computed on the CPU by oracle.operators.newton_schulz_rounded, and a second
set of roundings of the same size (fp32 sums flip some of them) doubles it: 2 e_fp16 in the Frobenius norm, plus
2^-19 for the fp32 sums (products of up to 2^12 terms, a few 2^-24 each, times the iteration's amplification of 8 at the
singular values that matter).  A bf16 result adds at most 2^-8 of each entry.
"""

import numpy as np
import pytest

from oracle import operators as O
from paper_2509_13232_b200 import inputs

pytestmark = pytest.mark.gpu


def gradient(rng, b, m, n, rank=None):
    r = max(1, min(m, n) // 4) if rank is None else rank
    g = rng.standard_normal((b, m, r)) @ rng.standard_normal((b, r, n)) / np.sqrt(r)
    if rank is None:
        g = g + 0.3 * rng.standard_normal((b, m, n))
    return (1e-3 * g).astype(np.float32)


def workspace(m, n, b):
    import torch
    from paper_2509_13232_b200 import binding as B
    k = B.spo_workspace_bytes(B.WS_MUON, T=m, d=n, B=b)
    ws = torch.full((k + 64,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN patterns in fp16
    return ws, k


def orthogonalize(g, out_bf16=False, g_bf16=False, **params):
    import torch
    from paper_2509_13232_b200 import binding as B
    b, m, n = g.shape
    G = torch.from_numpy(g).cuda()
    if g_bf16:
        G = G.bfloat16()
    out = torch.full((b, m, n), float("nan"), dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
    ws, k = workspace(m, n, b)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_orthogonalize(G, out, ws[:k], B.default_muon_params(**params), st)
    torch.cuda.synchronize()
    assert bool((ws[k:] == 0xFF).all())
    return out.float().cpu().numpy(), int(st[0])


def check(got, g, bf16, steps=5):
    for x, y in zip(got, g):
        want, rounded = O.newton_schulz(y, steps), O.newton_schulz_rounded(y, steps)
        norm = np.linalg.norm(want)
        allowed = 2 * np.linalg.norm(rounded - want) + 2.0**-19 * norm + (2.0**-8 * norm if bf16 else 0.0)
        assert np.linalg.norm(x - want) <= allowed, (np.linalg.norm(x - want) / norm, allowed / norm)
        worst = np.abs(rounded - want).max()
        size = np.sqrt(np.mean(want**2))
        assert np.abs(x - want).max() <= 4 * worst + 2.0**-16 * size + (2.0**-8 * np.abs(want).max() if bf16 else 0.0)


SHAPES = [(1, 1, 1), (1, 1, 7), (2, 5, 3), (3, 33, 17), (1, 64, 64), (1, 128, 512), (2, 300, 130), (1, 257, 513),
          (1, 1000, 273), (3, 256, 256), (1, 40, 3001), (2, 1500, 40), (1, 520, 776), (1, 800, 1202)]


@pytest.mark.parametrize("b,m,n", SHAPES)
@pytest.mark.parametrize("bf16", [False, True])
def test_orthogonalize(b, m, n, bf16):
    g = gradient(np.random.default_rng(m * 3 + n), b, m, n)
    if bf16:
        g = inputs.round_to_bf16(g)
    got, st = orthogonalize(g, out_bf16=bf16, g_bf16=bf16)
    assert st == 0
    check(got, g, bf16)


def iterate64(g, rounded):
    """oracle.operators.newton_schulz and newton_schulz_rounded for a batch, in 64 bits on the GPU: the sizes at which wide tiles
    are chosen take the CPU minutes."""
    import torch
    a, b, c = O.NS_COEFFICIENTS
    x = torch.from_numpy(g).cuda().double()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    s = 2.0 ** np.round(np.log2(np.sqrt(x.shape[2])))
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + 1e-7) * s
    half = (lambda z: z.half().double()) if rounded else (lambda z: z)
    for _ in range(5):
        hi = half(x)
        q = half(hi @ hi.transpose(1, 2) / s**2)
        poly = b * q + c * (q @ q)
        d = torch.diagonal(poly, dim1=1, dim2=2).unsqueeze(2).clone()
        torch.diagonal(poly, dim1=1, dim2=2).zero_()
        x = (a + d) * x + half(poly) @ hi
    x = x / s
    return x.transpose(1, 2) if tall else x


# one for each pair of tile widths (symmetric products, update) and orientation
@pytest.mark.parametrize("b,m,n", [(24, 130, 8200), (80, 2056, 130), (74, 130, 1040), (74, 1040, 130), (24, 260, 2056),
                                   (74, 2600, 130), (12, 1000, 2600), (12, 2600, 1000), (1, 3026, 3762), (2, 3738, 2428),
                                   (4, 1000, 2730)])
def test_large_batches_and_matrices(b, m, n):
    import torch
    rng = np.random.default_rng(b + m)
    k = min(b, 3)
    g = np.concatenate([gradient(rng, k, m, n, 40) + 3e-4 * rng.standard_normal((k, m, n)).astype(np.float32)] * -(-b // k))[:b]
    got, st = orthogonalize(g)
    assert st == 0
    want, rounded = iterate64(g[:k], False), iterate64(g[:k], True)
    norm = torch.linalg.vector_norm(want, dim=(1, 2))
    allowed = 2 * torch.linalg.vector_norm(rounded - want, dim=(1, 2)) + 2.0**-19 * norm
    assert bool((torch.linalg.vector_norm(torch.from_numpy(got[:k]).cuda().double() - want, dim=(1, 2)) <= allowed).all())
    for i in range(k, b):                                 # the same matrix again, on other tiles: the same bits
        assert np.array_equal(got[i], got[i % k])


@pytest.mark.parametrize("m,n,rank", [(256, 320, 1), (320, 256, 8), (512, 512, 40)])
def test_low_rank_updates_keep_their_rank(m, n, rank):
    """The case in which a rounding of the iterate is amplified most: directions that are exactly zero."""
    g = gradient(np.random.default_rng(rank), 1, m, n, rank)
    got, st = orthogonalize(g)
    assert st == 0
    check(got, g, False)
    sv = np.linalg.svd(got[0], compute_uv=False)
    assert np.all(sv[:rank] > 0.6) and np.all(sv[:rank] < 1.3) and np.all(sv[rank:] < 0.02)


@pytest.mark.parametrize("steps", [1, 2, 8])
def test_other_step_counts_and_a_large_scale(steps):
    g = gradient(np.random.default_rng(steps), 1, 130, 200) * 1e20
    got, st = orthogonalize(g, steps=steps)
    assert st == 0
    check(got, g, False, steps)


def test_zero_and_non_finite_matrices_of_a_batch():
    from paper_2509_13232_b200 import binding as B
    g = gradient(np.random.default_rng(0), 5, 70, 90)
    g[1] = 0.0
    g[2, 3, 4] = np.nan
    g[4, 69, 89] = -np.inf
    got, st = orthogonalize(g)
    assert st == B.DEV_NONFINITE
    assert np.all(got[1] == 0) and np.all(got[2] == 0) and np.all(got[4] == 0)
    check(got[[0, 3]], g[[0, 3]], False)


def test_result_may_replace_the_gradient_and_repeats_bit_for_bit():
    import torch
    from paper_2509_13232_b200 import binding as B
    g = gradient(np.random.default_rng(1), 2, 200, 333)
    first, _ = orthogonalize(g)
    G = torch.from_numpy(g).cuda()
    ws, k = workspace(200, 333, 2)
    B.spo_orthogonalize(G, G, ws[:k], B.default_muon_params(), None)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(G.cpu().numpy(), first)


@pytest.mark.parametrize("b,m,n,w_bf16,g_bf16,nesterov,mode", [
    (1, 96, 160, False, False, 1, 0), (2, 160, 96, True, False, 1, 1), (1, 333, 250, False, True, 0, 2),
    (3, 65, 131, True, True, 1, 2), (1, 512, 256, True, False, 0, 1), (1, 30, 2002, False, False, 1, 2)])
def test_muon_update(b, m, n, w_bf16, g_bf16, nesterov, mode):
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(m + n)
    g, mom = gradient(rng, b, m, n), 3 * gradient(rng, b, m, n)
    w = (0.02 * rng.standard_normal((b, m, n))).astype(np.float32)
    if g_bf16:
        g = inputs.round_to_bf16(g)
    if w_bf16:
        w = inputs.round_to_bf16(w)
    lr, mu, decay = (float(np.float32(x)) for x in (0.03, 0.9, 0.2))
    p = B.default_muon_params(lr=lr, momentum=mu, weight_decay=decay, nesterov=nesterov, scale_mode=mode)
    W = torch.from_numpy(w).cuda().to(torch.bfloat16 if w_bf16 else torch.float32)
    M, G = torch.from_numpy(mom).cuda(), torch.from_numpy(g).cuda().to(torch.bfloat16 if g_bf16 else torch.float32)
    ws, k = workspace(m, n, b)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    want_w, want_m = w.astype(np.float64), mom.astype(np.float64)
    slack = np.zeros(b)
    for _ in range(2):                                             # the second step continues from the first
        B.spo_muon_update(W, M, G, ws[:k], p, st)
        torch.cuda.synchronize()
        for i in range(b):
            u = mu * want_m[i] + g[i]
            u = g[i] + mu * u if nesterov else u
            gap = np.linalg.norm(O.newton_schulz_rounded(u) - O.newton_schulz(u)) + 2.0**-19 * np.sqrt(min(m, n))
            slack[i] += 2 * lr * O.muon_scale(m, n, mode) * gap
            want_w[i], want_m[i], _ = O.muon_update(want_w[i], want_m[i], g[i], lr, mu, decay, bool(nesterov), mode)
            slack[i] += (2.0**-8 if w_bf16 else 2.0**-22) * np.linalg.norm(want_w[i])
        np.testing.assert_allclose(M.cpu().numpy(), want_m, rtol=2.0**-21, atol=2.0**-21 * np.abs(want_m).max())
        for i in range(b):
            assert np.linalg.norm(W[i].float().cpu().numpy() - want_w[i]) <= slack[i]
    assert int(st[0]) == 0


@pytest.mark.parametrize("w_bf16", [False, True])
def test_a_non_finite_update_leaves_weights_and_momentum(w_bf16):
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(9)
    g = gradient(rng, 2, 60, 44)
    g[0, 0, 0] = np.inf
    W = torch.randn(2, 60, 44, device="cuda").to(torch.bfloat16 if w_bf16 else torch.float32)
    M = torch.randn(2, 60, 44, device="cuda")
    w0, m0 = W.clone(), M.clone()
    ws, k = workspace(60, 44, 2)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_muon_update(W, M, torch.from_numpy(g).cuda(), ws[:k], B.default_muon_params(weight_decay=0.5), st)
    torch.cuda.synchronize()
    assert int(st[0]) == B.DEV_NONFINITE
    assert torch.equal(W[0], w0[0]) and torch.equal(M[0], m0[0])
    assert not torch.equal(W[1], w0[1]) and not torch.equal(M[1], m0[1])


def test_captured_and_on_two_streams():
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(4)
    shapes = [(2, 200, 333), (1, 640, 130)]
    p = B.default_muon_params()
    G = [torch.from_numpy(gradient(rng, *s)).cuda() for s in shapes]
    out = [torch.empty_like(x) for x in G]
    ws = [workspace(s[1], s[2], s[0]) for s in shapes]
    for x, o, (w, k) in zip(G, out, ws):
        B.spo_orthogonalize(x, o, w[:k], p, None)
    torch.cuda.synchronize()
    ref = [o.clone() for o in out]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for x, o, (w, k), s in zip(G, out, ws, streams):
            with torch.cuda.stream(s):
                B.spo_orthogonalize(x, o, w[:k], p, None)
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(out, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, o, (w, k) in zip(G, out, ws):
            B.spo_orthogonalize(x, o, w[:k], p, None)
    for x in G:
        x.mul_(3.0)                              # the result does not depend on the scale (up to eps and roundings)
    for o in out:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for o, r in zip(out, ref):
        assert float((o - r).norm() / r.norm()) < 2e-2


def test_two_calls_at_once_that_each_fill_the_gpu():
    """The iteration's blocks wait for one another; two such launches on two streams must both come through."""
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(5)
    shapes = [(1, 2304, 2560), (2, 1800, 1300)]
    p = B.default_muon_params()
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    G = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in shapes]
    out = [torch.empty_like(x) for x in G]
    ws = [workspace(s[1], s[2], s[0]) for s in shapes]
    for x, o, (w, k) in zip(G, out, ws):
        B.spo_orthogonalize(x, o, w[:k], p, st)
    torch.cuda.synchronize()
    ref = [o.clone() for o in out]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(6):
        for x, o, (w, k), s in zip(G, out, ws, streams):
            with torch.cuda.stream(s):
                B.spo_orthogonalize(x, o, w[:k], p, st)
    torch.cuda.synchronize()
    assert int(st[0]) == 0
    assert all(torch.equal(o, r) for o, r in zip(out, ref))
    # an orthogonal matrix comes out: its singular values lie where five steps put those of a full-rank input
    sv = torch.linalg.svdvals(ref[0][0])
    assert 0.3 < float(sv.min()) and float(sv.max()) < 1.3
