"""The operators in the order in which a training step uses them: log-probs of the acting policy, advantages, loss and
gradients, the orthogonalised weight update, log-probs of the updated policy, and the tracker update from the
divergence between the two."""

import numpy as np
import pytest

from oracle import operators as O
from oracle import spo_oracle as S
from paper_2509_13232_b200 import inputs

pytestmark = pytest.mark.gpu


def test_one_policy_update_from_log_probs_to_log_probs():
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(17)
    lengths, d, V = [150, 37, 90, 64], 128, 1000
    n_seq, T = len(lengths), sum(lengths)
    lb = inputs.loss_batch(50, lengths, d, V, 0.05, True, 0.0, target="softmax")
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    f32 = dict(dtype=torch.float32, device="cuda")
    H, W, y, cu = up(lb.h).bfloat16(), up(lb.w).bfloat16(), up(lb.y), up(lb.cu_seqlens)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    scratch = lambda which, **k: torch.empty(max(B.spo_workspace_bytes(which, **k), 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    ws = scratch(B.WS_LOGPROBS, T=T, d=d, V=V, B=5)

    def log_probs():
        logp, lse, ent = (torch.empty(T, **f32) for _ in range(3))
        ids, tlp = torch.empty(T, 5, dtype=torch.int32, device="cuda"), torch.empty(T, 5, **f32)
        B.spo_logprobs(H, W, y, None, logp, lse, ent, ids, tlp, ws, st)
        return logp, ent, ids, tlp

    logp_old, ent, ids, tlp = log_probs()
    want = O.logprobs(lb.h, lb.w, lb.y, top_k=5)
    np.testing.assert_allclose(logp_old.cpu(), want["logp"], rtol=0, atol=1e-4)
    np.testing.assert_allclose(ent.cpu(), want["entropy"], rtol=0, atol=1e-3)
    np.testing.assert_allclose(tlp.cpu(), want["top_logp"], rtol=0, atol=1e-4)

    # advantages of four responses against a tracker of six prompts
    ab = rng.uniform(1.0, 10.0, (6, 2)).astype(np.float32)
    prompts, r = np.array([4, 0, 3, 1], np.int32), np.array([1, 0, 1, 1], np.float32)
    a_norm = torch.empty(n_seq, **f32)
    p = B.default_params()
    B.spo_advantages(up(ab), up(prompts), up(r), None, a_norm, None, scratch(B.WS_ADVANTAGES, B=n_seq), p, st)
    a64, b64 = ab[:, 0].astype(np.float64), ab[:, 1].astype(np.float64)
    want_a, _, _ = S.normalise_advantages(S.raw_advantage(a64, b64, prompts, r))

    # loss and gradients: with the acting policy's own log-probs every ratio is one
    loss, logp, lse, coef = torch.empty(4, **f32), *(torch.empty(T, **f32) for _ in range(3))
    dH, dW = torch.empty_like(H), torch.empty(V, d, **f32)
    B.spo_loss_fwd_bwd(H, W, y, logp_old, None, cu, a_norm, 1.0, loss, logp, lse, coef, None, dH, dW, 0,
                       scratch(B.WS_LOSS_FWD_BWD, T=T, d=d, V=V, B=n_seq), p, st)
    fwd = S.loss_forward(lb.h, lb.w, lb.y, want["logp"], None, lb.cu_seqlens, want_a)
    want_dh, want_dw = S.loss_backward(lb.h, lb.w, lb.y, fwd["lse"], fwd["coef"])
    assert abs(float(loss[0]) - fwd["loss"]) < 1e-3
    assert np.linalg.norm(dW.cpu().numpy() - want_dw) < 1e-2 * np.linalg.norm(want_dw)
    # the general backward with the loss's coefficients gives the same gradients
    dH2, dW2 = torch.empty_like(dH), torch.empty_like(dW)
    B.spo_logprobs_bwd(H, W, y, None, lse, None, coef, None, None, dH2, dW2, 0, scratch(B.WS_LOGPROBS_BWD, T=T, d=d, V=V), st)
    assert float((dW2 - dW).norm() / dW.norm()) < 1e-2 and float((dH2.float() - dH.float()).norm() / dH.float().norm()) < 1.5e-2

    # the weight update (momentum from an earlier step), against the same step on the library's own gradient
    mom = (0.1 * rng.standard_normal((V, d)) * float(dW.abs().max())).astype(np.float32)
    M = up(mom)
    mp = B.default_muon_params(lr=0.05, momentum=0.9, weight_decay=0.1, scale_mode=B.MUON_SCALE_RMS)
    lr, mu_, decay = (float(np.float32(x)) for x in (0.05, 0.9, 0.1))
    before = W.float().cpu().numpy()
    B.spo_muon_update(W, M, dW, scratch(B.WS_MUON, T=V, d=d, B=1), mp, st)
    want_w, want_m, want_o = O.muon_update(before, mom, dW.cpu().numpy(), lr, mu_, decay, True, 2)
    np.testing.assert_allclose(M.cpu(), want_m, rtol=1e-6, atol=1e-6 * np.abs(want_m).max())
    step = lr * O.muon_scale(V, d, 2)
    u = dW.cpu().numpy() + mu_ * want_m
    slack = 2 * step * np.linalg.norm(O.newton_schulz_rounded(u) - want_o) + (2.0**-8 + 2.0**-20) * np.linalg.norm(want_w)
    assert np.linalg.norm(W.float().cpu().numpy() - want_w) <= slack

    # the updated policy's log-probs, and the tracker update from the mean log-ratio of each response
    new, _, _, _ = log_probs()
    want_new = O.logprobs(lb.h, W.float().cpu().numpy(), lb.y)["logp"]
    np.testing.assert_allclose(new.cpu(), want_new, rtol=0, atol=1e-4)
    assert float((new - logp_old).abs().max()) > 1e-3
    kl = np.array([float((logp_old - new)[lb.cu_seqlens[i]:lb.cu_seqlens[i + 1]].mean()) for i in range(n_seq)], np.float32)
    kl = np.abs(kl)
    table = up(ab)
    B.spo_tracker_update(table, up(prompts), up(r), up(kl), 0, p, st)
    a1, b1 = S.tracker_update(a64, b64, prompts, r, kl.astype(np.float64), float(np.float32(p.d_half)))
    np.testing.assert_allclose(table.cpu(), np.stack([a1, b1], 1), rtol=1e-5, atol=1e-6)
    torch.cuda.synchronize()
    assert int(st[0]) == 0


def test_the_binding_refuses_before_any_launch():
    import torch
    from paper_2509_13232_b200 import binding as B
    H, W = torch.zeros(4, 64, device="cuda").bfloat16(), torch.zeros(10, 64, device="cuda").bfloat16()
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    y, ws = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    ok = dict(H=H, W=W, y=y, mask=None, logp=f(4), lse=f(4), entropy=None, top_ids=None, top_logp=None, ws=ws, d_status=None)
    B.spo_logprobs(**ok)
    for bad, err in ((dict(H=H.float()), TypeError), (dict(W=W[:, :32]), ValueError), (dict(y=y.long()), TypeError),
                     (dict(y=y[:3]), ValueError), (dict(lse=f(5)), ValueError), (dict(lse=f(8)[::2]), ValueError),
                     (dict(lse=None), TypeError), (dict(y=None), B.SpoError), (dict(logp=torch.zeros(4)), ValueError),
                     (dict(H=H.t().contiguous().t()), ValueError), (dict(mask=torch.ones(4, dtype=torch.bool, device="cuda")), TypeError),
                     (dict(top_ids=torch.zeros(4, 2, dtype=torch.int32, device="cuda")), ValueError),
                     (dict(ws=ws[:16]), B.SpoError), (dict(H=H.half(), W=W.half()), TypeError)):
        with pytest.raises(err):
            B.spo_logprobs(**{**ok, **bad})
    g = f(6, 8)
    p = B.default_muon_params()
    B.spo_orthogonalize(g, f(6, 8), ws, p, None)
    for args in ((g, f(8, 6)), (g[0], f(8)), (g, f(6, 16)[:, ::2]), (g.cpu(), f(6, 8)), (g.half(), f(6, 8))):
        with pytest.raises((TypeError, ValueError)):
            B.spo_orthogonalize(*args, ws, p, None)
    with pytest.raises(B.SpoError):
        B.spo_orthogonalize(g, f(6, 8), ws[:64], p, None)
    with pytest.raises((TypeError, ValueError)):
        B.spo_muon_update(f(6, 8), f(6, 8).bfloat16(), g, ws, p, None)
    torch.cuda.synchronize()
