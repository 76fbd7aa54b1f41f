"""One training step's end, as its parts are used together: final norm, loss from hidden states, gradients back through the norm, their
global norm, and the AdamW step on the vocabulary matrix (8-bit states) and the norm's weights (32 bits), for several steps."""

import numpy as np
import pytest

from oracle import operators as P
from oracle import spo_oracle as S
from oracle import step as O
from paper_2509_13232_b200 import inputs

pytestmark = pytest.mark.gpu


def test_norm_loss_gradients_and_update():
    import torch
    from paper_2509_13232_b200 import binding as B
    lengths, d, V = [90, 33, 61], 128, 700
    T = sum(lengths)
    lb = inputs.loss_batch(60, lengths, d, V, 0.05, True, 0.3, target="softmax", a_norm=np.array([0.7, -1.1, 0.4], np.float32))
    f32 = dict(dtype=torch.float32, device="cuda")
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    scratch = lambda which, **k: torch.empty(max(B.spo_workspace_bytes(which, **k), 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    rng = np.random.default_rng(3)
    stream_in, block_out = up(rng.standard_normal((T, d)).astype(np.float32)).bfloat16(), up(rng.standard_normal((T, d)).astype(np.float32)).bfloat16()
    weight, bias = up((1 + 0.1 * rng.standard_normal(d)).astype(np.float32)), up((0.1 * rng.standard_normal(d)).astype(np.float32))
    W32 = up(lb.w)
    W = W32.bfloat16()                                              # what the loss reads: the copy that the step keeps up to date
    y, mask, cu, a = up(lb.y), up(lb.mask), up(lb.cu_seqlens), up(lb.a_norm)
    h, H = torch.empty_like(stream_in), torch.empty_like(stream_in)
    mean, rstd, loss, lp, lse, coef = (torch.empty(n, **f32) for n in (T, T, 4, T, T, T))
    dH, dx, dW = torch.empty(T, d, **f32), torch.empty_like(h), torch.empty(V, d, **f32)
    dw, db = torch.empty(d, **f32), torch.empty(d, **f32)
    st, count, out = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty(4, **f32)
    nb = -(-V * d // B.ADAMW_BLOCK)
    cm, cv = torch.zeros(V * d, dtype=torch.int8, device="cuda"), torch.zeros(V * d, dtype=torch.uint8, device="cuda")
    sm, sv = torch.zeros(nb, **f32), torch.zeros(nb, **f32)
    small = [torch.zeros(d, **f32) for _ in range(4)]
    params = B.adamw_list([W32, weight, bias], [dW, dw, db], [cm, small[0], small[1]], [cv, small[2], small[3]], [sm, None, None], [sv, None, None],
                          [W, None, None], decay_scale=[1.0, 0.0, 0.0])
    grads = B.grad_list([dW, dw, db])
    p, ap = B.default_params(), B.default_adamw_params(lr=2e-3, weight_decay=0.1)
    lr, decay = (float(np.float32(x)) for x in (2e-3, 0.1))
    ws = {k: scratch(k, T=T, d=d, V=V, B=3) for k in (B.WS_LOSS_FWD_BWD, B.WS_LOGPROBS, B.WS_LAYERNORM_BWD, B.WS_GRAD_NORM)}
    host = lambda t: t.double().cpu().numpy()  # noqa: E731

    # the acting policy's log-probs of the tokens
    B.spo_layernorm_fwd(stream_in, block_out, weight, bias, None, H, h, mean, rstd, st)
    logp_old = torch.empty(T, **f32)
    B.spo_logprobs(H, W, y, None, logp_old, lse, None, None, None, ws[B.WS_LOGPROBS], st)

    def step():
        B.spo_layernorm_fwd(stream_in, block_out, weight, bias, None, H, h, mean, rstd, st)
        B.spo_loss_fwd_bwd(H, W, y, logp_old, mask, cu, a, 1.0, loss, lp, lse, coef, None, dH, dW, 0, ws[B.WS_LOSS_FWD_BWD], p, st)
        B.spo_layernorm_bwd(dH, h, weight, mask, mean, rstd, None, dx, dw, db, 0, ws[B.WS_LAYERNORM_BWD], st)
        B.spo_grad_norm(grads, out, ws[B.WS_GRAD_NORM], st, max_norm=0.05)
        B.spo_adamw_update(params, out[1:2], count, None, ap, st)

    m8, v8 = np.zeros(V * d, np.float32), np.zeros(V * d, np.float32)
    moments = {k: [np.zeros(d, np.float32), np.zeros(d, np.float32)] for k in ("weight", "bias")}
    for k in range(3):
        before = {n: host(t) for n, t in (("W32", W32), ("W", W), ("weight", weight), ("bias", bias))}
        step()
        torch.cuda.synchronize()
        # forward and loss, from the weights as they stood
        want = O.layernorm(host(stream_in), before["weight"], before["bias"], host(block_out), bf16=True)
        assert np.array_equal(host(h), want["h"])
        Hw = host(H)
        assert np.all(np.abs(Hw - want["y"]) <= 2.0**-8 * np.abs(want["y"]) + 1e-5)
        fwd = S.loss_forward(Hw, before["W"], lb.y, host(logp_old), lb.mask, lb.cu_seqlens, lb.a_norm.astype(np.float64))
        assert abs(float(loss[0]) - fwd["loss"]) < 2e-3
        want_dh, want_dw = S.loss_backward(Hw, before["W"], lb.y, fwd["lse"], fwd["coef"])
        assert np.linalg.norm(host(dW) - want_dw) < 1e-2 * np.linalg.norm(want_dw)
        assert np.linalg.norm(host(dH) - want_dh) < 1.5e-2 * np.linalg.norm(want_dh)
        # through the norm, from the gradient as it was handed on; gradients in double precision agree with one another
        back = O.layernorm_backward(host(dH), host(h), host(mean), host(rstd), before["weight"], mask=lb.mask)
        assert np.linalg.norm(host(dx) - back["dx"]) <= 2.0**-8 * np.linalg.norm(back["dx"]) + 1e-7
        assert np.linalg.norm(host(dw) - back["dw"]) <= 1e-5 * np.linalg.norm(back["dw"])
        assert np.linalg.norm(host(db) - back["db"]) <= 1e-5 * np.linalg.norm(back["db"])
        # norm, factor, step
        norm, factor = O.grad_norm([host(dW), host(dw), host(db)], max_norm=0.05)
        assert abs(float(out[0]) - norm) <= 1e-6 * norm and abs(float(out[1]) - factor) <= 1e-6 * factor
        f = out[1].cpu().numpy()
        w1, m1, v1, first = O.adamw(before["W32"].reshape(-1), host(dW).reshape(-1), m8, v8, k + 1, lr=lr, decay=decay, scale=f)
        assert np.all(np.abs(host(W32).reshape(-1) - w1) <= 2.0**-19 * first + 2.0**-23 * (np.abs(w1) + first))
        assert torch.equal(W, W32.bfloat16())
        codes = O.encode(m1, v1)
        for got, exp in zip((cm, sm, cv, sv), codes):
            assert np.array_equal(got.cpu().numpy(), exp)
        m8, v8 = O.decode(*codes)
        for name, t, g in (("weight", weight, dw), ("bias", bias, db)):
            w1, m1, v1, first = O.adamw(before[name], host(g), *moments[name], k + 1, lr=lr, scale=f)
            assert np.all(np.abs(host(t) - w1) <= 2.0**-19 * first + 2.0**-23 * (np.abs(w1) + first))
            moments[name] = [m1, v1]
        assert int(st[0]) == 0 and count.tolist() == [k + 1, 0]
    # the policy has moved: its log-probs are those of the definition for the new weights
    B.spo_layernorm_fwd(stream_in, block_out, weight, bias, None, H, h, mean, rstd, st)
    B.spo_logprobs(H, W, y, None, lp, lse, None, None, None, ws[B.WS_LOGPROBS], st)
    torch.cuda.synchronize()
    np.testing.assert_allclose(host(lp), P.logprobs(host(H), host(W), lb.y)["logp"], rtol=0, atol=1e-3)
    assert float((lp - logp_old).abs().max()) > 1e-3
