"""One scratch buffer of the size named for the longest batch serves all shorter ones, and nothing behind it is touched."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,V,K,most", [(1024, 32000, 20, 8192), (128, 5000, 8, 20000), (1088, 9000, 20, 6000), (64, 40000, 20, 4096)])
def test_one_buffer_for_every_length(d, V, K, most):
    import torch
    from paper_2509_13232_b200 import binding as B
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    H = ((torch.randn(most, d, generator=g, device="cuda") * 32).round() / 32).clamp(-7.75, 7.75).bfloat16()
    W = ((torch.randn(V, d, generator=g, device="cuda") * 8).round() / 256).bfloat16()
    y = torch.randint(0, V, (most,), generator=g, device="cuda", dtype=torch.int32)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    sizes = [B.spo_workspace_bytes(w, T=most, d=d, V=V, **k) for w, k in ((B.WS_LOGPROBS, dict(B=K)), (B.WS_LOGPROBS_BWD, {}))]
    fwd, bwd = (torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda") for n in sizes)
    ref = None
    for T in [most, 3840, 3300, 2049, 1000, 300, 257, 256, 129, 128, 127, 1]:
        if T > most:
            continue
        logp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        ids, tlp = torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, K, device="cuda")
        B.spo_logprobs(H[:T], W, y[:T], None, logp, lse, None, ids, tlp, fwd[:sizes[0]], st)
        dH, dW = torch.empty(T, d, device="cuda").bfloat16(), torch.empty(V, d, device="cuda").bfloat16()
        B.spo_logprobs_bwd(H[:T], W, y[:T], None, lse, None, torch.ones(T, device="cuda"), None, None, dH, dW, 0, bwd[:sizes[1]], st)
        torch.cuda.synchronize()
        assert int(st[0]) == 0 and bool(torch.isfinite(dH.float()).all()) and bool(torch.isfinite(dW.float()).all())
        if ref is None:
            ref = (ids, logp)
        assert torch.equal(ids, ref[0][:T])              # the logits are exact, so the order is the same on every path
        np.testing.assert_allclose(logp.cpu(), ref[1][:T].cpu(), rtol=0, atol=1e-4)
        assert bool((fwd[sizes[0]:] == 0xA5).all()) and bool((bwd[sizes[1]:] == 0xA5).all())
