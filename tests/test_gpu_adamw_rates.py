"""Rates that leave fp32 only with a tensor's own scale, its decay or the correction of early steps: no step is taken, and none is counted, as for
a rate that is not finite itself."""

import pytest

pytestmark = pytest.mark.gpu


def make(torch, B, bits, lr_scale, decay_scale, tensors):
    f = lambda n=1000, **k: [torch.full((n,), 0.5, device="cuda", **k) for _ in range(tensors)]  # noqa: E731
    w, g = f(), f()
    if bits == 32:
        m, v, ms, vs = f(), f(), None, None
    else:
        m, v = ([torch.full((1000,), 7, dtype=t, device="cuda") for _ in range(tensors)] for t in (torch.int8, torch.uint8))
        ms, vs = f(4), f(4)
    scales = [1.0] * (tensors - 1) + [lr_scale], [1.0] * (tensors - 1) + [decay_scale]
    return [w, g, m, v] + ([ms, vs] if bits == 8 else []), B.adamw_list(w, g, m, v, ms, vs, None, *scales)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("tensors", [1, 3, 401])
@pytest.mark.parametrize("lr,device_lr,lr_scale,weight_decay,decay_scale", [
    (1e30, None, 1e30, 0.0, 1.0), (1e38, None, 1.0, 0.0, 1.0), (1e-3, 1e30, -1e30, 0.0, 1.0), (1e30, None, 1.0, 1e30, 1.0), (1e20, None, 1e10, 1e5, 1e10),
    (1e-3, None, 1.0, 1e30, 1e30), (1e-3, float("inf"), 1.0, 0.0, 1.0), (1e-3, float("nan"), 1.0, 0.0, 1.0)])
def test_rates_that_leave_fp32_take_no_step(bits, tensors, lr, device_lr, lr_scale, weight_decay, decay_scale):
    import torch
    from paper_2509_13232_b200 import binding as B
    held, table = make(torch, B, bits, lr_scale, decay_scale, tensors)
    before = [[t.clone() for t in x] for x in held]
    st, step = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    rate = None if device_lr is None else torch.full((1,), device_lr, device="cuda")
    # (the first step's correction is ten: a rate of 1e38 is finite, and not times ten)
    B.spo_adamw_update(table, None, step, rate, B.default_adamw_params(lr=lr, weight_decay=weight_decay), st)
    torch.cuda.synchronize()
    assert int(st[0]) == B.DEV_NONFINITE and step.tolist() == [0, 0]
    assert all(torch.equal(a, b) for x, y in zip(before, held) for a, b in zip(x, y))


@pytest.mark.parametrize("bits", [8, 32])
def test_large_rates_that_fit_are_taken(bits):
    import torch
    from paper_2509_13232_b200 import binding as B
    for lr, lr_scale, weight_decay, decay_scale in ((1e30, 1e-30, 1e30, 1e-30), (1e-30, 1e30, 0.0, 1e38), (0.0, 1e38, 1e38, 1.0), (1e30, 1.0, 0.0, 1.0)):
        held, table = make(torch, B, bits, lr_scale, decay_scale, 1)
        st, step = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        B.spo_adamw_update(table, None, step, None, B.default_adamw_params(lr=lr, weight_decay=weight_decay), st)
        torch.cuda.synchronize()
        assert int(st[0]) == 0 and step.tolist() == [1, 0]
        assert all(bool(torch.isfinite(t.float()).all()) for x in held for t in x)
