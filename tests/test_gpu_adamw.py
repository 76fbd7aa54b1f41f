"""GPU parity of spo_grad_norm, spo_adamw_update and spo_adamw_decode with the definitions of oracle/step.py.

Moments, codes, scales and decoded values are fixed bit for bit, so they are compared as they are.  Tolerances of the rest, derived
before any run, with u = 2^-24: the norm is the root of a sum whose shares of up to eight squares carry at most 8 u of themselves: 4 u,
and its own rounding u.  A weight moves by  step m / (sqrt(v) root + eps) + pull w:  the approximate root (2 u), root, step and pull as fp32
(u each), the fused sums (u each) and the approximate quotient (4 u) make at most 16 u of the first term and 4 u of the second, and
the weight's own rounding is u (fp32) or 2^-8 (bf16) of its value.
"""

import math

import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu

U = 2.0**-24
F = np.float32


def tensors(seed, sizes, bits, w16, g16, copy, offset=0, spread=1.0):
    """Host values and their device tensors, each beginning `offset` elements into a buffer of its own, with guards around it."""
    import torch
    rng = np.random.default_rng(seed)
    out = []
    for n, b, a16, b16, with_copy in zip(sizes, bits, w16, g16, copy):
        size = np.exp(spread * rng.standard_normal(n // 64 + 1)).repeat(64)[:n]
        w, g = (0.02 * rng.standard_normal(n)).astype(F), (1e-3 * rng.standard_normal(n) * size).astype(F)
        w, g = (O.round_bf16(x).astype(F) if f else x for x, f in ((w, a16), (g, b16)))
        m, v = (5e-4 * rng.standard_normal(n) * size).astype(F), ((1e-3 * rng.standard_normal(n) * size)**2).astype(F)
        t = dict(n=n, bits=b, w=w, g=g, w16=a16, g16=b16)
        if b == 8:
            t["cm"], t["sm"], t["cv"], t["sv"] = O.encode(m, v)
            t["m"], t["v"] = O.decode(t["cm"], t["sm"], t["cv"], t["sv"])
        else:
            t["m"], t["v"] = m, v
        t["guards"] = []

        def place(x, dtype, t=t):
            x = torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()
            buf = torch.full((x.numel() + offset + 40,), 77, dtype=dtype, device="cuda")
            buf[offset:offset + x.numel()] = x
            t["guards"].append((buf, offset, x.numel()))
            return buf[offset:offset + x.numel()]

        t["dw"], t["dg"] = place(w, torch.bfloat16 if a16 else torch.float32), place(g, torch.bfloat16 if b16 else torch.float32)
        if b == 8:
            t["dm"], t["dv"], t["dsm"], t["dsv"] = (place(t["cm"], torch.int8), place(t["cv"], torch.uint8), place(t["sm"], torch.float32),
                                                    place(t["sv"], torch.float32))
        else:
            t["dm"], t["dv"], t["dsm"], t["dsv"] = place(m, torch.float32), place(v, torch.float32), None, None
        t["dcopy"] = place(np.zeros(n, F), torch.bfloat16) if with_copy else None
        out.append(t)
    return out


def table(ts, **more):
    from paper_2509_13232_b200 import binding as B
    col = lambda k: [t[k] for t in ts]  # noqa: E731
    return B.adamw_list(col("dw"), col("dg"), col("dm"), col("dv"), col("dsm"), col("dsv"), col("dcopy"), **more)


def advance(t, step, scale=1.0, lr=1e-3, decay=0.1, **kw):
    """The definition's step on the host values; returns the weight and how far the device's may be from it."""
    want, m, v, first = O.adamw(t["w"], t["g"], t["m"], t["v"], step, lr=lr, decay=decay, scale=scale, **kw)
    slack = 16 * U * first + 4 * U * np.abs(lr * decay * t["w"]) + (2.0**-8 if t["w16"] else U) * (np.abs(want) + first)
    if t["bits"] == 8:
        t["cm"], t["sm"], t["cv"], t["sv"] = O.encode(m, v)
        m, v = O.decode(t["cm"], t["sm"], t["cv"], t["sv"])
    t["m"], t["v"] = m, v
    return want, slack


def compare(t, want, slack):
    import torch
    got = t["dw"].double().cpu().numpy()
    err = np.abs(got - want)
    assert np.all(err <= slack), float((err / np.maximum(slack, 1e-300)).max())
    if t["bits"] == 8:
        assert np.array_equal(t["dsm"].cpu().numpy(), t["sm"]) and np.array_equal(t["dsv"].cpu().numpy(), t["sv"])
        assert np.array_equal(t["dm"].cpu().numpy(), t["cm"]) and np.array_equal(t["dv"].cpu().numpy(), t["cv"])
    else:
        assert np.array_equal(t["dm"].cpu().numpy(), t["m"]) and np.array_equal(t["dv"].cpu().numpy(), t["v"])
    if t["dcopy"] is not None and not t["w16"]:
        assert torch.equal(t["dcopy"], t["dw"].bfloat16())
    for buf, offset, n in t["guards"]:
        assert bool((buf[:offset] == 77).all()) and bool((buf[offset + n:] == 77).all())
    t["w"] = t["dw"].float().cpu().numpy()          # the next step goes on from the device's weight


def steps(ts, count=3, lr=1e-3, decay=0.1, scale=0.7, device_step=True, first=1, rates=None, decays=None, device_rate=False, **kw):
    import torch
    from paper_2509_13232_b200 import binding as B
    f32 = lambda x: torch.tensor([x], dtype=torch.float32, device="cuda")  # noqa: E731
    tab = table(ts, lr_scale=rates, decay_scale=decays)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    count_on = torch.tensor([first - 1, 0], dtype=torch.int32, device="cuda") if device_step else None
    for k in range(count):
        p = B.default_adamw_params(lr=123.0 if device_rate else lr, weight_decay=decay, step=1 if device_step else first + k, **kw)
        B.spo_adamw_update(tab, None if scale is None else f32(scale), count_on, f32(lr) if device_rate else None, p, st)
        torch.cuda.synchronize()
        for i, t in enumerate(ts):
            rate = lr * (rates[i] if rates else 1.0)
            want, slack = advance(t, first + k, 1.0 if scale is None else scale, rate, decay * (decays[i] if decays else 1.0), **kw)
            compare(t, want, slack)
    assert int(st[0]) == 0
    if device_step:
        assert count_on.tolist() == [first - 1 + count, 0]


SIZES = [1, 2, 3, 4, 5, 127, 128, 129, 255, 256, 257, 511, 2047, 2048, 2049, 5000, 12345]


@pytest.mark.parametrize("w16", [False, True])
@pytest.mark.parametrize("g16", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_every_size(bits, g16, w16):
    k = len(SIZES)
    steps(tensors(1, SIZES, [bits] * k, [w16] * k, [g16] * k, [not w16] * k))


@pytest.mark.parametrize("offset", [1, 2, 3, 4, 8])
@pytest.mark.parametrize("bits", [32, 8])
def test_views_that_begin_anywhere(bits, offset):
    k = len(SIZES)
    mix = [i % 2 == 0 for i in range(k)]
    steps(tensors(2, SIZES, [bits] * k, mix, mix[::-1], [True] * k, offset), count=2)


def test_mixed_types_rates_and_decays_in_one_call():
    rng = np.random.default_rng(0)
    k = 30
    sizes = [int(n) for n in np.exp(rng.uniform(0, 11, k))]
    flip = lambda: [bool(x) for x in rng.integers(0, 2, k)]  # noqa: E731
    ts = tensors(3, sizes, [8 if x else 32 for x in flip()], flip(), flip(), flip())
    steps(ts, rates=[float(F(x)) for x in rng.uniform(0.1, 3, k)], decays=[float(x) for x in rng.integers(0, 2, k)])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("device_step,first,device_rate,scale", [(False, 1, False, None), (False, 1000, True, 0.25), (True, 100000, False, 1.0),
                                                                 (True, 2**31 - 5, True, -1.5)])
def test_ways_to_give_step_rate_and_factor(bits, device_step, first, device_rate, scale):
    k = 4
    ts = tensors(4, [300, 4096, 2, 777], [bits] * k, [False] * k, [False] * k, [False] * k)
    steps(ts, 2, device_step=device_step, first=first, device_rate=device_rate, scale=scale)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(beta1=0.0), dict(beta2=0.0), dict(beta1=0.0, beta2=0.0), dict(beta1=0.95, beta2=0.95, eps=1e-15), dict(eps=0.1),
                                dict(beta1=0.99, beta2=0.99999)])
def test_other_constants(bits, kw):
    steps(tensors(5, [1000, 257], [bits] * 2, [False] * 2, [True] * 2, [False] * 2), **kw)


@pytest.mark.parametrize("few", [True, False])
def test_more_tensors_than_a_launch_takes(few):
    k = 13 if few else 850
    ts = tensors(6, [(7 * i) % 600 if i % 5 else 0 for i in range(k)], [8 if i % 3 else 32 for i in range(k)], [i % 2 == 0 for i in range(k)],
                 [i % 7 == 0 for i in range(k)], [False] * k)
    steps(ts, 2)


def test_large_tensor_in_8_bits():
    """Larger than the launch's blocks take in one round; the definition on a sample of its 8-bit blocks."""
    import torch
    from paper_2509_13232_b200 import binding as B
    n = 9 * 2**20 + 17
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    w, grad = 0.02 * r(), 1e-3 * r()
    cm, cv = (r() * 40).clamp(-127, 127).to(torch.int8), (r().abs() * 80).clamp(1, 255).to(torch.uint8)
    nb = -(-n // 256)
    sm, sv = 1e-3 * torch.rand(nb, generator=g, device="cuda") + 1e-4, 1e-6 * torch.rand(nb, generator=g, device="cuda") + 1e-7
    pick = np.unique(np.concatenate([np.arange(3), np.arange(nb - 3, nb), np.random.default_rng(0).integers(0, nb, 300)]))
    cut = lambda t: np.concatenate([t[b * 256:b * 256 + 256].cpu().numpy() for b in pick])  # noqa: E731
    before = [cut(x) for x in (w, grad, cm, cv)]
    s0 = [x.cpu().numpy()[pick] for x in (sm, sv)]
    B.spo_adamw_update(B.adamw_list([w], [grad], [cm], [cv], [sm], [sv]), None, None, None, B.default_adamw_params(lr=1e-3, step=10), None)
    torch.cuda.synchronize()
    m, v = O.decode(before[2], s0[0], before[3], s0[1])         # (the picked last block is whole up to its end: the rest are whole)
    want, m1, v1, first = O.adamw(before[0], before[1], m, v, 10, lr=1e-3)
    em, es, ev, et = O.encode(m1, v1)
    assert np.array_equal(cut(cm), em) and np.array_equal(cut(cv), ev)
    assert np.array_equal(sm.cpu().numpy()[pick], es) and np.array_equal(sv.cpu().numpy()[pick], et)
    assert np.all(np.abs(cut(w) - want) <= 16 * U * first + U * (np.abs(want) + first))


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_usable(bits):
    import torch
    from paper_2509_13232_b200 import binding as B
    (t,) = tensors(7, [1000], [bits], [False], [False], [True])
    for i, x in ((0, np.nan), (3, np.inf), (300, -np.inf), (999, 3e38), (511, 2.0**61)):
        t["g"][i] = x
    t["g"][600], t["g"][601] = 2.0**59, -2.0**60
    t["dg"].copy_(torch.from_numpy(t["g"]))
    w0 = t["w"].copy()
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_adamw_update(table([t]), None, None, None, B.default_adamw_params(lr=1e-3, weight_decay=0.1, step=5), st)
    torch.cuda.synchronize()
    assert int(st[0]) == B.DEV_NONFINITE
    compare(t, *advance(t, 5))
    for i in (0, 3, 300, 511, 999):
        assert t["w"][i] == w0[i]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["scale", "lr"])
def test_a_step_that_is_not_taken(value, which):
    import torch
    from paper_2509_13232_b200 import binding as B
    ts = tensors(8, [5000, 300], [32, 8], [False] * 2, [False] * 2, [False] * 2)
    keep = [[t[k].clone() for k in ("dw", "dm", "dv")] for t in ts]
    bad, count = torch.tensor([value], device="cuda"), torch.tensor([4, 0], dtype=torch.int32, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    tab, p = table(ts), B.default_adamw_params()
    B.spo_adamw_update(tab, bad if which == "scale" else None, count, bad if which == "lr" else None, p, st)
    torch.cuda.synchronize()
    assert int(st[0]) == B.DEV_NONFINITE and count.tolist() == [4, 0]
    for t, k in zip(ts, keep):
        assert all(torch.equal(t[n], x) for n, x in zip(("dw", "dm", "dv"), k))
    B.spo_adamw_update(tab, None, count, None, p, None)              # the next one is the fifth
    torch.cuda.synchronize()
    assert count.tolist() == [5, 0]


@pytest.mark.parametrize("bits", [32, 8])
def test_from_nothing_and_zero_gradients(bits):
    import torch
    from paper_2509_13232_b200 import binding as B
    (t,) = tensors(9, [700], [bits], [False], [False], [False])
    t["g"][256:512] = 0
    t["g"][5] = 1e-30                                               # its square is no number of fp32
    t["g"][600] = 1e-17                                             # v > 0 far below the block's largest
    t["m"][:], t["v"][:] = 0, 0
    t["dg"].copy_(torch.from_numpy(t["g"]))
    for k in ("dm", "dv", "dsm", "dsv"):
        if t[k] is not None:
            t[k].zero_()
    for step in (1, 2, 3):
        B.spo_adamw_update(table([t]), None, None, None, B.default_adamw_params(lr=1e-3, step=step), None)
        torch.cuda.synchronize()
        compare(t, *advance(t, step, decay=0.0))
    if bits == 8:
        assert int(t["dv"][600]) == 1 and int(t["dv"][5]) == 0 and bool((t["dv"][256:512] == 0).all())


def test_every_border_between_codes():
    """Moments on and beside the borders: beta = 0 puts the gradient itself, and its square, into the moments."""
    import torch
    from paper_2509_13232_b200 import binding as B
    for power, top in ((2, 127), (4, 255)):
        values = []
        for j in range(1, top + 1):
            b = F((j - 0.5)**power)
            values += [np.nextafter(b, F(0)), b, np.nextafter(b, F(np.inf))]
        n = -(-len(values) // 255) * 256
        x = np.zeros(n, F)
        body = np.resize(np.array(values, F), n // 256 * 255)
        x.reshape(-1, 256)[:, 0], x.reshape(-1, 256)[:, 1:] = F(float(top**power)), body.reshape(-1, 255)
        g = np.where(np.arange(n) % 3 == 0, -x, x) if power == 2 else np.sqrt(x.astype(np.float64)).astype(F)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        w, cm, cv = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        sm, sv = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
        B.spo_adamw_update(B.adamw_list([w], [dev(g.astype(F))], [cm], [cv], [sm], [sv]), None, None, None,
                           B.default_adamw_params(beta1=0.0, beta2=0.0), None)
        torch.cuda.synchronize()
        want = O.encode(g.astype(F), (g.astype(F) * g.astype(F)).astype(F))
        for a, b in zip((cm, sm, cv, sv), want):
            assert np.array_equal(a.cpu().numpy(), b)


def test_decode():
    import torch
    from paper_2509_13232_b200 import binding as B
    rng = np.random.default_rng(3)
    for n, offset in ((1, 0), (255, 0), (256, 1), (1000, 3), (100000, 0), (3000017, 0)):
        nb = -(-n // 256)
        cm, cv = rng.integers(-127, 128, n).astype(np.int8), rng.integers(0, 256, n).astype(np.uint8)
        sm, sv = rng.random(nb).astype(F), (rng.random(nb) * 1e-9).astype(F)
        dev = lambda a: torch.from_numpy(np.concatenate([np.zeros(offset, a.dtype), a])).cuda()[offset:]  # noqa: E731
        m, v = torch.full((n + 8,), 5.0, device="cuda"), torch.full((n + 8,), 5.0, device="cuda")
        B.spo_adamw_decode(dev(cm), dev(sm), dev(cv), dev(sv), m[:n], v[:n])
        torch.cuda.synchronize()
        for got, want in zip((m, v), O.decode(cm, sm, cv, sv)):
            assert np.array_equal(got[:n].cpu().numpy(), want) and bool((got[n:] == 5).all())
        only = torch.empty(n, device="cuda")
        B.spo_adamw_decode(None, None, dev(cv), dev(sv), None, only)
        assert torch.equal(only, v[:n])


# ------------------------------------------------------------------------------------------------ gradient norm
def run_norm(gs, max_norm=0.0, scale=1.0):
    import torch
    from paper_2509_13232_b200 import binding as B
    out = torch.full((4,), float("nan"), device="cuda")
    n = B.spo_workspace_bytes(B.WS_GRAD_NORM)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    B.spo_grad_norm(B.grad_list(gs), out, ws[:n], st, max_norm=max_norm, grad_scale=scale)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    return [float(x) for x in out.cpu()], int(st[0])


def check_norm(gs, max_norm=0.0, scale=1.0):
    (norm, factor, fine, _), st = run_norm(gs, max_norm, scale)
    want, want_factor = O.grad_norm([g.double().cpu().numpy() for g in gs], max_norm, scale)
    assert abs(norm - want) <= 5 * U * want and fine == 1.0 and st == 0
    assert abs(factor - want_factor) <= 6 * U * abs(want_factor)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_of_every_size(bf16, offset):
    import torch
    dt = torch.bfloat16 if bf16 else torch.float32
    for n in [1, 2, 7, 8, 9, 255, 8191, 8192, 8193, 100000, 5000011]:
        g = torch.randn(n + offset, device="cuda").to(dt)[offset:]
        check_norm([g])
        check_norm([g], max_norm=1.0, scale=0.125)


def test_norm_of_many_tensors():
    import torch
    rng = np.random.default_rng(0)
    gs = [torch.randn(int(n), device="cuda").to(torch.bfloat16 if i % 2 else torch.float32) for i, n in enumerate(np.exp(rng.uniform(0, 10, 50)))]
    gs.insert(3, torch.empty(0, device="cuda"))
    check_norm(gs, 1.0)
    check_norm(gs, 1e9, -2.0)
    many = [gs[i % len(gs)][:300] for i in range(2600)]             # three launches; the same gradient may come twice
    check_norm(many, 1.0)
    check_norm(many[:1201])
    check_norm(many[:41])
    assert run_norm([]) == ([0.0, 1.0, 1.0, 0.0], 0)
    assert run_norm([torch.zeros(100000, device="cuda")], 1.0) == ([0.0, 1.0, 1.0, 0.0], 0)


@pytest.mark.parametrize("bf16", [False, True])
def test_norm_at_the_ends_of_the_range(bf16):
    import torch
    dt = torch.bfloat16 if bf16 else torch.float32
    for size in (1e-36, 1e-30, 1e-20, 1e15, 1e25, 1e33):            # squares beyond fp32 in both directions
        for n in (5, 20000):
            check_norm([(torch.randn(n, device="cuda") * size).to(dt)], max_norm=1.0)
    mixed = torch.randn(40000, device="cuda").to(dt)
    mixed[::3] *= 1e-30
    check_norm([mixed])
    for bad in (float("nan"), float("inf")):
        g = torch.randn(30000, device="cuda").to(dt)
        g[12345] = bad
        (norm, factor, fine, _), st = run_norm([torch.ones(3, device="cuda"), g], 1.0)
        assert not np.isfinite(norm) and np.isnan(factor) and fine == 0.0 and st == 2
    (norm, factor, fine, _), st = run_norm([torch.full((100,), 3e38, device="cuda")], 1.0)      # 3e39 is no fp32 number
    assert norm == float("inf") and np.isnan(factor) and st == 2


def test_clipped_step_captured_and_replayed():
    """Norm, factor, step and its count from one captured graph, replayed with other gradients and another rate, against plain calls."""
    import torch
    from paper_2509_13232_b200 import binding as B
    mk = lambda: tensors(11, [3000, 513, 70000], [32, 8, 8], [False, True, False], [True, False, True], [True, False, True])  # noqa: E731
    sides = []
    for _ in range(2):
        ts = mk()
        sides.append(dict(ts=ts, tab=table(ts), grads=B.grad_list([t["dg"] for t in ts]), out=torch.zeros(4, device="cuda"),
                          ws=torch.zeros(B.spo_workspace_bytes(B.WS_GRAD_NORM), dtype=torch.uint8, device="cuda"),
                          step=torch.zeros(2, dtype=torch.int32, device="cuda"), lr=torch.tensor([1e-3], device="cuda")))
    p = B.default_adamw_params(weight_decay=0.1)

    def call(s):
        B.spo_grad_norm(s["grads"], s["out"], s["ws"], None, max_norm=0.5)
        B.spo_adamw_update(s["tab"], s["out"][1:2], s["step"], s["lr"], p, None)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(sides[0])
    for k in range(4):
        for s in sides:
            s["lr"].fill_(1e-3 / (k + 1))
            for i, t in enumerate(s["ts"]):
                g = torch.Generator(device="cuda")
                g.manual_seed(10 * k + i)
                t["dg"].copy_(1e-2 * torch.randn(t["n"], generator=g, device="cuda"))
        graph.replay()
        call(sides[1])
        torch.cuda.synchronize()
        assert torch.equal(sides[0]["out"], sides[1]["out"]) and sides[0]["step"].tolist() == sides[1]["step"].tolist() == [k + 1, 0]
        for a, b in zip(sides[0]["ts"], sides[1]["ts"]):
            assert all(a[n] is None or torch.equal(a[n], b[n]) for n in ("dw", "dm", "dv", "dsm", "dsv", "dcopy"))


def test_two_streams_at_once():
    import torch
    from paper_2509_13232_b200 import binding as B
    p = B.default_adamw_params(lr=1e-3)
    alone, both = [tensors(s, [200000, 1000], [8, 32], [False] * 2, [False] * 2, [False] * 2) for s in (1, 2)], \
        [tensors(s, [200000, 1000], [8, 32], [False] * 2, [False] * 2, [False] * 2) for s in (1, 2)]
    for ts in alone:
        for _ in range(5):
            B.spo_adamw_update(table(ts), None, None, None, p, None)
    torch.cuda.synchronize()
    tabs, streams = [table(ts) for ts in both], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for tab, s in zip(tabs, streams):
            with torch.cuda.stream(s):
                B.spo_adamw_update(tab, None, None, None, p, None)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for x, y in zip(a, b):
            assert all(x[n] is None or torch.equal(x[n], y[n]) for n in ("dw", "dm", "dv", "dsm", "dsv"))


def test_the_tables_refuse():
    import torch
    from paper_2509_13232_b200 import binding as B
    x = lambda n=512, dt=torch.float32: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
    ok = dict(weights=[x(), x()], grads=[x(), x()], m=[x(), x()], v=[x(), x()])
    B.adamw_list(**ok)
    whole = x(1024)
    eight = dict(weights=[x()], grads=[x()], m=[x(dt=torch.int8)], v=[x(dt=torch.uint8)], m_scale=[x(2)], v_scale=[x(2)])
    B.adamw_list(**eight)
    shared = x()
    B.adamw_list(**{**ok, "grads": [shared, shared]})               # reading the same gradient twice is no harm
    for bad, err in ((dict(weights=[shared, shared]), ValueError), (dict(m=[shared, shared]), ValueError), (dict(grads=[ok["weights"][1], x()]), ValueError),
                     (dict(weights=[whole[:512], whole[256:768]]), ValueError), (dict(grads=[x(), x(511)]), ValueError), (dict(m=[x(), x(100)]), ValueError),
                     (dict(weights=[x(), x(dt=torch.float16)]), TypeError), (dict(v=[x(), x(dt=torch.bfloat16)]), TypeError),
                     (dict(weights=[x(), x().cpu()]), ValueError), (dict(copies=[x(), None]), TypeError), (dict(m=[x()]), ValueError),
                     (dict(grads=[x(), None]), TypeError), (dict(grads=[x(), x(1024)[::2]]), ValueError), (dict(m_scale=[x(2), None]), ValueError),
                     (dict(lr_scale=[1.0]), ValueError)):
        with pytest.raises(err):
            B.adamw_list(**{**ok, **bad})
    for bad, err in ((dict(m_scale=[x(1)]), ValueError), (dict(v_scale=None), ValueError), (dict(m=[x(dt=torch.uint8)]), TypeError), (dict(v_scale=[x(2).half()]), ValueError)):
        with pytest.raises(err):
            B.adamw_list(**{**eight, **bad})
    tab, p, ws, out = B.adamw_list(**ok), B.default_adamw_params(), x(1 << 16, torch.uint8), x(4)
    for args in ((x(2), None, None), (None, x(2), None), (None, None, x(1, torch.float64)), (x(1).cpu(), None, None)):
        with pytest.raises((TypeError, ValueError)):
            B.spo_adamw_update(tab, *args, p, None)
    with pytest.raises(B.SpoError):
        B.spo_adamw_update(tab, None, None, None, B.default_adamw_params(step=0), None)
    g = B.grad_list([x()])
    for args in ((x(3), ws), (out, x(16, torch.uint8)), (out.cpu(), ws)):
        with pytest.raises((ValueError, B.SpoError)):
            B.spo_grad_norm(g, *args, None)
    with pytest.raises((TypeError, ValueError)):
        B.spo_adamw_decode(x(dt=torch.int8), x(2), None, None, x(), x())
    with pytest.raises(ValueError):
        B.spo_adamw_decode(x(dt=torch.int8), x(3), None, None, x(), None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("bf16", [False, True])
def test_norm_and_factor_are_rounded_once(bf16):
    """The codes of 8-bit states hang on the factor's last bit, so it is the definition's: rounded once from a sum in 64 bits."""
    import torch
    for seed in range(20):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        n = int(10 ** (2 + seed / 4))
        x = (torch.randn(n, generator=g, device="cuda") * torch.exp(2 * torch.randn(n, generator=g, device="cuda"))).to(torch.bfloat16 if bf16 else torch.float32)
        (norm, factor, _, _), _ = run_norm([x[:n // 3], x[n // 3:]], 1.0)
        want = float(x.double().square().sum().sqrt())
        assert norm == float(F(want)) and factor == float(F(min(1.0, 1.0 / want)))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_of_zeros_and_few_extremes(bf16, offset):
    """Chunks of zeros (of both signs) with single values from the whole range, aligned and not, and infinities and NaN anywhere in one.
    All squares are exact in 64 bits and few, so the norm is the exact one rounded once; below fp32's normal numbers, to its grid."""
    import torch
    dtype = torch.bfloat16 if bf16 else torch.float32
    least = 2.0**-133 if bf16 else 2.0**-149
    n = 3 * 4096 + 17
    base = torch.zeros(n + 1, device="cuda", dtype=dtype)
    x = base[offset:offset + n]
    x[1::3] = -0.0
    assert run_norm([x], 1.0)[0] == [0.0, 1.0, 1.0, 0.0]
    for value in (least, 3 * least, 2.0**-126, 2.0**-112, 2.0**-95, 2.0**-90, 2.0**-50, 1.0, 2.0**62, 2.0**100, 1.75 * 2.0**127):
        for places in ((0,), (4095,), (n - 1,), (7, 8, 4096, n - 2)):
            x.zero_()
            x[list(places)] = value
            want = value * math.sqrt(len(places))
            norm, factor, fine, _ = run_norm([x], 1.0)[0]
            if want < 3.4e38:
                assert norm == float(F(want)) and factor == float(F(min(1.0, 1.0 / want))) and fine == 1.0
            else:
                assert norm == math.inf and math.isnan(factor) and fine == 0.0
    for value in (math.inf, -math.inf, math.nan):
        for place in (0, 5000, n - 1):
            x.fill_(0.5)
            x[place] = value
            norm, factor, fine, _ = run_norm([x], 1.0)[0]
            assert not norm < math.inf and math.isnan(factor) and fine == 0.0
