"""Operators around the hidden states and behind the gradients, with their plain forms: layer norm and RMS norm with their
backward pass, the global norm of many gradients with its clip factor, and the AdamW step over many tensors with states in
32 or 8 bits.

With `own` false, `run` computes an operator from elementary torch operations; with `own` true it calls the library
through its binding.  `exact` restates each operator in 64 bits.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6                                  # of the norms
LAYER, RMS = 0, 1
BLOCK = 256                                 # elements of an 8-bit state that share a scale
BETA1, BETA2, ADAM_EPS = (float(np.float32(x)) for x in (0.9, 0.999, 1e-8))
LR, DECAY = (float(np.float32(x)) for x in (1e-4, 0.1))
MAX_NORM = 1.0
M_FLOOR, V_FLOOR = 2.0**-100, 2.0**-90      # least scales of 8-bit states


# ------------------------------------------------------------------------------------------------ cases
def _fwd(name, T, d, kind, dtype="bf16", residual=False, bias=False, masked=False, pad=0):
    return dict(name=name, op="norm_fwd", T=T, d=d, kind=kind, dtype=dtype, residual=residual, bias=bias, masked=masked, pad=pad)


def _bwd(name, T, d, kind, dtype="bf16", dy="bf16", residual=False, bias=False, masked=False):
    return dict(name=name, op="norm_bwd", T=T, d=d, kind=kind, dtype=dtype, dy=dy, residual=residual, bias=bias, masked=masked)


def _gn(name, sizes, g):
    return dict(name=name, op="grad_norm", sizes=sizes, g=g)


def _aw(name, sizes, bits, w="f32", g="bf16", copy=True, clip=False):
    return dict(name=name, op="adamw", sizes=sizes, bits=bits, w=w, g=g, copy=copy, clip=clip)


def listed():
    return [
        # the final norm of one decoding token (latency)
        _fwd("norm one token", 1, 4096, RMS, residual=True),
        # the tiny fp32 configuration, prompt rows masked out
        _fwd("norm tiny fp32", 317, 64, LAYER, dtype="f32", bias=True, masked=True),
        # rows of an odd width inside a wider buffer
        _fwd("norm odd width", 2003, 2730, LAYER, bias=True, pad=3),
        # the final norm of a mini-batch at the large configuration, residual added on the way
        _fwd("norm mini-batch", 24000, 4096, RMS, residual=True),
        # one short response of the small bf16 configuration
        _bwd("norm backward response", 203, 1024, LAYER, bias=True),
        # an odd width in fp32
        _bwd("norm backward odd fp32", 4001, 1365, LAYER, dtype="f32", dy="f32", bias=True),
        # the mini-batch, with the gradient that reaches the residual stream past the norm, and fp32 gradients of H
        _bwd("norm backward mini-batch", 24000, 4096, RMS, dy="f32", residual=True, masked=True),
        # the gradients of one layer's projections
        _gn("gradient norm of a layer", "2x16777216+2x4194304+3x50331648+2x4096", "bf16"),
        # norms and biases of a model: many small tensors, 32-bit states (latency)
        _aw("adamw norms and biases", "129x4096", 32, w="f32", g="f32", copy=False),
        # the projections of one layer: fp32 weights, bf16 copy, clipped by their norm
        _aw("adamw layer clipped", "2x16777216+2x4194304+3x50331648+2x4096", 32, clip=True),
        # odd-sized projections and their biases, bf16 weights without a copy
        _aw("adamw 8 bits ragged", "4x2730000+4x2731", 8, w="bf16", copy=False),
        # the vocabulary matrix of the large configuration, with the fp32 gradient that the loss writes
        _aw("adamw 8 bits vocabulary", "1x622329856", 8, g="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "grad_norm", "adamw", "adamw"])
    if op in ("norm_fwd", "norm_bwd"):
        kind, dtype = rng.choice([LAYER, RMS]), rng.choice(["bf16", "bf16", "f32"])
        while True:
            T, d = _log_int(rng, 1, 24000), _log_int(rng, 16, 16384)
            if rng.random() < 0.6:
                d = max(64, d // 64 * 64)
            if T * d * (1 if dtype == "bf16" else 2) <= 24000 * 4096:
                break
        case = dict(op=op, T=T, d=d, kind=kind, dtype=dtype, residual=rng.random() < 0.5, bias=rng.random() < 0.4,
                    masked=rng.random() < 0.3)
        if op == "norm_fwd":
            case["pad"] = rng.choice([0, 0, 8, 5])
        else:
            case["dy"] = rng.choice(["bf16", "f32"]) if dtype == "bf16" else "f32"
        return case
    parts = []
    for _ in range(rng.randint(1, 4)):
        count = rng.choice([1, 1, 2, 4, 20, 60])
        parts.append("%dx%d" % (count, _log_int(rng, 1, 60000000 // count)))
    sizes, g = "+".join(parts), rng.choice(["bf16", "f32"])
    if op == "grad_norm":
        return dict(op=op, sizes=sizes, g=g)
    w = rng.choice(["f32", "bf16"])
    return dict(op=op, sizes=sizes, bits=rng.choice([8, 32]), w=w, g=g, copy=w == "f32" and rng.random() < 0.6,
                clip=rng.random() < 0.4)


def _sizes(case):
    """Elements of each tensor."""
    got = []
    for part in case["sizes"].split("+"):
        count, n = part.split("x")
        got += [int(n)] * int(count)
    return got


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _float(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _prepare_norm(case, g):
    T, d, dt = case["T"], case["d"], _float(case["dtype"])
    s = dict(case=case)
    # hidden states of unequal rows and columns, with an offset of the row's own
    x = _randn(g, T, d + case.get("pad", 0)) * torch.exp(0.3 * _randn(g, d + case.get("pad", 0)))
    x = x * torch.exp(0.5 * _randn(g, T, 1)) + 0.5 * _randn(g, T, 1)
    s["x"] = x.to(dt)[:, :d]
    s["weight"] = (1.0 + 0.2 * _randn(g, d)).to(dt)
    s["bias"] = (0.1 * _randn(g, d)).to(dt) if case["bias"] else None
    s["mask"] = (torch.rand(T, generator=g, device=DEV) < 0.75).to(torch.uint8) if case["masked"] else None
    if case["op"] == "norm_fwd":
        s["residual"] = _randn(g, T, d).to(dt) if case["residual"] else None
        return s
    h = s["x"].float()
    s["mean"] = h.mean(1) if case["kind"] == LAYER else None
    c = h - s["mean"][:, None] if case["kind"] == LAYER else h
    s["rstd"] = torch.rsqrt(c.square().mean(1) + EPS)
    s["dy"] = (1e-3 * _randn(g, T, d)).to(_float(case["dy"]))
    s["dh"] = (1e-3 * _randn(g, T, d)).to(dt) if case["residual"] else None
    return s


def _prepare_step(case, g):
    """Weights, gradients and states in one buffer each; every tensor begins on a block of its own and the rest of its last
    block is zero."""
    sizes = _sizes(case)
    at, total = [], 0
    for n in sizes:
        at.append((total, n))
        total += -(-n // BLOCK) * BLOCK
    s = dict(case=case, at=at, blocks=total // BLOCK)
    live = torch.ones(total, dtype=torch.bool, device=DEV)
    for begin, n in at:
        live[begin + n:begin + -(-n // BLOCK) * BLOCK] = False

    def spread(scale):      # blocks of unequal size, as rows of weight gradients are
        t = _randn(g, s["blocks"], BLOCK).mul_(torch.exp(_randn(g, s["blocks"], 1)).mul_(scale)).view(-1)
        return t.mul_(live)

    s["g"] = spread(1e-3).to(_float(case["g"]))
    if case["op"] == "grad_norm":
        return s
    s["w"] = spread(0.02).to(_float(case["w"]))
    s["copy"] = s["w"].to(torch.bfloat16) if case["copy"] else None
    if case["bits"] == 32:
        s["m"], s["v"] = spread(3e-4), spread(3e-4).square_()
    else:
        z = _randn(g, s["blocks"], BLOCK).clamp_(-3.5, 3.5).view(-1).mul_(live)
        s["m"] = torch.sign(z).mul_(torch.sqrt(z.abs() / 3.5).mul_(127).round_()).to(torch.int8)
        z = _randn(g, s["blocks"], BLOCK).clamp_(-3.5, 3.5).view(-1).mul_(live)
        s["v"] = torch.sqrt(z.abs_().div_(3.5)).mul_(255).ceil_().to(torch.uint8)
        s["m_scale"] = 1e-3 * torch.exp(0.5 * _randn(g, s["blocks"]))
        s["v_scale"] = 1e-6 * torch.exp(0.5 * _randn(g, s["blocks"]))
    s["factor"] = torch.full((1,), 0.75, device=DEV)
    s["step"] = torch.tensor([1000, 0], dtype=torch.int32, device=DEV)      # steps taken so far, and a spare word
    return s


def prepare(case, seed):
    g = _generator(seed)
    return _prepare_norm(case, g) if case["op"] in ("norm_fwd", "norm_bwd") else _prepare_step(case, g)


# ------------------------------------------------------------------------------------------------ plain forms
def _norm_fwd_plain(s):
    c, dt = s["case"], s["x"].dtype
    h = s["x"].float()
    out = {}
    live = None if s["mask"] is None else s["mask"].bool()[:, None]
    if s["residual"] is not None:
        h = (h + s["residual"].float()).to(dt)
        out["h"] = h if live is None else torch.where(live, h, torch.zeros_like(h))
        h = h.float()
    if c["kind"] == LAYER:
        mean = h.mean(1)
        out["mean"] = mean if live is None else torch.where(live[:, 0], mean, 0.0)
        h = h - mean[:, None]
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    out["rstd"] = rstd if live is None else torch.where(live[:, 0], rstd, 0.0)
    y = h * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out["y"] = (y if live is None else torch.where(live, y, 0.0)).to(dt)
    return out


def _norm_bwd_plain(s):
    c = s["case"]
    dy, xh = s["dy"].float(), s["x"].float()
    if s["mask"] is not None:
        dy = torch.where(s["mask"].bool()[:, None], dy, 0.0)
    if c["kind"] == LAYER:
        xh = xh - s["mean"][:, None]
    xh = xh * s["rstd"][:, None]
    a = dy * s["weight"].float()
    dx = a - xh * (a * xh).mean(1, keepdim=True)
    if c["kind"] == LAYER:
        dx = dx - a.mean(1, keepdim=True)
    dx = dx * s["rstd"][:, None]
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    if s["mask"] is not None:
        dx = torch.where(s["mask"].bool()[:, None], dx, 0.0)
    out = dict(dx=dx.to(s["x"].dtype), dw=(dy * xh).sum(0))
    if c["bias"]:
        out["db"] = dy.sum(0)
    return out


def _grad_norm_plain(s):
    norm = s["g"].double().square().sum().sqrt()
    factor = torch.clamp(MAX_NORM / norm, max=1.0)
    return dict(norm=norm.float(), factor=factor.float())


def _decode(m, m_scale, v, v_scale):
    m = m.view(-1, BLOCK).float()
    m = m * m.abs() * (m_scale * (1.0 / 16129.0))[:, None]
    v = v.view(-1, BLOCK).float()
    v = v * v
    return m.view(-1), (v * v * (v_scale * (1.0 / 255.0**4))[:, None]).view(-1)


def _encode(x, floor, count, power):
    """(codes of the magnitudes, scales): a code is the number of borders (j - 1/2)^power, j = 1 .. count, at or below the value."""
    x = x.view(-1, BLOCK).abs()
    scale = x.amax(1).clamp(min=floor)
    border = torch.tensor([(j - 0.5)**power for j in range(1, count + 1)], dtype=torch.float32, device=x.device)
    top = torch.full_like(scale, float(count**power))
    code = torch.bucketize(x * (top / scale)[:, None], border, right=True, out_int32=True)
    return code.view(-1), scale


def _adamw_plain(s):
    c = s["case"]
    f = _grad_norm_plain(s)["factor"] if c["clip"] else s["factor"]
    g = s["g"].float() * f
    if c["bits"] == 8:
        m, v = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    s["step"][:1].add_(1)
    t = s["step"][0].double()
    rate = (-LR / torch.expm1(t * math.log(BETA1))).float()
    root = torch.sqrt(-torch.expm1(t * math.log(BETA2))).float()
    w = s["w"].float()
    w = w - (rate * (m / (torch.sqrt(v) / root + ADAM_EPS)) + (LR * DECAY) * w)
    s["w"].copy_(w)
    out = dict(w=s["w"], step=s["step"])
    if c["copy"]:
        s["copy"].copy_(w)
        out["copy"] = s["copy"]
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
        return out
    code, scale = _encode(m, M_FLOOR, 127, 2)
    s["m"].copy_(torch.where(m < 0, -code, code))
    s["m_scale"].copy_(scale)
    code, scale = _encode(v, V_FLOOR, 255, 4)
    s["v"].copy_(torch.where(v > 0, code.clamp(min=1), code))
    s["v_scale"].copy_(scale)
    out["m"], out["v"] = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
    return out


# ------------------------------------------------------------------------------------------------ the library's calls
def _own_buffers(s, B):
    """Output buffers, scratch and tables of tensors, made at a state's first call and kept, as a training or serving loop
    keeps them."""
    c = s["case"]
    s["status"] = torch.zeros(4, dtype=torch.int32, device=DEV)
    f32 = dict(dtype=torch.float32, device=DEV)
    if c["op"] == "norm_fwd":
        T, d, dt = c["T"], c["d"], s["x"].dtype
        s["y"] = torch.empty(T, d, dtype=dt, device=DEV)
        s["h"] = torch.empty(T, d, dtype=dt, device=DEV) if c["residual"] else None
        s["mean"] = torch.empty(T, **f32) if c["kind"] == LAYER else None
        s["rstd"] = torch.empty(T, **f32)
        s["ready"] = True
        return
    if c["op"] == "norm_bwd":
        T, d = c["T"], c["d"]
        s["dx"] = torch.empty(T, d, dtype=s["x"].dtype, device=DEV)
        s["dw"] = torch.empty(d, **f32)
        s["db"] = torch.empty(d, **f32) if c["bias"] else None
        s["ws"] = torch.empty(B.spo_workspace_bytes(B.WS_LAYERNORM_BWD, T=T, d=d), dtype=torch.uint8, device=DEV)
        s["ready"] = True
        return
    cut = lambda name: [s[name][b:b + n] for b, n in s["at"]]  # noqa: E731
    scales = lambda name: [s[name][b // BLOCK:b // BLOCK + -(-n // BLOCK)] for b, n in s["at"]]  # noqa: E731
    if c["op"] == "grad_norm" or c["clip"]:
        s["grads"] = B.grad_list(cut("g"))
        s["norm"] = torch.empty(4, **f32)
        s["ws"] = torch.empty(B.spo_workspace_bytes(B.WS_GRAD_NORM, N=s["g"].numel()), dtype=torch.uint8, device=DEV)
    if c["op"] == "adamw":
        eight = c["bits"] == 8
        s["tensors"] = B.adamw_list(cut("w"), cut("g"), cut("m"), cut("v"), scales("m_scale") if eight else None,
                                    scales("v_scale") if eight else None, cut("copy") if c["copy"] else None)
        s["params"] = B.default_adamw_params(lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY)
        if eight:
            s["m_out"], s["v_out"] = torch.empty(s["m"].numel(), **f32), torch.empty(s["v"].numel(), **f32)
    s["ready"] = True


def _run_own(s):
    from paper_2509_13232_b200 import binding as B
    if "ready" not in s:
        _own_buffers(s, B)
    c = s["case"]
    if c["op"] == "norm_fwd":
        B.spo_layernorm_fwd(s["x"], s["residual"], s["weight"], s["bias"], s["mask"], s["y"], s["h"], s["mean"], s["rstd"],
                            s["status"], eps=EPS, kind=c["kind"])
        return {k: s[k] for k in ("h", "mean", "rstd", "y") if s[k] is not None}
    if c["op"] == "norm_bwd":
        B.spo_layernorm_bwd(s["dy"], s["x"], s["weight"], s["mask"], s["mean"], s["rstd"], s["dh"], s["dx"], s["dw"], s["db"], 0,
                            s["ws"], s["status"], kind=c["kind"])
        return {k: s[k] for k in ("dx", "dw", "db") if s[k] is not None}
    if "grads" in s:
        B.spo_grad_norm(s["grads"], s["norm"], s["ws"], s["status"], max_norm=MAX_NORM)
        if c["op"] == "grad_norm":
            return dict(norm=s["norm"][0], factor=s["norm"][1])
    B.spo_adamw_update(s["tensors"], s["norm"][1:2] if c["clip"] else s["factor"], s["step"], None, s["params"], s["status"])
    out = dict(w=s["w"], step=s["step"])
    if c["copy"]:
        out["copy"] = s["copy"]
    if c["bits"] == 8:
        B.spo_adamw_decode(s["m"], s["m_scale"], s["v"], s["v_scale"], s["m_out"], s["v_out"])
        out["m"], out["v"] = s["m_out"], s["v_out"]
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"norm_fwd": _norm_fwd_plain, "norm_bwd": _norm_bwd_plain, "grad_norm": _grad_norm_plain,
            "adamw": _adamw_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    size = lambda t: 2 if t == "bf16" else 4  # noqa: E731
    if case["op"] in ("norm_fwd", "norm_bwd"):
        T, d, b, layer = case["T"], case["d"], size(case["dtype"]), case["kind"] == LAYER
        row = 4 * (2 if layer else 1) + case["masked"]
        if case["op"] == "norm_fwd":
            return dict(bytes=T * d * b * (4 if case["residual"] else 2) + d * b * (1 + case["bias"]) + T * row,
                        flops=T * d * (8.0 if layer else 5.0))
        return dict(bytes=T * d * (size(case["dy"]) + b * (3 if case["residual"] else 2)) + d * (b + 4 * (1 + case["bias"])) + T * row,
                    flops=T * d * 14.0)
    n = sum(_sizes(case))
    if case["op"] == "grad_norm":
        return dict(bytes=n * size(case["g"]), flops=2.0 * n)
    # 8 bits: the codes in and out, their scales, and the values that they stand for
    state = 4 + 16 / BLOCK + 8 if case["bits"] == 8 else 16
    return dict(bytes=n * (2 * size(case["w"]) + size(case["g"]) + 2 * case["copy"] + state), flops=n * (16.0 + 2 * case["clip"]))


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_norm(s):
    c = s["case"]
    keep = torch.ones(c["T"], dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].bool()
    x, w = s["x"].double(), s["weight"].double()
    if c["op"] == "norm_fwd":
        out = {}
        if c["residual"]:
            out["h"] = x + s["residual"].double()
            x = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()     # h as it is stored
        mu = x.sum(1) / c["d"] if c["kind"] == LAYER else torch.zeros(c["T"], dtype=torch.float64, device=DEV)
        rstd = ((x - mu[:, None])**2).sum(1).div(c["d"]).add(EPS).pow(-0.5)
        if c["kind"] == LAYER:
            out["mean"] = mu
        out["rstd"] = rstd
        out["y"] = torch.addcmul(torch.zeros_like(w) if s["bias"] is None else s["bias"].double(), (x - mu[:, None]) * rstd[:, None], w)
        for k in out:
            out[k][~keep] = 0.0
        return out
    # gradients through the formula's parts: xh = rstd (x - mean), with mean and rstd as given
    dy = s["dy"].double()
    dy[~keep] = 0.0
    mu = s["mean"].double() if c["kind"] == LAYER else torch.zeros(c["T"], dtype=torch.float64, device=DEV)
    r = s["rstd"].double()[:, None]
    xh = (x - mu[:, None]) * r
    out = dict(dw=torch.einsum("td,td->d", dy, xh))
    if c["bias"]:
        out["db"] = dy.sum(0)
    up = dy * w
    along = torch.einsum("td,td->t", up, xh)[:, None] / c["d"]
    level = up.sum(1, keepdim=True) / c["d"] if c["kind"] == LAYER else 0.0
    dx = r * (up - level - along * xh)
    if s["dh"] is not None:
        dx += s["dh"].double()
    dx[~keep] = 0.0
    out["dx"] = dx
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm_fwd", "norm_bwd"):
        return _exact_norm(s)
    f = 1.0
    if case["op"] == "grad_norm" or case["clip"]:
        total = sum(float(torch.linalg.vector_norm(s["g"][b:b + n].double()))**2 for b, n in s["at"])
        norm = math.sqrt(total)
        f = MAX_NORM / norm if norm > MAX_NORM else 1.0
        if case["op"] == "grad_norm":
            return dict(norm=torch.tensor(norm, dtype=torch.float64), factor=torch.tensor(f, dtype=torch.float64))
    else:
        f = float(s["factor"][0])
    g = s["g"].double() * f
    if case["bits"] == 8:       # the state's values; the new codes have no counterpart in 64 bits
        m = s["m"].double()
        m = m.abs().mul_(m).view(-1, BLOCK).mul_(s["m_scale"].double()[:, None] / 127**2).view(-1)
        v = s["v"].double().pow_(4).view(-1, BLOCK).mul_(s["v_scale"].double()[:, None] / 255**4).view(-1)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square_()
    t = int(s["step"][0]) + 1
    w = s["w"].double()
    w = (1 - LR * DECAY) * w - LR * (m / (1 - BETA1**t)) / ((v / (1 - BETA2**t)).sqrt_() + ADAM_EPS)
    out = dict(w=w, step=torch.tensor([t, 0], dtype=torch.int32, device=DEV))
    if case["copy"]:
        out["copy"] = w
    out["m"], out["v"] = (None, None) if case["bits"] == 8 else (m, v)
    return out
