"""Operators around the policy loss, with their plain forms: log-probabilities of given tokens straight from hidden
states (with entropy and top alternatives), their backward pass, and the orthogonalised (Muon) weight update.

With `own` false, `run` computes an operator from elementary torch operations in 32 bits; with `own` true it calls the
library through its binding.  `exact` restates each operator in 64 bits.
"""

import math

import torch

own = False

DEV = "cuda"
NS = (3.4445, -4.7750, 2.0315)      # quintic Newton-Schulz coefficients of the Muon optimiser
NS_STEPS = 5
NS_EPS = 1e-7


# ------------------------------------------------------------------------------------------------ cases
def _lp(name, T, d, V, dtype="bf16", top_k=0, entropy=True, masked=False, inv_t=1.0, pad=0):
    return dict(name=name, op="logprobs", T=T, d=d, V=V, dtype=dtype, top_k=top_k, entropy=entropy, masked=masked,
                inv_t=inv_t, pad=pad)


def _bw(name, T, d, V, dtype="bf16", entropy=True, masked=False, inv_t=1.0):
    return dict(name=name, op="logprobs_bwd", T=T, d=d, V=V, dtype=dtype, entropy=entropy, masked=masked, inv_t=inv_t)


def _ns(name, op, batch, m, n, dtype="f32"):
    return dict(name=name, op=op, batch=batch, m=m, n=n, dtype=dtype)


def listed():
    return [
        # one new token of one sequence: the whole of W is read for a single row (latency, HBM stream)
        _lp("logprobs one token", 1, 4096, 151936, top_k=20),
        # a decoding batch, last-token rows of a wider buffer, sampled at temperature 0.7
        _lp("logprobs decode batch", 48, 4096, 151936, top_k=8, inv_t=1.0 / 0.7, pad=64),
        # the tiny fp32 configuration, prompt tokens masked out
        _lp("logprobs tiny fp32", 317, 64, 512, dtype="f32", top_k=5, masked=True),
        # one long response of the small bf16 configuration, no alternatives wanted
        _lp("logprobs one response", 1531, 1024, 151936),
        # old log-probs of a mini-batch chunk at the large configuration, tool tokens masked out
        _lp("logprobs mini-batch", 8000, 4096, 151936, top_k=8, masked=True),
        # gradient of log-probs and entropy, one short response over a mid-sized vocabulary
        _bw("backward short response", 203, 1024, 32000, masked=True),
        # the tiny fp32 configuration
        _bw("backward tiny fp32", 317, 64, 512, dtype="f32"),
        # a few responses at the large configuration
        _bw("backward mini-batch", 4001, 4096, 151936, inv_t=1.0 / 0.9),
        # a small projection: many launches on little data
        _ns("orthogonalize small", "orthogonalize", 1, 128, 512),
        # the gradient of a feed-forward projection, more rows than columns, accumulated in bf16
        _ns("orthogonalize tall", "orthogonalize", 1, 12288, 4096, dtype="bf16"),
        # the step of one attention output projection
        _ns("muon square", "muon_update", 1, 4096, 4096),
        # four layers' odd-sized projections in one call
        _ns("muon ragged layers", "muon_update", 4, 1000, 2730),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_bwd", "orthogonalize", "muon_update"])
    if op in ("orthogonalize", "muon_update"):
        batch = rng.choice([1, 1, 2, 3, 5])
        while True:
            m, n = _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)
            if _ns_flops(batch, m, n) <= _ns_flops(1, 12288, 4096):
                break
        return dict(op=op, batch=batch, m=m, n=n, dtype=rng.choice(["f32", "bf16"]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    inv_t = rng.choice([1.0, 1.0, 1.25, 1.0 / 0.7])
    entropy, masked = rng.random() < 0.6, rng.random() < 0.4
    if dtype == "f32":
        T, d, V = _log_int(rng, 1, 700), 4 * _log_int(rng, 8, 256), _log_int(rng, 300, 20000)
    else:
        d = 64 * _log_int(rng, 1, 64)
        V = _log_int(rng, 500, 151936)
        T = _log_int(rng, 1, 6000 if op == "logprobs" else 3000)
    case = dict(op=op, T=T, d=d, V=V, dtype=dtype, entropy=entropy, masked=masked, inv_t=inv_t)
    if op == "logprobs":
        case["top_k"] = rng.choice([0, 1, 5, 8, 20])
        case["pad"] = rng.choice([0, 0, 8, 128])
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _float(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] in ("orthogonalize", "muon_update"):
        b, m, n = case["batch"], case["m"], case["n"]
        r = max(1, min(m, n) // 4)

        def gradient():     # a strong low-rank part under noise, as gradients of projections have
            return (_randn(g, b, m, r) @ _randn(g, b, r, n)) * (1e-3 / math.sqrt(r)) + 3e-4 * _randn(g, b, m, n)

        state = dict(case=case, G=gradient().to(_float(case["dtype"])))
        if case["op"] == "muon_update":
            state["W"] = (0.02 * _randn(g, b, m, n)).to(torch.bfloat16)
            state["momentum"] = 5.0 * gradient()
            state["lr"], state["mu"], state["decay"] = 0.02, 0.95, 0.1
        return state
    T, d, V = case["T"], case["d"], case["V"]
    H, W = _randn(g, T, d + case.get("pad", 0)), _randn(g, V, d).mul_(0.02 if d > 512 else 0.05)
    if case.get("top_k"):
        # Values on a grid (steps 2^-5 and 2^-9), so that every logit is an exact 32-bit sum whatever the order of its
        # terms: the order of the alternatives is then the definition's and not that of the summation.
        H.mul_(32).round_().div_(32).clamp_(-7.75, 7.75)
        W.mul_(512).round_().div_(512)
    H, W = H.to(_float(case["dtype"]))[:, :d], W.to(_float(case["dtype"]))
    state = dict(case=case, H=H, W=W, inv_t=case["inv_t"], top_k=case.get("top_k", 0), entropy=case["entropy"])
    state["y"] = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    state["mask"] = (torch.rand(T, generator=g, device=DEV) < 0.75).to(torch.uint8) if case["masked"] else None
    if case["op"] == "logprobs_bwd":
        z = (H.float() @ W.float().T) * case["inv_t"]
        state["lse"] = torch.logsumexp(z, 1)
        z.sub_(state["lse"][:, None])
        state["ent"] = -(z.exp() * z).sum(1)
        state["g_logp"] = _randn(g, T) / T
        state["g_lse"] = 0.01 * _randn(g, T) / T
        state["g_ent"] = 0.1 * _randn(g, T) / T if case["entropy"] else None
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _keys(z):
    """64-bit keys whose descending order is that of the values, equal ones by ascending column."""
    bits = (z + 0.0).view(torch.int32).to(torch.int64)
    bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    return (bits << 32) | (z.shape[1] - 1 - torch.arange(z.shape[1], device=z.device))


def _logprobs_plain(s):
    z = s["H"].float() @ s["W"].float().T
    top = torch.topk(_keys(z), s["top_k"], dim=1).values if s["top_k"] else None
    z = z * s["inv_t"]
    big = z.amax(1)
    e = torch.exp(z - big[:, None])
    total = e.sum(1)
    lse = big + torch.log(total)
    live = torch.ones_like(lse) if s["mask"] is None else s["mask"].float()
    out = dict(logp=torch.where(live > 0, z.gather(1, s["y"].long()[:, None])[:, 0] - lse, 0.0),
               lse=torch.where(live > 0, lse, 0.0))
    if s["entropy"]:
        out["entropy"] = torch.where(live > 0, lse - (e * z).sum(1) / total, 0.0)
    if top is not None:
        ids = z.shape[1] - 1 - (top & 0xFFFFFFFF)
        out["top_ids"] = torch.where(live[:, None] > 0, ids, -1).to(torch.int32)
        out["top_logp"] = torch.where(live[:, None] > 0, z.gather(1, ids) - lse[:, None], 0.0)
    return out


def _logprobs_bwd_plain(s):
    H, W = s["H"].float(), s["W"].float()
    u = (H @ W.T).mul_(s["inv_t"]).sub_(s["lse"][:, None])        # log p
    a = s["g_lse"] - s["g_logp"]
    p = torch.exp(u)
    if s["g_ent"] is not None:
        g = p * (a[:, None] - s["g_ent"][:, None] * (u + s["ent"][:, None]))
    else:
        g = p * a[:, None]
    g.scatter_add_(1, s["y"].long()[:, None], s["g_logp"][:, None])
    g.mul_(s["inv_t"])
    if s["mask"] is not None:
        g.mul_(s["mask"].float()[:, None])
    return dict(dH=(g @ W).to(s["H"].dtype), dW=(g.T @ H).to(s["W"].dtype))


def _newton_schulz_plain(x):
    """[b, m, n], m <= n"""
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        gram = x @ x.mT
        x = NS[0] * x + (NS[1] * gram + NS[2] * (gram @ gram)) @ x
    return x


def _orthogonalize_plain(s):
    x = s["G"].float()
    x = _newton_schulz_plain(x.mT).mT if x.shape[1] > x.shape[2] else _newton_schulz_plain(x)
    return dict(out=x.to(torch.bfloat16).contiguous())


def _muon_plain(s):
    g = s["G"].float()
    s["momentum"].mul_(s["mu"]).add_(g)
    x = g + s["mu"] * s["momentum"]
    x = _newton_schulz_plain(x.mT).mT if x.shape[1] > x.shape[2] else _newton_schulz_plain(x)
    scale = 0.2 * math.sqrt(max(x.shape[1], x.shape[2]))
    s["W"].copy_(s["W"].float() * (1.0 - s["lr"] * s["decay"]) - s["lr"] * scale * x)
    return dict(W=s["W"], momentum=s["momentum"])


# ------------------------------------------------------------------------------------------------ the library's calls
def _own_buffers(s, B):
    """Output buffers and scratch, allocated at a state's first call and kept, as a training or serving loop keeps them."""
    c = s["case"]
    s["status"] = torch.zeros(4, dtype=torch.int32, device=DEV)
    if c["op"] in ("orthogonalize", "muon_update"):
        s["params"] = B.default_muon_params(steps=NS_STEPS, coef_a=NS[0], coef_b=NS[1], coef_c=NS[2], eps=NS_EPS)
        if c["op"] == "muon_update":
            for k, v in (("lr", s["lr"]), ("momentum", s["mu"]), ("weight_decay", s["decay"]), ("nesterov", 1),
                         ("scale_mode", B.MUON_SCALE_RMS)):
                setattr(s["params"], k, v)
        else:
            s["out"] = torch.empty(c["batch"], c["m"], c["n"], dtype=torch.bfloat16, device=DEV)
        n = B.spo_workspace_bytes(B.WS_MUON, T=c["m"], d=c["n"], B=c["batch"])
    else:
        T, d, V = c["T"], c["d"], c["V"]
        f32 = dict(dtype=torch.float32, device=DEV)
        if c["op"] == "logprobs":
            s["logp"], s["lse"] = torch.empty(T, **f32), torch.empty(T, **f32)
            s["ent"] = torch.empty(T, **f32) if s["entropy"] else None
            k = s["top_k"]
            s["top_ids"] = torch.empty(T, k, dtype=torch.int32, device=DEV) if k else None
            s["top_logp"] = torch.empty(T, k, **f32) if k else None
            n = B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=d, V=V, B=k)
        else:
            s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(s["W"])
            n = B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=T, d=d, V=V)
    s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


def _run_own(s):
    from paper_2509_13232_b200 import binding as B
    if "ws" not in s:
        _own_buffers(s, B)
    op = s["case"]["op"]
    if op == "logprobs":
        B.spo_logprobs(s["H"], s["W"], s["y"], s["mask"], s["logp"], s["lse"], s["ent"], s["top_ids"], s["top_logp"],
                       s["ws"], s["status"], inv_temperature=s["inv_t"])
        out = dict(logp=s["logp"], lse=s["lse"])
        if s["entropy"]:
            out["entropy"] = s["ent"]
        if s["top_k"]:
            out["top_ids"], out["top_logp"] = s["top_ids"], s["top_logp"]
        return out
    if op == "logprobs_bwd":
        B.spo_logprobs_bwd(s["H"], s["W"], s["y"], s["mask"], s["lse"], s["ent"] if s["entropy"] else None, s["g_logp"],
                           s["g_lse"], s["g_ent"], s["dH"], s["dW"], 0, s["ws"], s["status"],
                           inv_temperature=s["inv_t"])
        return dict(dH=s["dH"], dW=s["dW"])
    if op == "orthogonalize":
        B.spo_orthogonalize(s["G"], s["out"], s["ws"], s["params"], s["status"])
        return dict(out=s["out"])
    B.spo_muon_update(s["W"], s["momentum"], s["G"], s["ws"], s["params"], s["status"])
    return dict(W=s["W"], momentum=s["momentum"])


def run(state):
    if own:
        return _run_own(state)
    return {"logprobs": _logprobs_plain, "logprobs_bwd": _logprobs_bwd_plain, "orthogonalize": _orthogonalize_plain,
            "muon_update": _muon_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ accounting
def _ns_flops(batch, m, n):
    """The Gram matrix and its square are symmetric (half their products), the third product is full."""
    m, n = min(m, n), max(m, n)
    return NS_STEPS * batch * (3.0 * m * m * n + 1.0 * m ** 3)


def work(case):
    if case["op"] in ("orthogonalize", "muon_update"):
        e = case["batch"] * case["m"] * case["n"]
        size = 2 if case["dtype"] == "bf16" else 4
        moved = e * size + (e * 2 if case["op"] == "orthogonalize" else e * (2 * 2 + 2 * 4))
        return dict(bytes=moved, flops=_ns_flops(case["batch"], case["m"], case["n"]))
    T, d, V = case["T"], case["d"], case["V"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "logprobs":
        return dict(bytes=(T + V) * d * size + T * (4 + 8 + 4 * bool(case["entropy"]) + 8 * case["top_k"]),
                    flops=2.0 * T * d * V)
    return dict(bytes=2 * (T + V) * d * size + T * 24, flops=6.0 * T * d * V)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("orthogonalize", "muon_update"):
        x = s["G"].double()
        res = {}
        if case["op"] == "muon_update":
            res["momentum"] = s["mu"] * s["momentum"].double() + x
            x = x + s["mu"] * res["momentum"]
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + NS_EPS)
        a, b, c = NS
        for _ in range(NS_STEPS):
            # a X + b (X X^T) X + c (X X^T)^2 X, evaluated over the smaller of the two Gram matrices
            if x.shape[1] <= x.shape[2]:
                q = x @ x.transpose(1, 2)
                x = a * x + b * (q @ x) + c * (q @ (q @ x))
            else:
                q = x.transpose(1, 2) @ x
                x = a * x + b * (x @ q) + c * ((x @ q) @ q)
        if case["op"] == "orthogonalize":
            return dict(out=x)
        step = s["lr"] * 0.2 * math.sqrt(max(case["m"], case["n"]))
        res["W"] = s["W"].double() - s["lr"] * s["decay"] * s["W"].double() - step * x
        return res
    H, W, it = s["H"].double(), s["W"].double(), case["inv_t"]
    T, V = case["T"], case["V"]
    rows = max(1, int(4e8) // V)
    keep = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].bool()
    if case["op"] == "logprobs":
        parts = []
        for t in range(0, T, rows):
            raw = H[t:t + rows] @ W.T
            lp = torch.log_softmax(raw * it, dim=1)
            k = keep[t:t + rows]
            y = s["y"][t:t + rows].long()
            o = dict(logp=lp.gather(1, y[:, None])[:, 0] * k, lse=torch.logsumexp(raw * it, 1) * k)
            if case["entropy"]:
                o["entropy"] = -(lp.exp() * lp).sum(1) * k
            if case["top_k"]:
                order, ids = raw.clone(), []
                for _ in range(case["top_k"]):
                    best = order.amax(1, keepdim=True)
                    col = torch.arange(V, device=DEV).expand_as(order).masked_fill(order != best, V).amin(1, keepdim=True)
                    ids.append(col)
                    order.scatter_(1, col, -math.inf)
                ids = torch.cat(ids, 1)
                o["top_ids"] = ids.masked_fill(~k[:, None], -1).to(torch.int32)
                o["top_logp"] = lp.gather(1, ids).masked_fill(~k[:, None], 0.0)
            parts.append(o)
        return {key: torch.cat([o[key] for o in parts]) for key in parts[0]}
    dH, dW = torch.empty_like(H), torch.zeros_like(W)
    for t in range(0, T, rows):
        sl = slice(t, t + rows)
        lp = (H[sl] @ W.T) * it - s["lse"][sl].double()[:, None]
        p = lp.exp()
        dz = -p * s["g_logp"][sl].double()[:, None] + p * s["g_lse"][sl].double()[:, None]
        if s["g_ent"] is not None:
            dz -= s["g_ent"][sl].double()[:, None] * p * (lp + s["ent"][sl].double()[:, None])
        at = torch.arange(dz.shape[0], device=DEV)
        dz[at, s["y"][sl].long()] += s["g_logp"][sl].double()
        dz[~keep[sl]] = 0.0
        dH[sl] = it * (dz @ W)
        dW += it * (dz.T @ H[sl])
    return dict(dH=dH, dW=dW)
