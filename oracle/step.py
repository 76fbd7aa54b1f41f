"""Float64 CPU definitions of the norms around the hidden states and of what follows the gradients: layer norm and RMS norm with their
gradients, the global gradient norm, and the AdamW step with states in 32 or 8 bits.

Test infrastructure only: numpy, written from the formulas, sharing nothing with the CUDA path.  Pinned in tests/test_step_host.py by
closed forms and finite differences.  The moments and codes of adamw() are formed in fp32, operation by operation, because that is how
they are defined; everything else is in 64 bits.
"""

from __future__ import annotations

import math

import numpy as np

LAYER, RMS = 0, 1
BLOCK = 256
F = np.float32


def round_bf16(x):
    """Nearest bf16 (ties to even) of finite values, as float64."""
    b = np.asarray(x, F).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(F).astype(np.float64)


def layernorm(x, weight=None, bias=None, residual=None, mask=None, eps=1e-6, kind=LAYER, bf16=False):
    """dict(h, mean, rstd, y); h is x + residual rounded to the rows' type, as it is stored."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        s = (np.asarray(x, F) + np.asarray(residual, F)).astype(F)
        h = round_bf16(s) if bf16 else s.astype(np.float64)
    t, d = h.shape
    mean = h.mean(axis=1) if kind == LAYER else np.zeros(t)
    c = h - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
    w = np.ones(d) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(d) if bias is None else np.asarray(bias, np.float64)
    out = dict(h=h, mean=mean, rstd=rstd, y=c * rstd[:, None] * w + b)
    if mask is not None:
        off = np.asarray(mask) == 0
        for k in out:
            out[k] = np.where(off if out[k].ndim == 1 else off[:, None], 0.0, out[k])
    return out


def layernorm_backward(dy, x, mean, rstd, weight=None, dh=None, mask=None, kind=LAYER):
    """dict(dx, dw, db) for the statistics as given."""
    dy, x = np.array(dy, np.float64), np.array(x, np.float64)
    t, d = x.shape
    keep = np.ones(t, bool) if mask is None else np.asarray(mask) != 0
    dy[~keep], x[~keep] = 0.0, 0.0
    mu = np.where(keep, np.asarray(mean, np.float64), 0.0) if kind == LAYER else np.zeros(t)
    r = np.where(keep, np.asarray(rstd, np.float64), 0.0)
    xh = (x - mu[:, None]) * r[:, None]
    a = dy * (np.ones(d) if weight is None else np.asarray(weight, np.float64))
    inner = a - xh * (a * xh).mean(axis=1, keepdims=True)
    if kind == LAYER:
        inner = inner - a.mean(axis=1, keepdims=True)
    dx = r[:, None] * inner
    if dh is not None:
        dx = dx + np.where(keep[:, None], np.asarray(dh, np.float64), 0.0)
    return dict(dx=dx, dw=(dy * xh).sum(axis=0), db=dy.sum(axis=0), xh=xh, a=a)


def grad_norm(grads, max_norm=0.0, scale=1.0):
    """(norm, factor)"""
    norm = abs(scale) * math.sqrt(math.fsum(float((np.asarray(g, np.float64)**2).sum()) for g in grads))
    return norm, scale * (max_norm / norm if max_norm > 0 and norm > max_norm else 1.0)


def _blocks(x):
    n = x.size
    return np.concatenate([x.reshape(-1), np.zeros(-n % BLOCK, x.dtype)]).reshape(-1, BLOCK)


def decode(m, m_scale, v, v_scale):
    """fp32 values of 8-bit states."""
    n = m.size
    c = _blocks(np.asarray(m, np.int32)).astype(F)
    um = (np.asarray(m_scale, F) * F(1.0 / 127**2))[:, None]
    q = _blocks(np.asarray(v, np.int64)).astype(F)
    uv = (np.asarray(v_scale, F) * F(1.0 / 255**4))[:, None]
    q2 = q * q
    return (c * np.abs(c) * um).reshape(-1)[:n], (q2 * q2 * uv).reshape(-1)[:n]


def encode(m, v):
    """(m codes, m scales, v codes, v scales) of fp32 moments."""
    out = []
    n = m.size
    for x, floor, top, power in ((m, 2.0**-100, 127, 2), (v, 2.0**-90, 255, 4)):
        b = np.abs(_blocks(np.asarray(x, F)))
        scale = np.maximum(b.max(axis=1), F(floor))
        border = np.array([(j - 0.5)**power for j in range(1, top + 1)]).astype(F)
        to = (F(float(top**power)) / scale)[:, None]
        code = np.searchsorted(border, (b * to).reshape(-1), side="right")[:n]
        out += [code, scale]
    cm = np.where(np.asarray(m) < 0, -out[0], out[0]).astype(np.int8)
    cv = np.where(np.asarray(v) > 0, np.maximum(out[2], 1), out[2]).astype(np.uint8)
    return cm, out[1], cv, out[3]


def adamw(w, g, m, v, t, lr=1e-6, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, scale=1.0):
    """(w float64 before rounding, m, v fp32, the magnitude of the change's first term): arguments m and v are fp32 values.  Gradients
    that are not usable change nothing."""
    w = np.asarray(w, np.float64)
    m, v, g = (np.asarray(x, F) for x in (m, v, g))
    lr, beta1, beta2, eps, decay = (float(F(x)) for x in (lr, beta1, beta2, eps, decay))
    with np.errstate(over="ignore", invalid="ignore"):
        g = (g * F(scale)).astype(F)
        g2 = g * g
        bad = ~(g2 <= F(2.0**120))
        m1 = m * F(beta1) + g * F(1.0 - beta1)
        v1 = v * F(beta2) + g2 * F(1.0 - beta2)
    m1, v1 = np.where(bad, m, m1).astype(F), np.where(bad, v, v1).astype(F)
    u = (m1.astype(np.float64) / (1.0 - beta1**t)) / (np.sqrt(v1.astype(np.float64) / (1.0 - beta2**t)) + eps)
    first = np.where(bad, 0.0, lr * u)
    return np.where(bad, w, w - first - lr * decay * w), m1, v1, np.abs(first)
