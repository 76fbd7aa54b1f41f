"""Float64 CPU definitions of the operators around the policy loss: log-probabilities from hidden states with their
gradients, and the orthogonalised (Muon) weight update.

Test infrastructure only, like the rest of this package: numpy, written from the formulas, sharing nothing with the
CUDA path.  Pinned in tests/test_operators_host.py by closed forms and finite differences.
"""

from __future__ import annotations

import numpy as np

NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def logprobs(h, w, y=None, mask=None, inv_t=1.0, top_k=0):
    """dict(z, logp, lse, entropy, top_ids, top_logp); z are the logits before the temperature.  A target outside the
    vocabulary has logp -inf; masked rows are zero (ids -1)."""
    z = np.asarray(h, np.float64) @ np.asarray(w, np.float64).T
    u = inv_t * z
    big = u.max(axis=1, keepdims=True)
    lse = (big + np.log(np.exp(u - big).sum(axis=1, keepdims=True)))[:, 0]
    logq = u - lse[:, None]
    t, v = z.shape
    out = dict(z=z, lse=lse, entropy=-(np.exp(logq) * logq).sum(axis=1))
    if y is not None:
        y = np.asarray(y)
        ok = (y >= 0) & (y < v)
        out["logp"] = np.where(ok, logq[np.arange(t), np.where(ok, y, 0)], -np.inf)
    order = np.lexsort((np.broadcast_to(np.arange(v), z.shape), -z), axis=1)[:, :top_k]
    out["top_ids"], out["top_logp"] = order.astype(np.int32), np.take_along_axis(logq, order, axis=1)
    if mask is not None:
        off = np.asarray(mask) == 0
        for k in ("logp", "lse", "entropy", "top_logp"):
            if k in out:
                out[k][off] = 0.0
        out["top_ids"][off] = -1
    return out


def logprobs_backward(h, w, y, mask, lse, entropy, g_logp, g_lse, g_entropy, inv_t=1.0):
    """(dH, dW, |dz| summed termwise): gradients of sum g_logp logp + g_lse lse + g_entropy entropy."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    t, v = h.shape[0], w.shape[0]
    zero = np.zeros(t)
    gl, gs, ge = (zero if g is None else np.asarray(g, np.float64) for g in (g_logp, g_lse, g_entropy))
    ent = zero if entropy is None else np.asarray(entropy, np.float64)
    y = np.full(t, -1) if y is None else np.asarray(y)
    ok = (y >= 0) & (y < v)
    gl = np.where(ok, gl, 0.0)
    on = np.ones(t, bool) if mask is None else np.asarray(mask) != 0
    h = np.where(on[:, None], h, 0.0)
    logq = inv_t * (h @ w.T) - np.asarray(lse, np.float64)[:, None]
    p = np.where(on[:, None], np.exp(np.where(on[:, None], logq, 0.0)), 0.0)
    size = p * (np.abs(gs - gl)[:, None] + np.abs(ge)[:, None] * (np.abs(logq) + np.abs(ent)[:, None]))
    dz = p * ((gs - gl)[:, None] - ge[:, None] * (logq + ent[:, None]))
    rows = np.nonzero(ok & on)[0]
    dz[rows, y[rows]] += gl[rows]
    size[rows, y[rows]] += np.abs(gl[rows])
    dz, size = inv_t * dz, inv_t * size
    return dz @ w, dz.T @ h, size


def newton_schulz(g, steps=5, coefficients=NS_COEFFICIENTS, eps=1e-7):
    """Newton-Schulz iteration X <- a X + b (X X^T) X + c (X X^T)^2 X from X = G / (|G|_F + eps)."""
    a, b, c = coefficients
    x = np.asarray(g, np.float64)
    x = x / (np.linalg.norm(x) + eps)
    for _ in range(steps):
        q = x @ x.T
        x = a * x + (b * q + c * (q @ q)) @ x
    return x


def muon_scale(m, n, mode):
    """0: 1;  1: sqrt(max(1, m / n));  2: 0.2 sqrt(max(m, n))."""
    return (1.0, np.sqrt(max(1.0, m / n)), 0.2 * np.sqrt(max(m, n)))[mode]


def muon_update(w, momentum, g, lr, mu, weight_decay=0.0, nesterov=True, mode=0, steps=5,
                coefficients=NS_COEFFICIENTS, eps=1e-7):
    """(new W, new momentum, orthogonalised update)."""
    w, g = np.asarray(w, np.float64), np.asarray(g, np.float64)
    m = mu * np.asarray(momentum, np.float64) + g
    o = newton_schulz(g + mu * m if nesterov else m, steps, coefficients, eps)
    return (1.0 - lr * weight_decay) * w - lr * muon_scale(*w.shape, mode) * o, m, o


def newton_schulz_rounded(g, steps=5, coefficients=NS_COEFFICIENTS, eps=1e-7):
    """The same iteration with fp16 roundings where the library documents them (the iterate where it is an operand, scaled by a
    power of two, but not in the term a X; the Gram matrix and the polynomial once each, the latter's diagonal not at all), everything
    else in 64 bits: what those roundings alone do to a given input, which is what a tolerance has to allow for."""
    a, b, c = coefficients
    x = np.asarray(g, np.float64)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    half = lambda z: z.astype(np.float16).astype(np.float64)  # noqa: E731
    s = 2.0 ** np.round(np.log2(np.sqrt(max(x.shape))))
    x = x / (np.linalg.norm(x) + eps) * s
    for _ in range(steps):
        hi = half(x)
        q = half(hi @ hi.T / s**2)
        poly = b * q + c * (q @ q)
        diagonal = np.diag(poly)
        x = (a + diagonal)[:, None] * x + half(poly - np.diag(diagonal)) @ hi
    return (x.T if tall else x) / s
