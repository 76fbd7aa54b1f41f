"""Vocabulary rows whose logits are -inf or the type's lowest value (banned tokens, padding of the vocabulary): they have
probability zero, those of -inf are never listed, and everything else is what it is without them, on every path.  Tolerances:
test_gpu_logprobs's, on the rows that are left."""

import numpy as np
import pytest

from oracle import operators as O
from tests.test_gpu_logprobs import call_bwd, call_fwd, check_bwd, make, tolerances, upstream

pytestmark = pytest.mark.gpu

# T, d, V, bf16, alternatives: streamed rows, narrow and wide tiles with every list length, fp32 in one and in several segments
FORMS = [(1, 64, 3000, True, 20), (4, 64, 3000, True, 8), (50, 128, 20000, True, 0), (200, 64, 3000, True, 20),
         (200, 64, 3000, True, 8), (200, 128, 3000, True, 0), (200, 1088, 3000, True, 8), (300, 1088, 3000, True, 0),
         (40, 64, 3000, False, 20), (700, 64, 900, False, 5)]


def banned_columns(V):
    ban = np.zeros(V, bool)
    ban[0:40] = True                       # the first columns of all: more than the 32 that are reduced at a time
    ban[V // 4:V // 4 + 700] = True        # whole tiles and whole splits
    ban[V // 2::7] = True
    ban[-90:] = True                       # the ragged end
    return ban


def inputs_with(ban, T, d, V, bf16, value, feature):
    """The first feature of every row is `feature`, and its weight is `value` for banned columns, zero for the others."""
    h, w, _, rng = make(T + d + V, T, d, V, bf16=bf16, grid=True)
    h[:, 0] = feature
    w[:, 0] = 0.0
    w[ban] = 0.0
    w[ban, 0] = value
    y = rng.choice(np.nonzero(~ban)[0], T).astype(np.int32)
    return h, w, y, rng


def lowest(bf16):
    return -float(np.float32(2.0**127 * (2 - (2.0**-7 if bf16 else 2.0**-23))))


@pytest.mark.parametrize("entropy", [True, False])
@pytest.mark.parametrize("T,d,V,bf16,K", FORMS)
@pytest.mark.parametrize("infinite", [True, False])
def test_forward(T, d, V, bf16, K, infinite, entropy):
    ban = banned_columns(V)
    h, w, y, _ = inputs_with(ban, T, d, V, bf16, -np.inf if infinite else lowest(bf16), 1.0)
    keep = np.nonzero(~ban)[0]
    place = np.cumsum(~ban) - 1
    want = O.logprobs(h, w[keep], place[y], None, 1.0, K)
    y[0] = 3                               # a banned target
    got = call_fwd(h, w, y, None, K, 1.0, bf16=bf16, entropy=entropy)
    assert got["status"] == 0 and got["logp"][0] <= -3e38 and np.isneginf(got["logp"][0]) == infinite
    _, tol, tol_ent = tolerances(h, w[keep], 1.0, want)
    np.testing.assert_allclose(got["lse"], want["lse"], rtol=0, atol=tol)
    np.testing.assert_allclose(got["logp"][1:], want["logp"][1:], rtol=0, atol=tol)
    if entropy:
        np.testing.assert_allclose(got["entropy"], want["entropy"], rtol=0, atol=tol_ent)
    if K:
        np.testing.assert_array_equal(got["top_ids"], keep[want["top_ids"]])
        np.testing.assert_allclose(got["top_logp"], want["top_logp"], rtol=0, atol=tol)


@pytest.mark.parametrize("T,d,V,bf16", [(3, 64, 2000, True), (3, 64, 50000, True), (200, 64, 2000, True), (200, 1088, 2010, True),
                                        (30, 64, 2010, False), (1, 64, 50001, False)])
@pytest.mark.parametrize("infinite", [True, False])
def test_fewer_left_than_alternatives(T, d, V, bf16, infinite):
    K = 20
    ban = np.ones(V, bool)
    ban[[77, 600, 1500, 1999]] = False
    h, w, y, _ = inputs_with(ban, T, d, V, bf16, -np.inf if infinite else lowest(bf16), 1.0)
    keep = np.nonzero(~ban)[0]
    want = O.logprobs(h, w[keep], None, None, 1.0, 4)
    got = call_fwd(h, w, y, None, K, 1.0, bf16=bf16)
    _, tol, tol_ent = tolerances(h, w[keep], 1.0, want)
    assert got["status"] == 0
    np.testing.assert_allclose(got["lse"], want["lse"], rtol=0, atol=tol)
    np.testing.assert_allclose(got["entropy"], want["entropy"], rtol=0, atol=tol_ent)
    np.testing.assert_array_equal(got["top_ids"][:, :4], keep[want["top_ids"]])
    if infinite:
        assert np.all(got["top_ids"][:, 4:] == -1) and np.all(np.isneginf(got["top_logp"][:, 4:]))
    else:                                  # equal logits, by ascending id
        assert np.all(got["top_ids"][:, 4:] == np.nonzero(ban)[0][None, :16]) and np.all(got["top_logp"][:, 4:] <= -3e38)


@pytest.mark.parametrize("T,d,bf16", [(3, 64, True), (200, 64, True), (200, 1088, True), (30, 64, False)])
def test_nothing_left_at_all(T, d, bf16):
    from paper_2509_13232_b200 import binding as B
    V = 700
    h, w, y, _ = inputs_with(np.arange(V) < V - 1, T, d, V, bf16, -np.inf, 1.0)
    w[V - 1] = w[0]
    got = call_fwd(h, w, y, None, 5, 1.0, bf16=bf16)
    assert got["status"] == B.DEV_NONFINITE
    assert np.all(np.isneginf(got["lse"])) and np.all(got["top_ids"] == -1)


@pytest.mark.parametrize("which", [(1, 1, 1), (1, 0, 0)])
@pytest.mark.parametrize("T,d,V,bf16", [(4, 64, 3000, True), (300, 64, 3000, True), (200, 1088, 3000, True), (40, 64, 3000, False)])
def test_backward(T, d, V, bf16, which):
    """Finite weights whose logits overflow to -inf: no gradient from them, and none to them."""
    ban = banned_columns(V)
    h, w, y, rng = inputs_with(ban, T, d, V, bf16, float(np.float32(-(2.0**127))), 4.0)
    keep = np.nonzero(~ban)[0]
    place = np.cumsum(~ban) - 1
    fwd = O.logprobs(h, w[keep], place[y], None, 1.0)
    gl, gs, ge = upstream(rng, T, which)
    want = O.logprobs_backward(h, w[keep], place[y], None, fwd["lse"], fwd["entropy"], gl, gs, ge)
    dh, dw, st = call_bwd(h, w, y, None, fwd["lse"], fwd["entropy"], gl, gs, ge, 1.0, bf16=bf16)
    assert st == 0 and np.all(dw[ban] == 0)
    check_bwd(dh, dw[keep], want, h, w[keep], None, 1.0, fwd, bf16, False, False)


@pytest.mark.parametrize("T,d,V,bf16", [(3, 64, 50000, True), (200, 64, 2010, True), (200, 1088, 2010, True), (30, 64, 2010, False),
                                        (1, 64, 50001, False)])
def test_order_among_banned_columns(T, d, V, bf16):
    """Logits of about the lowest value everywhere but in four columns, the highest of them one to a group of columns."""
    K = 20
    ban = np.ones(V, bool)
    ban[[77, 600, 1500, 1999]] = False
    h, w, _, _ = inputs_with(ban, T, d, V, bf16, lowest(bf16), 1.0)
    first = 5 + 97 * np.arange(19)                      # none of the four, never two in a group of 64
    assert np.all(ban[first])
    w[first, 0] = -(2.0**126) * (1 + np.arange(19) / 32.0).astype(np.float32)
    got = call_fwd(h, w, None, None, K, 1.0, bf16=bf16)
    want = O.logprobs(h, w, None, None, 1.0, K)["top_ids"]
    assert got["status"] == 0 and np.all(np.sort(want[:, 4:], axis=1) == np.sort(first[:16]))
    np.testing.assert_array_equal(got["top_ids"], want)
