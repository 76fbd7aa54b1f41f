"""Scratch of the log-probability calls: a size that the library names for T rows serves every shorter batch, so that a loop can
allocate once for its longest."""

import numpy as np
import pytest

from paper_2509_13232_b200 import binding as B
from paper_2509_13232_b200 import build as spo_build

SHAPES = [(4096, 151936), (1024, 32000), (64, 300), (2048, 20011), (1088, 1)]


def lengths():
    rng = np.random.default_rng(0)
    edges = [k * 256 + e for k in range(1, 80) for e in (-1, 1)] + [512, 9472, 18944]
    return sorted(set(range(0, 300)) | set(edges) | {int(t) for t in np.exp(rng.uniform(0, np.log(2e5), 300))})


@pytest.fixture(scope="module", autouse=True)
def library():
    spo_build.build()


@pytest.mark.parametrize("d,V", SHAPES)
@pytest.mark.parametrize("K", [0, 1, 8, 9, 20])
def test_forward_sizes_grow_with_the_rows(d, V, K):
    if K > V:
        return
    sizes = [B.spo_workspace_bytes(B.WS_LOGPROBS, T=t, d=d, V=V, B=K) for t in lengths()]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[-1] < 2 << 30


@pytest.mark.parametrize("d,V", SHAPES)
def test_backward_sizes_grow_with_the_rows(d, V):
    sizes = [B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=t, d=d, V=V) for t in lengths()]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_lists_take_no_more_than_the_logits_and_their_places():
    """15 row tiles over 125 tiles of columns: lists of up to 20 groups where a split's half has 8."""
    T, V = 3840, 32000
    size = B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=1024, V=V, B=20)
    assert size < 1.2 * T * V * 4
