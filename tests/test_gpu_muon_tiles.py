"""Newton-Schulz on each pair of tile widths that its rule chooses (symmetric products, update), in both orientations, against the
definition in 64 bits; the tolerance is test_gpu_muon's.  A matrix that stands in the batch twice gives the same bits on other tiles."""

import numpy as np
import pytest

from tests.test_gpu_muon import gradient, iterate64, orthogonalize

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,m,n", [
    (1, 500, 900), (1, 900, 500), (3, 4000, 300), (90, 100, 128), (75, 300, 100),      # 128, 128
    (1, 1000, 2730), (1, 2730, 1000), (200, 100, 1000),                                # 128, 256
    (20, 300, 300), (20, 310, 290),                                                    # 256, 128
    (2, 1500, 1500), (16, 1030, 1024), (76, 520, 130),                                 # 256, 256
    (1, 4000, 4100), (1, 4100, 4000),                                                  # 512, 256
])
def test_every_pair_of_tile_widths(b, m, n):
    import torch
    rng = np.random.default_rng(b + m)
    k = min(b, 3)
    g = np.concatenate([gradient(rng, k, m, n, 40) + 3e-4 * rng.standard_normal((k, m, n)).astype(np.float32)] * -(-b // k))[:b]
    got, st = orthogonalize(g)
    assert st == 0
    want, rounded = iterate64(g[:k], False), iterate64(g[:k], True)
    norm = torch.linalg.vector_norm(want, dim=(1, 2))
    allowed = 2 * torch.linalg.vector_norm(rounded - want, dim=(1, 2)) + 2.0**-19 * norm
    assert bool((torch.linalg.vector_norm(torch.from_numpy(got[:k]).cuda().double() - want, dim=(1, 2)) <= allowed).all())
    for i in range(k, b):
        assert np.array_equal(got[i], got[i % k])
