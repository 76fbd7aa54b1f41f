"""Norms on both sides of every width at which another form takes over: one warp, 128 threads, 512, 1024, the largest rows whose weights and
inputs fit shared memory, and the longest that a block holds; few rows and more rows than blocks, with all that a row may carry.  Tolerances: those of
tests/test_gpu_layernorm.py."""

import pytest

from oracle import step as O
from tests.test_gpu_layernorm import case, check_bwd, check_fwd, grads, run_bwd, run_fwd

pytestmark = pytest.mark.gpu

BF16 = [249, 250, 256, 257, 4088, 4089, 4090, 4096, 4097, 4104, 8185, 8186, 8192, 8193, 8200, 14336, 16376, 16377, 16378, 16384, 16385]
FP32 = [125, 126, 128, 129, 2045, 2046, 2048, 2049, 2052, 4093, 4094, 4096, 4097, 4100, 8189, 8190, 8192, 8196, 14333, 14334, 14336, 14340, 16381, 16384, 16385]


@pytest.mark.parametrize("kind", [O.LAYER, O.RMS])
@pytest.mark.parametrize("d,x16", [(d, True) for d in BF16] + [(d, False) for d in FP32])
def test_both_sides_of_every_form(d, x16, kind):
    for T in (3, 170):
        some = 2 if T * d > 10**6 else 4                     # (the definitions in 64 bits take most of the time)
        for extra in (dict(residual=True, masked=True, pad=3), dict(), dict(residual=True, pad=8), dict(bias=False, masked=True))[:some]:
            c = case(d + T, T, d, kind, x16, **{"y16": x16, "w16": not x16, **extra})
            check_fwd(c, run_fwd(c))
        for dy16, dh, extra in ((False, True, dict(masked=True, pad=3)), (False, True, {}), (True, True, dict(pad=8)), (True, False, dict(masked=True)))[:some]:
            c = case(d + T, T, d, kind, x16, x16, not x16, bias=False, **extra)
            dy, dh = grads(d, c, dy16, dh)
            check_bwd(c, run_bwd(c, dy, dh), dy, dh)
