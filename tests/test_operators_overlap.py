"""spo_logprobs_bwd refuses gradients that share memory with what they are computed from: H and W are read again after the first
rows of the results have been written.  Addresses are looked at on the host and never dereferenced."""

import ctypes

import pytest

from paper_2509_13232_b200 import binding as B
from paper_2509_13232_b200 import build as spo_build

T, D, V = 8, 64, 100
H, W, DH, DW = 0x10000, 0x20000, 0x40000, 0x60000          # 8 x 64 and 100 x 64 elements of 2 bytes: 0x400 and 0x3200 bytes


@pytest.fixture(scope="module")
def lib():
    spo_build.build()
    return B.lib()


def call(lib, h=H, w=W, dh=DH, dw=DW, dht=1, dwt=1, ld=D, rows=T):
    p = ctypes.c_void_p
    return lib.spo_logprobs_bwd(p(h), ld, p(w), 1, p(0x1000), None, p(0x2000), None, p(0x3000), None, None, rows, D, V, 1.0, p(dh), dht,
                                p(dw), dwt, 0, p(1 << 40), 0, None, None)         # (no scratch: nothing is ever launched)


@pytest.mark.parametrize("bad", [
    dict(dh=H), dict(dh=H + 0x3F0), dict(dh=H - 0x3F0), dict(dh=W), dict(dh=W + 0x31F0), dict(dw=W), dict(dw=W - 0x31F0), dict(dw=H),
    dict(dh=DW), dict(dw=DH + 0x3F0), dict(dh=H - 0x7F0, dht=0), dict(dw=W - 0x63F0, dwt=0), dict(dh=H + 0xB00, ld=256),
    dict(dh=H + (1 << 50), ld=1 << 62)])
def test_shared_memory_is_refused(lib, bad):
    assert call(lib, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("good", [
    dict(), dict(dh=H + 0x400), dict(dh=H - 0x400), dict(dw=W + 0x3200), dict(dw=W - 0x3200), dict(dh=DW - 0x400), dict(dh=H - 0x800, dht=0),
    dict(dw=W - 0x6400, dwt=0), dict(dw=DH + 0x400)])
def test_neighbours_are_not(lib, good):
    assert call(lib, **good) in (B.ERR_UNSUPPORTED_ARCH, B.ERR_WORKSPACE_TOO_SMALL)
