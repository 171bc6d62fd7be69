"""Where the calls in microscaled 4-bit floating point end, as the header says it; nothing is launched."""
import ctypes

import pytest

from paper_2304_09049_amd import binding as dg

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
SHAPE, RANGE = 2, 3
TOO_MANY = 1 << 31


def rows(call, N=2, K=40, sx=40, sc=32, ss=4):
    L = dg.lib()
    return L.dg_quantize_mx4(FAKE, 1, N, K, sx, FAKE, sc, FAKE, ss, None) if call == "quantize" else L.dg_dequantize_mx4(FAKE, sc, FAKE, ss, N, K, FAKE, 1, sx, None)


def product(call, M=4, N=2, K=40, so=4, sw=32, sws=4):
    L = dg.lib()
    if call == "gemm":
        return L.dg_gemm_mx4(FAKE, sw, FAKE, sws, FAKE, 32, FAKE, 4, M, N, K, None, FAKE, 1, so, None)
    return L.dg_linear_mx4(FAKE, sw, FAKE, sws, FAKE, 1, 40, M, N, K, None, FAKE, 1 << 40, FAKE, 1, so, None)


@pytest.mark.parametrize("call", ["quantize", "dequantize"])
def test_rows(call):
    assert rows(call, N=TOO_MANY) == SHAPE and rows(call, N=-1) == SHAPE and rows(call, K=0) == SHAPE
    assert rows(call, K=(1 << 24) + 1, sx=1 << 25) == RANGE and rows(call, sc=(1 << 26) + 16) == RANGE and rows(call, ss=(1 << 26) + 4) == RANGE


@pytest.mark.parametrize("call", ["gemm", "linear"])
def test_products(call):
    assert product(call, N=TOO_MANY) == SHAPE and product(call, M=TOO_MANY, so=TOO_MANY) == SHAPE
    assert product(call, K=(1 << 24) + 1) == RANGE and product(call, sw=(1 << 26) + 16) == RANGE and product(call, sws=(1 << 26) + 4) == RANGE
    assert product(call, M=1 << 24, N=1 << 20, so=1 << 24) == RANGE
