"""A quantised decoder layer's calls, what needs no GPU: sizes, and that bad arguments are refused before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from decoder_reference import Cache, quantize4, quantize8
from paper_2304_09049_amd import binding as dg

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
NULL, SHAPE, RANGE, BUFFER, UNSUPPORTED = 1, 2, 3, 4, 5


def test_sizes():
    assert dg.dg_linear_i8_work_bytes(3, 1000) == 3 * (1008 + 4)
    assert dg.dg_linear_i8_work_bytes(0, 8) == 0 and dg.dg_linear_i8_work_bytes(8, 1 << 17) == 0
    for bits in (8, 4):
        for dim in (64, 128, 256):
            assert dg.dg_cache_bytes(dg.cache_desc(7, 48, 3, dim, bits)) == Cache(7, 48, 3, dim, bits).bytes.size
    for bad in ((0, 16, 1, 64, 8), (1, 8, 1, 64, 8), (1, 16, 0, 64, 8), (1, 16, 1, 96, 8), (1, 16, 1, 64, 2), (1 << 27, 16, 1, 64, 8)):
        assert dg.dg_cache_bytes(dg.cache_desc(*bad)) == 0
    d = dg.cache_desc(64, 16, 2, 64, 8)
    assert dg.dg_paged_attention_work_bytes(d, 0, 4, 1, 100) == 0 and dg.dg_paged_attention_work_bytes(d, 1, 3, 1, 100) == 0
    assert dg.dg_paged_attention_work_bytes(d, 1, 4, 1, 10) == 0                     # too short to be cut


def test_quantize_tokens_refusals():
    f = dg.lib().dg_quantize_tokens
    call = lambda x=FAKE, t=0, N=2, K=8, s=8, c=FAKE, sc=8, o=FAKE: f(x, t, N, K, s, c, sc, o, None)  # noqa: E731
    assert call(x=None) == NULL and call(c=None) == NULL and call(o=None) == NULL
    assert call(N=-1) == SHAPE and call(K=0) == SHAPE and call(s=7) == SHAPE and call(sc=7) == SHAPE
    assert call(K=1 << 17, s=1 << 17, sc=1 << 17) == RANGE and call(t=3) == UNSUPPORTED
    assert call(N=0, x=None, c=None) == 0                                             # no tokens: nothing to do


def test_gemm_refusals():
    L = dg.lib()

    def call(w=FAKE, sw=8, a=FAKE, sa=8, M=4, N=2, K=8, sm=FAKE, sn=FAKE, o=FAKE, t=0, so=4):
        return L.dg_gemm_i8(w, sw, a, sa, M, N, K, sm, sn, None, o, t, so, None)

    assert [call(w=None), call(a=None), call(sm=None), call(sn=None), call(o=None)] == [NULL] * 5
    assert [call(M=0), call(N=-1), call(K=0), call(sw=7), call(sa=7), call(so=3)] == [SHAPE] * 6
    assert call(K=1 << 17, sw=1 << 17, sa=1 << 17) == RANGE and call(t=9) == UNSUPPORTED
    assert call(N=0, a=None, o=None) == 0

    def linear(x=FAKE, xt=1, sx=8, N=2, K=8, work=FAKE, bytes_=40, o=FAKE, t=1, w=FAKE):
        return L.dg_linear_i8(w, 8, x, xt, sx, 4, N, K, FAKE, None, work, bytes_, o, t, 4, None)

    assert [linear(x=None), linear(work=None), linear(o=None), linear(w=None)] == [NULL] * 4
    assert [linear(bytes_=39), linear(work=ctypes.c_void_p(0x1004))] == [BUFFER] * 2
    assert linear(sx=7) == SHAPE and linear(xt=4) == UNSUPPORTED and linear(N=0, work=None) == 0


def test_cache_refusals():
    L = dg.lib()
    good = dg.cache_desc(4, 16, 2, 64, 8)
    size = dg.dg_cache_bytes(good)

    def write(d=good, c=FAKE, n=size, k=FAKE, v=FAKE, t=0, T=3, slots=FAKE):
        return L.dg_cache_write(ctypes.byref(d) if d else None, c, n, k, v, t, T, 128, 64, 128, 64, slots, None)

    def read(d=good, c=FAKE, n=size, slots=FAKE, T=3, k=FAKE, v=FAKE, t=0):
        return L.dg_cache_read(ctypes.byref(d) if d else None, c, n, slots, T, k, v, t, None)

    assert [write(d=None), write(c=None), write(k=None), write(v=None), write(slots=None)] == [NULL] * 5
    assert [read(d=None), read(c=None), read(slots=None)] == [NULL] * 3
    for f in (write, read):
        assert [f(n=size - 1), f(c=ctypes.c_void_p(0x1008))] == [BUFFER] * 2
        assert [f(T=-1), f(d=dg.cache_desc(4, 24, 2, 64, 8)), f(d=dg.cache_desc(0, 16, 2, 64, 8))] == [SHAPE] * 3
        assert [f(t=5), f(d=dg.cache_desc(4, 16, 2, 80, 8)), f(d=dg.cache_desc(4, 16, 2, 64, 3))] == [UNSUPPORTED] * 3
        assert f(d=dg.cache_desc(1 << 27, 16, 2, 64, 8)) == RANGE and f(T=0, slots=None) == 0
    assert read(k=None, v=None) == 0


def test_attention_refusals():
    L = dg.lib()
    good = dg.cache_desc(64, 64, 2, 64, 8)
    size = dg.dg_cache_bytes(good)

    def call(d=good, c=FAKE, n=size, q=FAKE, t=1, T=2, Hq=4, start=FAKE, ctx=FAKE, table=FAKE, B=2, width=30, max_q=1, max_ctx=1000, o=FAKE,
             work=FAKE, bytes_=1 << 30):
        return L.dg_paged_attention(ctypes.byref(d) if d else None, c, n, q, t, T, Hq, 256, 64, start, ctx, table, B, width, max_q, max_ctx,
                                    0.125, 1, o, 256, 64, work, bytes_, None)

    assert [call(d=None), call(c=None), call(q=None), call(start=None), call(ctx=None), call(table=None), call(o=None)] == [NULL] * 7
    assert [call(Hq=3), call(B=-1), call(max_q=-1), call(T=-1), call(width=-1), call(max_ctx=-1)] == [SHAPE] * 6
    assert [call(t=0), call(t=7), call(d=dg.cache_desc(64, 64, 2, 32, 8))] == [UNSUPPORTED] * 3
    assert [call(B=1 << 30), call(max_q=1 << 30), call(B=1 << 20, max_q=1 << 12)] == [RANGE] * 3
    need = dg.dg_paged_attention_work_bytes(good, 2, 4, 1, 1000)
    assert need > 0 and call(n=size - 1) == BUFFER and call(bytes_=need - 1) == BUFFER and call(work=ctypes.c_void_p(0x1004)) == BUFFER
    assert call(work=None) == NULL
    assert call(B=0, table=None) == 0 and call(T=0, q=None) == 0 and call(max_q=0, q=None) == 0


def test_binding_checks():
    host = torch.zeros(4, 16, dtype=torch.int8)
    x, kv, slots = torch.zeros(4, 16), torch.zeros(2, 1, 64), torch.zeros(2, dtype=torch.int32)
    d, cache = dg.cache_desc(1, 16, 1, 64, 8), torch.zeros(16 * 136, dtype=torch.uint8)
    for call in (lambda: dg.dg_quantize_tokens(x), lambda: dg.dg_gemm_i8(host, host, x, x, out=x), lambda: dg.dg_linear_i8(host, x, x),
                 lambda: dg.dg_cache_write(d, cache, kv, kv, slots), lambda: dg.dg_cache_read(d, cache, slots, kv, kv),
                 lambda: dg.dg_paged_attention(d, cache, kv, slots, slots, slots[None], 1, 16)):
        with pytest.raises(ValueError, match="must live in device memory"):
            call()
    with pytest.raises(TypeError, match="must be a CacheDesc"):
        dg.dg_cache_write((1, 16, 1, 64, 8), cache, kv, kv, slots)
    with pytest.raises(TypeError, match="must be a tensor"):
        dg.dg_quantize_tokens([1.0], host, x)


def test_the_reference_against_hand_computed_codes():
    c, s = quantize8(np.array([[1.0, -2.0, 0.5, 127 / 64], [0, 0, 0, 0], [1, np.inf, 0, 0]], np.float32))
    assert s[0] == np.float32(2) / np.float32(127) and c[0].tolist() == [64, -127, 32, 126] and s[1] == 0 and c[1].tolist() == [0] * 4
    assert np.isnan(s[2]) and c[2].tolist() == [0] * 4
    c, s, z = quantize4(np.array([[-1.0, 0.5, 0.0, 0.25]], np.float32))
    assert z[0] == -1 and abs(s[0] - 0.1) < 1e-7 and c[0].tolist() == [0, 15, 10, 12]
