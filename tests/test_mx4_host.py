"""Layers in microscaled 4-bit floating point and layers of experts, what needs no GPU: sizes, refusals before anything is launched, the plain reference itself."""
import ctypes

import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1008)
NULL, SHAPE, RANGE, BUFFER, UNSUPPORTED = 1, 2, 3, 4, 5


def test_sizes():
    assert dg.dg_linear_mx4_work_bytes(3, 1000) == 3 * (32 * 16 + 32) and dg.dg_linear_mx4_work_bytes(2, 33) == 2 * (32 + 4)
    assert dg.dg_linear_mx4_work_bytes(0, 8) == 0 and dg.dg_linear_mx4_work_bytes(8, (1 << 24) + 1) == 0
    assert dg.dg_route_tokens_work_bytes(0, 8) == 0 and dg.dg_route_tokens_work_bytes(4, 1025) == 0 and dg.dg_route_tokens_work_bytes(4, 8) >= 4 * 8 * 4
    assert dg.dg_experts_mx4_work_bytes(0, 1, 8, 8) == 0 and dg.dg_experts_mx4_work_bytes(1, 65, 8, 8) == 0 and dg.dg_experts_mx4_work_bytes(1, 1, 8, 8) > 0
    assert dg.dg_experts_mx4_work_bytes(1 << 20, 8, 4096, 1024) == dg.dg_experts_mx4_work_bytes(4096, 8, 4096, 1024)       # (worked through in turns)


def test_quantize_refusals():
    def q(x=FAKE, t=0, N=2, K=40, s=40, c=FAKE, sc=32, o=FAKE, so=4):
        return dg.lib().dg_quantize_mx4(x, t, N, K, s, c, sc, o, so, None)

    def d(x=FAKE, t=0, N=2, K=40, s=40, c=FAKE, sc=32, o=FAKE, so=4):
        return dg.lib().dg_dequantize_mx4(c, sc, o, so, N, K, x, t, s, None)

    for f in (q, d):
        assert [f(x=None), f(c=None), f(o=None)] == [NULL] * 3
        assert [f(N=-1), f(K=0), f(s=39), f(sc=31), f(so=1)] == [SHAPE] * 5
        assert f(K=(1 << 24) + 1, s=1 << 25) == RANGE and f(t=3) == UNSUPPORTED
        assert [f(c=ODD), f(sc=40), f(o=ctypes.c_void_p(0x1002)), f(so=6)] == [BUFFER] * 4
        assert f(N=0, x=None, c=None, o=None) == 0


def test_product_refusals():
    L = dg.lib()

    def gemm(w=FAKE, sw=32, ws=FAKE, sws=4, a=FAKE, sa=32, as_=FAKE, sas=4, M=4, N=2, K=40, o=FAKE, t=0, so=4):
        return L.dg_gemm_mx4(w, sw, ws, sws, a, sa, as_, sas, M, N, K, None, o, t, so, None)

    def linear(w=FAKE, sw=32, ws=FAKE, sws=4, x=FAKE, xt=1, sx=40, M=4, N=2, K=40, o=FAKE, t=1, so=4, work=FAKE, size=72):
        return L.dg_linear_mx4(w, sw, ws, sws, x, xt, sx, M, N, K, None, work, size, o, t, so, None)

    for f in (gemm, linear):
        assert [f(w=None), f(ws=None), f(o=None)] == [NULL] * 3
        assert [f(M=0), f(N=-1), f(K=0), f(sw=16), f(sws=0), f(so=3)] == [SHAPE] * 6
        assert f(K=(1 << 24) + 1) == RANGE and f(M=1 << 30, N=1 << 30, so=1 << 30) == RANGE and f(sw=(1 << 26) + 16) == RANGE and f(t=9) == UNSUPPORTED
        assert [f(w=ODD), f(sw=40), f(sws=5), f(ws=ctypes.c_void_p(0x1001))] == [BUFFER] * 4
        assert f(N=0, o=None) == 0
    assert [gemm(a=None), gemm(as_=None)] == [NULL] * 2 and gemm(sa=16) == SHAPE and gemm(a=ODD) == BUFFER and gemm(sas=6) == BUFFER
    assert [linear(x=None), linear(work=None)] == [NULL] * 2 and [linear(size=71), linear(work=ODD)] == [BUFFER] * 2
    assert linear(sx=39) == SHAPE and linear(xt=4) == UNSUPPORTED


def test_route_refusals():
    def f(x=FAKE, xt=1, T=2, K=8, sx=8, R=FAKE, rt=1, E=6, sr=8, top=2, mode=0, ids=FAKE, w=FAKE, work=FAKE, size=1 << 20):
        return dg.lib().dg_route_tokens(x, xt, T, K, sx, R, rt, E, sr, None, top, mode, 1.0, ids, w, work, size, None)

    assert [f(x=None), f(R=None), f(ids=None), f(w=None), f(work=None)] == [NULL] * 5
    assert [f(T=-1), f(K=0), f(E=0), f(top=0), f(top=7), f(sx=7), f(sr=7)] == [SHAPE] * 7
    assert [f(E=1025), f(E=100, top=65), f(T=1 << 30), f(K=1 << 31, sx=1 << 31, sr=1 << 31)] == [RANGE] * 4
    assert [f(xt=3), f(rt=2), f(xt=0, rt=1), f(mode=3), f(mode=-1)] == [UNSUPPORTED] * 5
    assert [f(size=dg.dg_route_tokens_work_bytes(2, 6) - 1), f(work=ODD)] == [BUFFER] * 2
    assert f(T=0, x=None, ids=None, work=None) == 0


def experts_desc(**change):
    base = dict(experts=3, hidden=40, inner=70, reserved=0, up=0x1000, up_scales=0x1000, down=0x1000, down_scales=0x1000, up_row=32, up_expert=32 * 140,
                up_scales_row=4, up_scales_expert=4 * 140, down_row=48, down_expert=48 * 40, down_scales_row=4, down_scales_expert=160)
    base.update(change)
    return dg.ExpertsDesc(**base)


def test_experts_refusals():
    def f(x=FAKE, t=1, T=2, sx=40, ids=FAKE, w=FAKE, top=2, work=FAKE, size=1 << 20, o=FAKE, so=40, desc=None, **change):
        d = experts_desc(**change)
        return dg.lib().dg_experts_mx4(ctypes.byref(d) if desc is None else None, x, t, T, sx, ids, w, top, work, size, o, so, None)

    assert [f(desc=0), f(x=None), f(ids=None), f(w=None), f(work=None), f(o=None), f(up=0), f(up_scales=0), f(down=0), f(down_scales=0)] == [NULL] * 10
    assert [f(experts=0), f(hidden=0), f(inner=-1), f(T=-1), f(top=0), f(sx=39), f(so=39), f(up_row=16), f(down_row=32), f(up_scales_row=0), f(up_expert=-16)] == [SHAPE] * 11
    assert [f(experts=(1 << 16) + 1), f(top=65), f(T=1 << 26), f(hidden=(1 << 20) + 1), f(inner=(1 << 20) + 1)] == [RANGE] * 5
    assert [f(t=0), f(t=5), f(reserved=1)] == [UNSUPPORTED] * 3
    assert [f(up=0x1008), f(up_row=40), f(up_expert=40), f(down_scales=0x1002), f(down_scales_row=6), f(down_scales_expert=42), f(work=ODD),
            f(size=dg.dg_experts_mx4_work_bytes(2, 2, 40, 70) - 1)] == [BUFFER] * 8
    assert f(T=0, x=None, ids=None, w=None, work=None, o=None) == 0


def test_binding_checks():
    x, codes, scales, up = torch.zeros(4, 32), torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8), torch.zeros(1, 4, 16, dtype=torch.uint8)
    ids = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: dg.dg_quantize_mx4(x, codes, scales), lambda: dg.dg_dequantize_mx4(codes, scales, out=x), lambda: dg.dg_gemm_mx4(codes, scales, codes, scales, out=x),
                 lambda: dg.dg_linear_mx4(codes, scales, x), lambda: dg.dg_route_tokens(x, x, 2),
                 lambda: dg.dg_experts_mx4(up, up[..., 0], up, up[..., 0], x, ids, x[:, :2])):
        with pytest.raises(ValueError, match="must live in device memory"):
            call()
    with pytest.raises(TypeError, match="must be a tensor"):
        dg.dg_gemm_mx4([1], scales, codes, scales, out=x)
    with pytest.raises(KeyError):
        dg.dg_route_tokens(x, x, 2, mode="hard", work=codes)
    with pytest.raises(ValueError, match="31 columns"):
        dg.dg_dequantize_mx4(codes, scales, K=31, out=x)


def test_the_reference_against_hand_computed_codes():
    assert [ref.nearest_code(a) for a in (0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 9.0)] == [0, 1, 2, 2, 4, 4, 6, 6, 7, 7]
    x = torch.zeros(1, 40)
    x[0, :5] = torch.tensor([6.0, -0.25, 0.75, -5.0, 2.5])          # scale 1
    x[0, 32], x[0, 39] = 0.11, -0.0                                  # 0.11 = 1.76 / 16: scale 1/64, 7.04 -> 6
    codes, scales = ref.quantize(x)
    assert codes[0, 0, :6].tolist() == [7, 8, 2, 14, 4, 0] and codes[0, 1, 0] == 7 and codes[0, 1, 7] == 8 and scales.tolist() == [[127, 121]]
    assert ref.values(ref.pack(codes), scales, 40)[0, [0, 3, 32]].tolist() == [6.0, -4.0, 6 / 64]
    x[0, 3] = float("inf")
    codes, scales = ref.quantize(x)
    assert scales.tolist() == [[255, 121]] and not codes[0, 0].any() and torch.isnan(ref.values(ref.pack(codes), scales, 40)[0, :32]).all()
    grid = torch.arange(0, 1024).double() / 128
    codes, _ = ref.quantize(torch.cat((torch.full((1024, 1), 4.0), grid[:, None].float()), 1)[grid < 8])
    assert codes[:, 0, 1].tolist() == [ref.nearest_code(a) for a in grid.tolist()]


def test_the_reference_chooses_by_the_rules():
    R = torch.tensor([[1.0], [2.0], [2.0], [-1.0]])
    ids, w = ref.route(torch.tensor([[1.0], [-1.0], [float("nan")]]), R, 2, "softmax", None, 1.0)
    assert ids.tolist() == [[1, 2], [3, 0], [0, 1]] and w[0].tolist() == [0.5, 0.5] and torch.isnan(w[2]).all()
    ids, w = ref.route(torch.ones(1, 1), R, 3, "sigmoid", torch.tensor([float("-inf"), float("-inf"), 0.0, float("-inf")]), 2.0)
    assert ids.tolist() == [[2, -1, -1]] and w.tolist() == [[2.0, 0, 0]]
