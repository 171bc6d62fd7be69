"""Every tile of the 4-bit product in every type of result, with and without a bias, into rows that begin anywhere."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def operand(gen, N, K):
    """Quantised blocks of many sizes on the device, and their values there in 64 bits."""
    sizes = torch.randint(-6, 3, (N, -(-K // 32)), generator=gen, device=DEV).float().exp2()
    x = torch.randn(N, K, generator=gen, device=DEV) * sizes.repeat_interleave(32, 1)[:, :K]
    codes, scales = dg.dg_quantize_mx4(x)
    return codes, scales, dg.dg_dequantize_mx4(codes, scales, K).double()     # (values of 4 bits and a power of two are exact in binary32)


@pytest.fixture(scope="module")
def operands():
    made = {}

    def of(N, M, K):
        if (N, M, K) not in made:
            made.clear()
            gen = torch.Generator(device=DEV).manual_seed(N + M + K)
            A, W, bias = operand(gen, N, K), operand(gen, M, K), 20 * torch.randn(M, generator=gen, device=DEV)
            # (the bound's sums in binary32, some 2^-20 of themselves off: far less than what it leaves)
            made[N, M, K] = A, W, bias, A[2] @ W[2].t(), (A[2].abs().float() @ W[2].abs().float().t()).double() * 1.001
        return made[N, M, K]
    return of


FEW, MANY = ("16x16", "16x32", "32x16", "32x32"), ("32x64", "64x64", "128x64", "128x128", "256x128", "256x256")


# the last two: more tiles of 256 x 256 than compute units, of two stages and of five
@pytest.mark.parametrize("tile,N,M,K", [(tile, *size) for size in ((5, 7, 40), (130, 262, 1250), (300, 515, 2080), (2100, 8300, 512), (2100, 8300, 1250))
                                        for tile in (FEW + MANY if size[0] < 1000 else MANY)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_tile(tile, dtype, bias, N, M, K, operands, monkeypatch):
    (A, As, _), (W, Ws, _), b, want, size = operands(N, M, K)
    if bias:
        want, size = want + b.double(), size + b.abs()
    off = size * ((K / 64 + 32) * 2.0 ** -24 + 64 * 2.0 ** -28)               # (as in mx4_reference.product)
    off = off + ref.rounding(want.abs() + off, ref.TYPES[dtype])
    monkeypatch.setenv("DG_GEMM_MX4_TILE", tile)
    room = torch.full((N + 1, M + 9), 5.0, dtype=ref.TYPES[dtype], device=DEV)
    out = dg.dg_gemm_mx4(W, Ws, A, As, bias=b if bias else None, out=room[:N, 3:M + 3])
    assert ((out.double() - want).abs() <= off).all()
    assert (room[:, :3] == 5).all() and (room[:, M + 3:] == 5).all() and (room[N] == 5).all()
    whole = dg.dg_gemm_mx4(W, Ws, A, As, bias=b if bias else None, dtype=ref.TYPES[dtype])
    assert torch.equal(whole, out)
