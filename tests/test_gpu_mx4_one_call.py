"""A linear layer in microscaled 4-bit floating point as one call and as two: the same bits."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def spread(gen, N, K):
    """Blocks of many sizes: of blocks of one size the sums are exact, and their order does not show."""
    sizes = torch.randint(-8, 4, (N, -(-K // 32)), generator=gen, device=DEV).float().exp2()
    return torch.randn(N, K, generator=gen, device=DEV) * sizes.repeat_interleave(32, 1)[:, :K]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(150, 4096), (4096, 2049), (4100, 3000), (5120, 1056), (6143, 2048), (6144, 2048), (8000, 1400), (8192, 4096), (16400, 1090), (32000, 1024), (70000, 544)])
def test_one_token(M, K, dtype):
    """Wherever the token begins: on a word it is quantised within the product."""
    gen = torch.Generator(device=DEV).manual_seed(M + K)
    W, Ws = dg.dg_quantize_mx4(spread(gen, M, K))
    bias = torch.randn(M, generator=gen, device=DEV)
    wide = torch.zeros(1, K + 4, device=DEV, dtype=ref.TYPES[dtype])
    x = spread(gen, 1, K).to(ref.TYPES[dtype])
    codes, scales = dg.dg_quantize_mx4(x)
    for b in (None, bias):
        want = dg.dg_gemm_mx4(W, Ws, codes, scales, bias=b, dtype=x.dtype)
        for at in range(4):
            wide[:, at:at + K] = x
            assert torch.equal(dg.dg_linear_mx4(W, Ws, wide[:, at:at + K], bias=b), want)


@pytest.mark.parametrize("N,M,K", [(2, 4100, 3000), (9, 6000, 1024), (40, 333, 2085), (200, 700, 4097), (1000, 520, 2600)])
def test_more_tokens(N, M, K):
    gen = torch.Generator(device=DEV).manual_seed(N + M + K)
    W, Ws = dg.dg_quantize_mx4(spread(gen, M, K))
    x = spread(gen, N, K + 1).bfloat16()[:, 1:]
    assert torch.equal(dg.dg_linear_mx4(W, Ws, x), dg.dg_gemm_mx4(W, Ws, *dg.dg_quantize_mx4(x), dtype=x.dtype))
