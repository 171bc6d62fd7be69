"""Experts whose weights are at the ends of what a block's scale holds."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E, K, F = 5, 64, 96


def codes_up_to(gen, most, *size):
    """Two codes a byte, of the levels 0 ... most and their negatives."""
    c = torch.randint(0, most + 1, (*size, 2), generator=gen) + 8 * torch.randint(0, 2, (*size, 2), generator=gen)
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("byte,most", [(252, 7), (253, 5), (254, 3)])
def test_large_scales(byte, most, T, dtype):
    """Elements below 2^128 are what they are, whatever the scale; one of 2^128 or more counts as infinite."""
    gen = torch.Generator().manual_seed(byte + T)
    up, ups = codes_up_to(gen, 7, E, 2 * F, K // 2), torch.full((E, 2 * F, 4), 66, dtype=torch.uint8)             # (h of some 2^-110, and results of some 2^10)
    down, downs = codes_up_to(gen, most, E, K, -(-F // 32) * 16), torch.full((E, K, 4), byte, dtype=torch.uint8)
    x = torch.randn(T, K, generator=gen).to(dtype)
    ids, w = torch.randint(0, E - 1, (T, 2), generator=gen, dtype=torch.int32), torch.rand(T, 2, generator=gen) * 2.0 ** -10
    want, off = ref.experts(ref.values(up, ups[..., :2], K), ref.values(down, downs[..., :3], F), x.double(), ids, w, dtype)

    def run():
        return dg.dg_experts_mx4(up.to(DEV), ups.to(DEV)[..., :2], down.to(DEV), downs.to(DEV)[..., :3], x.to(DEV), ids.to(DEV), w.to(DEV))

    clean = run()
    assert torch.isfinite(want).all() and want.abs().max() > 2.0 ** -14
    ref.assert_within(clean, want, off)
    if byte > 252:
        ids[T // 2, 0], down[E - 1, 7, 3] = E - 1, 0x77                                                            # (6 * 2^126 or 2^127)
        got, others = run(), torch.arange(T) != T // 2
        assert torch.equal(got[others], clean[others]) and not torch.isfinite(got[T // 2, 7])


def test_the_quantiser_writes_no_element_of_2_to_the_128():
    most = torch.finfo(torch.float32).max
    x = torch.full((3, 64), most, device=DEV)
    x[1], x[2, ::2] = -most, 2.0 ** 127
    codes, scales = dg.dg_quantize_mx4(x)
    assert int(scales.max()) == 252 and torch.isfinite(dg.dg_dequantize_mx4(codes, scales)).all()
