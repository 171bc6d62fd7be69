"""Experts of several tiles a workgroup, whose loads run on from one tile into the next, and of more pairs than a pass takes, against 64 bits."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def some_weights(gen, E, rows, size):
    """Any codes, and scales that differ by 2^-3 ... 2^0 so that one that is another block's shows: of [E][rows] rows of `size`, on the device."""
    blocks = -(-size // 32)
    codes = torch.randint(0, 256, (E, rows, 16 * blocks), generator=gen, device=DEV, dtype=torch.uint8)
    if size % 32:                                                     # (codes from `size` on are 0)
        left = size % 32
        codes[..., 16 * blocks - 16 + (left + 1) // 2:] = 0
        if left % 2:
            codes[..., 16 * blocks - 16 + left // 2] &= 15
    scales = torch.full((E, rows, -(-blocks // 4) * 4), 255, device=DEV, dtype=torch.uint8)
    scales[..., :blocks] = torch.randint(118, 122, (E, rows, blocks), generator=gen, device=DEV, dtype=torch.uint8)
    return codes, scales[..., :blocks]


def check(gen, E, K, F, x, ids, weights):
    """Each expert's pairs together, by the formula and with the bound of mx4_reference.experts."""
    up, ups = some_weights(gen, E, 2 * F, K)
    down, downs = some_weights(gen, E, K, F)
    out = dg.dg_experts_mx4(up, ups, down, downs, x, ids, weights)
    want, off, e24 = torch.zeros(x.shape, dtype=torch.float64), torch.zeros(x.shape, dtype=torch.float64), 2.0 ** -24
    wide, its, w = x.cpu().double(), ids.cpu(), weights.cpu().double()
    for e in its.unique().tolist():
        t, j = (its == e).nonzero(as_tuple=True)
        vu, vd = ref.values(up[e].cpu(), ups[e].cpu(), K), ref.values(down[e].cpu(), downs[e].cpu(), F)
        g, u = (wide[t] @ vu.t()).split(F, 1)
        og, ou = ((wide[t].abs() @ vu.abs().t()) * ((K / 16 + 32) * e24 + 64 * 2.0 ** -28)).split(F, 1)
        s = g * torch.sigmoid(g)
        h = s * u
        oh = 1.1 * og * (u.abs() + ou) + s.abs() * ou + h.abs() * (2.0 ** -17 + 16 * e24)
        want.index_add_(0, t, w[t, j, None] * (h @ vd.t()))
        off.index_add_(0, t, w[t, j, None].abs() * (oh @ vd.abs().t() + h.abs() @ vd.abs().t() * ((F / 16 + 32 + ids.shape[1] + 4) * e24 + 64 * 2.0 ** -28)))
    ref.assert_within(out, want, off + ref.rounding(want.abs() + off, x.dtype))
    assert torch.equal(dg.dg_experts_mx4(up, ups, down, downs, x, ids, weights), out)


def tokens(gen, T, K, dtype):
    return torch.randn(T, K, generator=gen, device=DEV).to(ref.TYPES[dtype])


def some_of(gen, T, E, top, which):
    """`top` different ones of `which` experts, spread over all E, a token."""
    names = torch.randperm(E, generator=gen, device=DEV)[:which]
    ids = torch.stack([names[torch.randperm(which, generator=gen, device=DEV)[:top]] for _ in range(T)]).to(torch.int32)
    return ids, torch.softmax(torch.randn(T, top, generator=gen, device=DEV), -1)


# up's stages are ceil(K / 256), down's ceil(F / 256); a workgroup has tiles behind one another from 6 (of 64 rows of up, 128 of down) on
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("E,T,top,which", [(128, 64, 2, 11), (200, 65, 2, 11)])
@pytest.mark.parametrize("K,F", [(320, 330), (700, 500), (1100, 385), (1300, 1100), (2100, 330)])
def test_tiles_behind_one_another(K, F, E, T, top, which, dtype):
    gen = torch.Generator(device=DEV).manual_seed(K + F + E)
    check(gen, E, K, F, tokens(gen, T, K, dtype), *some_of(gen, T, E, top, which))


# by 32 pairs: tiles are twice as large
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("K,F", [(320, 700), (1300, 641), (1100, 700), (2100, 1100)])
def test_tiles_behind_one_another_for_many_pairs(K, F, dtype):
    """Some 160 pairs for each of the eight experts that are named: a workgroup comes back for the next 32."""
    gen = torch.Generator(device=DEV).manual_seed(K + F)
    check(gen, 128, K, F, tokens(gen, 256, K, dtype), *some_of(gen, 256, 128, 5, 8))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,E", [(256, 64), (100, 300), (256, 1), (300, 40)])
def test_all_tokens_name_one_expert(T, E, dtype):
    gen = torch.Generator(device=DEV).manual_seed(T + E)
    ids = torch.full((T, 1), E // 2, dtype=torch.int32, device=DEV)
    check(gen, E, 600, 410, tokens(gen, T, 600, dtype), ids, torch.rand(T, 1, generator=gen, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_turns_of_large_experts(dtype):
    gen = torch.Generator(device=DEV).manual_seed(7)
    check(gen, 6, 2048, 1056, tokens(gen, 515, 2048, dtype), *some_of(gen, 515, 6, 2, 6))
