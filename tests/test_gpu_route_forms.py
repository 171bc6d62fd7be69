"""The router's kernels for many tokens, and one work buffer for batches of all sizes."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def operands(gen, T, K, E, dtype, rdtype):
    x = torch.randn(T, K, generator=gen, device=DEV).to(ref.TYPES[dtype])
    return x, (torch.randn(E, K, generator=gen, device=DEV) * K ** -0.5).to(ref.TYPES[rdtype])


@pytest.mark.parametrize("K,E", [(1024, 64), (1100, 16), (200, 130)])
def test_one_buffer_for_all_batches(K, E):
    gen = torch.Generator(device=DEV).manual_seed(E)
    x, R = operands(gen, 1300, K, E, "bf16", "bf16")
    work = torch.empty(dg.dg_route_tokens_work_bytes(1300, E), dtype=torch.uint8, device=DEV)
    for T in (1300, 1, 768, 3, 769, 512, 40, 1024, 200, 41):
        ids, w = dg.dg_route_tokens(x[:T], R, 4, work=work)
        alone = dg.dg_route_tokens(x[:T], R, 4)
        assert torch.equal(ids, alone[0]) and torch.equal(w, alone[1])
        logits = (x[:T].cpu().double() @ R.cpu().double().t()).float()
        want = torch.sort(logits, dim=1, descending=True, stable=True)
        assert torch.equal(ids.cpu().long(), want.indices[:, :4])
        # a softmax over four: exponents of at most some 10, two exponentials, a sum of 4 and a quotient
        ref.assert_within(w, torch.softmax(want.values[:, :4].double(), 1), torch.full((T, 4), 64 * 2.0 ** -24, dtype=torch.float64))


@pytest.mark.parametrize("dtype,rdtype", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("T,K,E", [(4100, 200, 128), (4111, 1031, 130), (8200, 72, 64), (2060, 520, 256)])
def test_tiles_of_32(T, K, E, dtype, rdtype):
    """512 tiles and more, the last ones ragged."""
    gen = torch.Generator(device=DEV).manual_seed(T + K)
    x, R = operands(gen, T, K + 3, E, dtype, rdtype)
    x, R = x[:, 1:K + 1], R[:, 3:]                                    # (rows that begin anywhere)
    bias = 0.1 * torch.randn(E, generator=gen, device=DEV)
    ids, w = dg.dg_route_tokens(x, R, 5, mode="sigmoid", bias=bias)
    logits = (x.double() @ R.double().t()).float().cpu()
    choice = torch.sigmoid(logits.double()) + bias.cpu().double()
    want = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(ids.cpu().long(), want)
    chance = torch.sigmoid(logits.double()).gather(1, want)
    # five sigmoids, each an exponential, a sum and a quotient, their sum and a quotient, all below 1
    ref.assert_within(w, chance / chance.sum(1, keepdim=True), torch.full((T, 5), 32 * 2.0 ** -24, dtype=torch.float64))


def test_sigmoids_that_binary32_does_not_hold():
    """Of logits from -60 to -700 too the weights are the sigmoids' shares; of those whose sigmoids are 0 in 64 bits they are 0."""
    low = torch.tensor([-60.0, -80.5, -87.0, -89.0, -95.0, -103.0, -104.0, -120.0, -300.0, -700.0])
    R = torch.ones(7, 4)
    R[1], R[2], R[5] = 1.015625, 0.984375, 2.0                        # (exact: what the logits are is known)
    x = low[:, None].expand(-1, 4) / 4
    for scale in (1.0, 2.5):
        ids, w = dg.dg_route_tokens(x.to(DEV).contiguous(), R.to(DEV), 3, mode="sigmoid", factor=scale)
        want_ids, want = ref.route(x, R, 3, "sigmoid", None, scale)
        assert torch.equal(ids.cpu(), want_ids)
        # three sigmoids in binary32 (an exponential each: a few units), a sum, a quotient and a product
        ref.assert_within(w, want, 32 * 2.0 ** -24 * want)
        assert ((w.sum(1) - scale).abs() <= scale * 8 * 2.0 ** -24).all()
    ids, w = dg.dg_route_tokens(torch.full((2, 4), -300.0, device=DEV), torch.ones(3, 4, device=DEV), 2, mode="sigmoid")
    assert ids.tolist() == [[0, 1]] * 2 and (w == 0).all()            # exp(-1200)
