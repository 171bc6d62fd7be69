"""The example layer of experts: its calls together, each against 64 bits on what the one before gave it."""
import pytest
import torch

import mx4_reference as ref
from paper_2304_09049_amd import binding as dg
from paper_2304_09049_amd.decoder_layer import ExpertsLayer, PagedSequences

pytestmark = pytest.mark.gpu
HIDDEN, HEADS, KV_HEADS, DIM, EXPERTS, INNER, SHARED, TOP = 256, 4, 2, 64, 8, 96, 160, 3


def layer_of(seed=4, mode="softmax", bias=False):
    gen = torch.Generator().manual_seed(seed)
    sizes = ((HEADS + 2 * KV_HEADS) * DIM, HIDDEN), (HIDDEN, HEADS * DIM), (EXPERTS, HIDDEN), (EXPERTS, 2 * INNER, HIDDEN), (EXPERTS, HIDDEN, INNER), (2 * SHARED, HIDDEN), (HIDDEN, SHARED)
    weights = [(torch.randn(*size, generator=gen) * size[-1] ** -0.5).cuda() for size in sizes]
    b = (0.1 * torch.randn(EXPERTS, generator=gen)).cuda() if bias else None
    return ExpertsLayer(*weights, HEADS, KV_HEADS, DIM, TOP, mode, b), weights, gen


def quantised(w):
    """What a row-wise quantised matrix (or one per expert) stands for, in 64 bits."""
    flat = w.cpu().flatten(0, -2)
    codes, scales = ref.quantize(flat)
    return ref.values(ref.pack(codes), scales, w.shape[-1]).view(w.shape)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("mode,bias", [("softmax", False), ("softmax_all", True), ("sigmoid", True)])
@pytest.mark.parametrize("new", [[1, 0, 0], [1, 1, 1], [40, 1, 9], [70, 64, 100]])
def test_feed_forward(new, mode, bias, dtype):
    layer, weights, gen = layer_of(sum(new), mode, bias)
    router, up, down, shared_up, shared_down = weights[2:]
    x = torch.randn(sum(new), HIDDEN, generator=gen).to(dtype).cuda()
    h = layer.attend(x, PagedSequences(dg.cache_desc(24, 16, KV_HEADS, DIM, 8), 3, x.device), new)
    assert h.dtype == dtype
    got = layer.feed_forward(h)
    ids, w = dg.dg_route_tokens(h, layer.router, TOP, mode, layer.bias)
    want_ids, want_w = ref.route(h.cpu(), router.cpu(), TOP, mode, None if layer.bias is None else layer.bias.cpu(), 1.0)
    assert torch.equal(ids.cpu(), want_ids)
    assert ((w.cpu() - want_w).abs() <= 64 * 2.0 ** -24 * want_w).all()              # (two exponentials of some 2^-22 each, a sum of 8 and a quotient)
    chosen = dg.dg_experts_mx4(*layer.experts, h, ids, w)
    ref.assert_within(chosen, *ref.experts(quantised(up), quantised(down), h.cpu().double(), ids.cpu(), w.cpu(), dtype))
    both = dg.dg_linear_mx4(*layer.shared_up, h)
    ref.assert_within(both, *ref.product(quantised(h), quantised(shared_up), None, dtype))
    middle = torch.nn.functional.silu(both[:, :SHARED]) * both[:, SHARED:]
    shared = dg.dg_linear_mx4(*layer.shared_down, middle)
    ref.assert_within(shared, *ref.product(quantised(middle), quantised(shared_down), None, dtype))
    assert torch.equal(got, chosen + shared)


def test_a_step_without_new_tokens():
    layer, _, gen = layer_of()
    sequences = PagedSequences(dg.cache_desc(8, 16, KV_HEADS, DIM, 8), 2, torch.device("cuda"))
    x = torch.randn(5, HIDDEN, generator=gen).bfloat16().cuda()
    assert layer.step(x, sequences, [2, 3]).isfinite().all()
    none = layer.step(x[:0], sequences, [0, 0])
    assert none.shape == (0, HIDDEN) and none.dtype == x.dtype


@pytest.mark.parametrize("tokens", [1, 5, 33])
def test_the_feed_forward_part_in_a_graph(tokens):
    """Captured once and replayed on other tokens, with the same calls run eagerly between the replays."""
    layer, _, gen = layer_of()
    h = torch.randn(tokens, HIDDEN, generator=gen).bfloat16().cuda()
    layer.feed_forward(h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.feed_forward(h)
    for _ in range(4):
        h.copy_(torch.randn(tokens, HIDDEN, generator=gen).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, layer.feed_forward(h))
