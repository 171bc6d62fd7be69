"""The example layer at the ends of what it takes."""
import pytest
import torch

from paper_2304_09049_amd import binding as dg
from paper_2304_09049_amd.decoder_layer import DecoderLayer, PagedSequences

pytestmark = pytest.mark.gpu


def layer_of(w_ff=None):
    gen = torch.Generator(device="cuda").manual_seed(2)
    hidden, heads, kv_heads, dim = 256, 4, 2, 64
    weights = [torch.randn(n, m, device="cuda", generator=gen) * m ** -0.5 for n, m in ((8 * dim, hidden), (hidden, heads * dim), (hidden, hidden))]
    return DecoderLayer(*weights[:2], weights[2] if w_ff is None else w_ff(weights[2]), heads, kv_heads, dim), dg.cache_desc(8, 16, kv_heads, dim, 8)


def test_a_step_without_new_tokens():
    layer, desc = layer_of()
    sequences = PagedSequences(desc, 2, torch.device("cuda"))
    x = torch.randn(5, 256, device="cuda").bfloat16()
    first = layer.step(x, sequences, [2, 3])
    held = sequences.cache.clone()
    none = layer.step(x[:0], sequences, [0, 0])
    assert none.shape == (0, 256) and none.dtype == x.dtype
    assert torch.equal(sequences.cache, held) and sequences.lengths == [2, 3] and first.isfinite().all()


def test_a_feed_forward_channel_of_zeros():
    def change(w):
        w[7] = 0
        return w
    layer, desc = layer_of(change)
    sequences = PagedSequences(desc, 1, torch.device("cuda"))
    x = torch.randn(20, 256, device="cuda").half()
    h = layer.attend(x, sequences, [20])
    y = layer.feed_forward(h)
    assert y.isfinite().all() and (y[:, 7] == 0).all() and (y[:, 8] != 0).any()
