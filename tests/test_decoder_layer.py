"""The example layer's bookkeeping, without a GPU."""
import pytest
import torch

from paper_2304_09049_amd import binding as dg
from paper_2304_09049_amd.decoder_layer import DecoderLayer, PagedSequences


def test_pages_go_to_the_sequences_as_tokens_come():
    s = PagedSequences(dg.cache_desc(5, 16, 1, 64, 8), 2, "cpu")
    slots, start, ctx, table = s.extend([17, 0])
    assert start.tolist() == [0, 17, 17] and ctx.tolist() == [17, 0] and table.tolist() == [s.pages[0], [-1, -1]]
    assert slots.tolist() == [s.pages[0][t // 16] * 16 + t % 16 for t in range(17)]
    slots, start, ctx, table = s.extend([15, 33])
    assert len(s.pages[0]) == 2 and len(s.pages[1]) == 3 and not s.free and ctx.tolist() == [32, 33] and start.tolist() == [0, 15, 48]
    assert sorted(s.pages[0] + s.pages[1]) == [0, 1, 2, 3, 4]
    slots, *_ = s.extend([0, 0])
    assert slots.numel() == 0


def test_a_pool_that_does_not_suffice_stays_as_it_was():
    s = PagedSequences(dg.cache_desc(3, 16, 1, 64, 8), 2, "cpu")
    s.extend([16, 3])
    before = [list(p) for p in s.pages], list(s.lengths), list(s.free)
    with pytest.raises(MemoryError, match="2 more pages are needed, 1 of 3 are free"):
        s.extend([1, 14])
    assert ([list(p) for p in s.pages], list(s.lengths), list(s.free)) == before
    for wrong in ([1], [1, 1, 1], [1, -1]):
        with pytest.raises(ValueError, match="for 2 sequences"):
            s.extend(wrong)
    assert ([list(p) for p in s.pages], list(s.lengths), list(s.free)) == before
    s.extend([1, 13])
    assert s.lengths == [17, 16] and not s.free


def test_two_bit_weights_of_channels_that_are_zero():
    w = torch.tensor([[2.0, -2.0, 0.4, -1.2], [0.0, 0.0, 0.0, 0.0], [0.0, 0.0, -1e-30, 0.0]])
    codes, scale = DecoderLayer.two_bits(w)
    assert codes.dtype == torch.uint8 and codes.tolist() == [[3, 0, 2, 1], [2, 2, 2, 2], [2, 2, 0, 2]]
    assert scale.tolist() == [1.0, 0.0, w[2, 2].abs().item() / 2]
