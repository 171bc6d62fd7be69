"""What the example layer of experts refuses, without a GPU."""
import pytest
import torch

from paper_2304_09049_amd.decoder_layer import DecoderLayer, ExpertsLayer


def shapes(experts=4, hidden=64, inner=32, shared=96):
    return dict(w_qkv=(256, hidden), w_out=(hidden, 128), router=(experts, hidden), up=(experts, 2 * inner, hidden), down=(experts, hidden, inner),
                shared_up=(2 * shared, hidden), shared_down=(hidden, shared))


@pytest.mark.parametrize("change,match", [({"up": (4, 64, 32)}, "experts on 64"), ({"up": (3, 64, 64)}, "experts on 64"), ({"up": (4, 32, 64)}, "experts on 64"),
                                          ({"down": (4, 32, 32)}, "experts on 64"), ({"down": (5, 64, 32)}, "experts on 64"), ({"router": (4, 32)}, "experts on 32"),
                                          ({"shared_up": (96, 64)}, "shared up"), ({"shared_up": (192, 32)}, "shared up"), ({"shared_down": (32, 96)}, "shared up"),
                                          ({"top": 5}, "5 of 4 experts"), ({"top": 0}, "0 of 4 experts")])
def test_weights_that_do_not_fit(change, match):
    top = change.pop("top", 2) if "top" in change else 2
    weights = {name: torch.zeros(size) for name, size in {**shapes(), **change}.items()}
    with pytest.raises(ValueError, match=match):
        ExpertsLayer(**weights, heads=2, kv_heads=1, dim=64, top=top)


def test_it_is_the_layer_with_another_feed_forward_part():
    assert issubclass(ExpertsLayer, DecoderLayer) and ExpertsLayer.attend is DecoderLayer.attend and ExpertsLayer.step is DecoderLayer.step
