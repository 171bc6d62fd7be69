"""Attention: what a row gives goes by its own query and by the tokens that it sees, whatever stands beside it."""
import numpy as np
import pytest
import torch

from test_gpu_decoder import Batch, as_f32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,ctx,Hq,H,D", [(1, 300, 16, 1, 128), (40, 500, 4, 2, 64), (9, 100, 2, 1, 256)])
@pytest.mark.parametrize("power", [20, 30, 38, 60, 100])
def test_queries_of_very_different_sizes(power, new, ctx, Hq, H, D, bits, rows, monkeypatch):
    """Every third row's query 2^power times its neighbours': the neighbours' outputs are what they are without it.  Both runs are within a weight's rounding
    (2^-11 of the sum of weights times values, here at most the largest value), their scores' errors (below 2^-11 too: logits of at most some tens, 2^-16 of
    them) and a bfloat16's rounding (2^-8 of the output) of the exact result: their difference is within twice that."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    batch = Batch([new], [ctx], Hq, H, D, 16, bits, "bf16", seed=power)
    plain = as_f32(batch.run())
    large = torch.arange(new * Hq).view(new, Hq) % 3 == 1
    batch.q[large] *= 2.0 ** power
    got = as_f32(batch.run())
    off = 2 * (2.0 ** -8 * np.abs(plain) + 2 * 2.0 ** -11 * max(np.abs(v).max() for v in batch.v))
    assert (np.abs(got - plain) <= off)[~large.numpy()].all()
