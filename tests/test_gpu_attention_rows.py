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


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,ctx,Hq,H,D", [(1, 300, 16, 1, 128), (40, 500, 4, 2, 64), (9, 100, 2, 1, 256)])
def test_a_row_is_the_same_beside_any_other(new, ctx, Hq, H, D, bits, rows, monkeypatch):
    """Whatever the neighbours ask for, a row's bits stay."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    batch = Batch([new], [ctx], Hq, H, D, 16, bits, "bf16", seed=3)
    plain = batch.run()
    other = (torch.arange(new * Hq).view(new, Hq) % 3 == 1)
    for change in (lambda q: q * 2.0 ** 40, lambda q: q * 2.0 ** -40, lambda q: q.flip(0), lambda q: q * 0, lambda q: q * 8, lambda q: q * float("nan")):
        q = batch.q.clone()
        q[other] = change(q[other])
        assert torch.equal(batch.run(q=q.cuda())[~other], plain[~other])


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,ctx,Hq,H,D", [(3, 300, 4, 1, 128), (40, 500, 4, 2, 64), (130, 200, 2, 1, 64), (9, 100, 2, 1, 256)])
def test_a_large_value_that_a_row_does_not_see(new, ctx, Hq, H, D, bits, rows, monkeypatch):
    """Finite keys and values of any size in tokens that only later rows see: the earlier rows' bits stay."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    def batch(size, keys=1.0):
        def change(b, k, v):
            v[-1] *= size
            v[-2] *= size
            k[-1] *= keys
        return Batch([new], [ctx], Hq, H, D, 16, bits, "bf16", seed=4, change=change)
    plain = batch(1.0).run()
    assert plain.isfinite().all()
    for size, keys in ((1e6, 1.0), (1e12, 1.0), (1e20, 1e-10), (1e30, 1.0), (1e-30, 1e20), (0.0, 0.0)):
        assert torch.equal(batch(size, keys).run()[:-2], plain[:-2]), (size, keys)


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,ctx,Hq,H,D", [(1, 300, 8, 1, 128), (1, 3000, 4, 2, 64), (40, 500, 4, 2, 64), (9, 200, 2, 1, 256)])
def test_a_large_value_that_counts_for_nothing(new, ctx, Hq, H, D, bits, rows, monkeypatch):
    """A visible token whose logit is hundreds below the others': its values, of any size, change no bit."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    at = [0, ctx // 3, ctx - new - 1]
    def batch(size):
        def change(b, k, v):
            k[:, :, 5] = 0.0
            k[at] = 0.0
            k[at, :, 5] = -100.0
            v[at] *= size
        made = Batch([new], [ctx], Hq, H, D, 16, bits, "bf16", seed=4, change=change)
        made.q[:, :, 5] = 100.0                                      # logits of -10000 / 8 and less
        return made
    plain = batch(1.0).run()
    for size in (1e6, 1e12, 1e30, 1e-30, 0.0):
        assert torch.equal(batch(size).run(), plain), size
