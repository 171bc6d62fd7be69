"""Attention on the GPU within the bound of attention_bound.py, on queries that show a token that is missing, out of place or counted twice."""
import numpy as np
import pytest
import torch

from attention_bound import UNIT, attention_bound, stored, telling_queries
from test_gpu_decoder import LAYOUTS, TYPES, Batch, as_f32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def one_thread():
    """(the oracle's products are small: threads only wait for one another)"""
    threads = torch.get_num_threads()
    torch.set_num_threads(1)
    yield
    torch.set_num_threads(threads)


class Told(Batch):
    """A batch that keeps what it wrote, and whose queries are the telling ones."""

    def __init__(self, new, ctx, Hq, H, D, page, bits, dtype, seed=0, change=None, turn=0):
        written = []
        def keep(b, k, v):
            if change:
                change(b, k, v)
            written.append((k.clone(), v.clone()))
        super().__init__(new, ctx, Hq, H, D, page, bits, dtype, seed=seed, change=keep)
        self.bits = bits
        self.kv = [tuple(x.to(TYPES[dtype]).float() for x in kv) for kv in written]
        for b, (n, c) in enumerate(zip(new, ctx)):
            rows = slice(self.start[b], self.start[b + 1])
            if n and c >= 30:
                self.q[rows] = telling_queries(self.q[rows], self.kv[b][0], c - n, True, page, turn, D ** -0.5)

    def within(self, got, causal=True):
        got, q = as_f32(got).astype(np.float64), self.q.float().numpy()
        for b, (n, c) in enumerate(zip(self.new, self.ctx)):
            rows = slice(self.start[b], self.start[b + 1])
            k, v = (stored(x.numpy(), self.bits) for x in self.kv[b])
            want, off = attention_bound(q[rows], k, v, c - n, self.desc.dim ** -0.5, causal, self.bits, self.dtype)
            worst = (np.abs(got[rows] - want) / off).max() if n else 0
            print(f"sequence {b}: {n} on {c}, worst {worst:.2f} of the bound")
            assert worst <= 1, (b, n, c, worst)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_attention(layout, bits, dtype):
    for turn in range(3):
        batch = Told(*LAYOUTS[layout], bits, dtype, seed=100 + layout, turn=turn)
        batch.within(batch.run())
    batch.within(batch.run(causal=False), causal=False)


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits,dtype", [(8, "f16"), (8, "bf16"), (4, "f16"), (4, "bf16")])
@pytest.mark.parametrize("layout", [3, 4, 7, 10, 11, 13])
def test_attention_by_any_number_of_rows(layout, bits, dtype, rows, monkeypatch):
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    for turn in range(3):
        batch = Told(*LAYOUTS[layout], bits, dtype, seed=200 + layout, turn=turn)
        batch.within(batch.run())


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,ctx", [(1, 300), (1, 3000), (45, 700)])
@pytest.mark.parametrize("what", ["large", "small", "a few large", "a few small", "a ramp", "half zero", "zero but for large ones", "all alike", "an outlier"])
def test_values_of_any_size(what, new, ctx, bits, rows, monkeypatch):
    """bfloat16's range of values, and tokens of very different ones beside one another: the bound is relative to what a row's weights and values add up to."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    def change(b, k, v):
        few = [5, 40, ctx // 2, ctx - new // 2 - 1]
        if what == "large":
            v *= 1e30
        if what == "small":
            v *= 1e-24
        if what == "a few large":
            v[few] *= 1e20
        if what == "a few small":
            v[few] *= 1e-25
        if what == "a ramp":
            v *= torch.logspace(-12, 12, ctx)[:, None, None]
        if what == "half zero":
            v[::2] = 0
        if what == "zero but for large ones":
            v[[t for t in range(ctx) if t % 64 != 17]] = 0
            v *= 1e30
        if what == "all alike":
            v[::3] = v[::3, :, :1]
            v[1::3] = 1e10
        if what == "an outlier":
            v[ctx // 3] *= 1e6
    for turn in range(3):
        batch = Told([new], [ctx], 4, 2, 64, 16, bits, "bf16", seed=7, turn=turn, change=change)
        batch.within(batch.run())


def cancelling(weights, bits):
    """Two tokens of nearly the same logit whose values cancel, among others that count for nothing: the output is the weights' difference, so that what a weight
    loses is large beside the output's own rounding.  Queries [24][1][64], keys and values [40][1][64]; with `weights(w)` in place of w, the outputs, else None."""
    gen = torch.Generator().manual_seed(5)
    q, k, v = torch.zeros(24, 1, 64), torch.zeros(40, 1, 64), torch.randn(40, 1, 64, generator=gen)
    q[:, 0, 0] = torch.linspace(4.0, 12.0, 24)
    k[:, 0, 0] = -1000.0
    k[11, 0, 0], k[30, 0, 0] = 1.0, 0.98
    v[30] = -v[11]
    q, k, v = q.half(), k.half(), v.half()
    (kv, _, _), (vv, _, mid) = (stored(x.float().numpy(), bits) for x in (k, v))
    logit = 0.125 * (q[:, 0].double().numpy() @ kv[:, 0].astype(np.float64).T)
    w = np.exp(logit - logit.max(1, keepdims=True))
    V, c = vv[:, 0].astype(np.float64), vv[:, 0].astype(np.float64) - mid[:, 0, None]
    want = w @ V / w.sum(1, keepdims=True)
    # the output's own rounding, and 2^-18 of what cancels (weights in two halves 2^-22, their powers 2^-21, logits below 4 to 2^-22 each)
    off = UNIT["f16"] * np.abs(want) + 2.0 ** -18 * (w @ np.abs(V)) / w.sum(1, keepdims=True) + 2.0 ** -25
    return q, k, v, want, off, None if weights is None else (weights(w) @ c + w @ (V - c)) / w.sum(1, keepdims=True)


@pytest.mark.parametrize("rows", ["16", "32", "128"])
@pytest.mark.parametrize("bits", [8, 4])
def test_binary16_outputs_take_more_than_binary16_of_a_weight(bits, rows, monkeypatch):
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    q, k, v, want, off, _ = cancelling(None, bits)
    def change(b, keys, values):
        keys.copy_(k)
        values.copy_(v)
    batch = Batch([24], [40], 1, 1, 64, 16, bits, "f16", change=change)
    got = as_f32(batch.run(q=q.cuda(), causal=False))[:, 0]
    assert (np.abs(got - want) <= off).all(), (np.abs(got - want) / off).max()


@pytest.mark.parametrize("rows", ["16", "32"])
@pytest.mark.parametrize("bits", [8, 4])
def test_binary16_outputs_of_a_long_context_are_rounded_once(bits, rows, monkeypatch):
    """Over tens of thousands of tokens alike, what the kernels add to the outputs' own rounding is at most a fifth of that: the errors' root mean square is
    within sqrt(1 + 1 / 25) < 1.02 of the rounding's."""
    monkeypatch.setenv("DG_ATTENTION_ROWS", rows)
    ctx, Hq, H, D = 60000, 16, 4, 128
    written = []
    def keep(b, k, v):
        written.append((k.half().float(), v.half().float()))
    batch = Batch([1], [ctx], Hq, H, D, 64, bits, "f16", seed=9, change=keep)
    got = as_f32(batch.run()).astype(np.float64)[0]
    (kv, _, _), (vv, _, _) = (stored(x.numpy(), bits) for x in written[0])
    off, own = 0.0, 0.0
    for j in range(Hq):
        s = D ** -0.5 * (kv[:, j // 4].astype(np.float64) @ batch.q[0, j].double().numpy())
        w = np.exp(s - s.max())
        want = (w @ vv[:, j // 4].astype(np.float64)) / w.sum()
        off += np.square(got[j] - want).sum()
        own += np.square(want.astype(np.float16) - want).sum()
    print(f"errors {np.sqrt(off / own):.4f} times the rounding's")
    assert off <= 1.02 ** 2 * own
