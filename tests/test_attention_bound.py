"""The bound that attention is held to, held itself against oracles that are wrong: each has to be rejected."""
import numpy as np
import pytest
import torch

from attention_bound import attention_bound, edges, stored, telling_queries, weights_of
from test_gpu_decoder import LAYOUTS, TYPES

LONG = [LAYOUTS[i] for i in (1, 2, 3, 4, 7, 10, 11, 13)]


@pytest.fixture(autouse=True)
def one_thread():
    """(the products here are small: threads only wait for one another)"""
    threads = torch.get_num_threads()
    torch.set_num_threads(1)
    yield
    torch.set_num_threads(threads)


def sequences(layout, bits, dtype, turn):
    """A layout's sequences: queries, what is stored of keys and values, the past, the page."""
    new, ctx, Hq, H, D, page = layout
    gen = torch.Generator().manual_seed(turn + 10 * bits)
    for n, c in zip(new, ctx):
        k, v = (torch.randn(c, H, D, generator=gen).to(TYPES[dtype]) for _ in range(2))
        q = (2 * torch.randn(n, Hq, D, generator=gen)).to(TYPES[dtype])
        if n and c >= 30:
            q = telling_queries(q, k, c - n, True, page, turn, D ** -0.5)
            yield q.float().numpy(), stored(k.float().numpy(), bits), stored(v.float().numpy(), bits), c - n, page


def without(tokens):
    """The softmax of what is left when each row loses a token."""
    def change(w, V, page):
        seen = (w > 0).sum(1)
        w = w.clone()
        w[torch.arange(len(w)), torch.tensor([min(max(tokens(int(s), page), 0), max(int(s) - 1, 0)) for s in seen])] = 0
        return w / w.sum(1, keepdim=True).clamp_min(1e-300), V
    return change


def newest_swapped(w, V, page):
    """Each row's last two tokens changing places."""
    w, row, last = w.clone(), torch.arange(len(w)), ((w > 0).sum(1) - 1).clamp_min(1)
    w[row, last], w[row, last - 1] = w[row, last - 1], w[row, last]
    return w, V


def first_twice(w, V, page):
    w = w.clone()
    w[:, 0] *= 2
    return w / w.sum(1, keepdim=True).clamp_min(1e-300), V


def rounded_weights(bits):
    def change(w, V, page):
        step = 2.0 ** (torch.floor(torch.log2(w.clamp_min(1e-300))) - (bits - 1))
        return torch.round(w / step) * step, V
    return change


WRONG = {  # what each row has instead of its softmax and the values
    "newest missing": without(lambda seen, page: seen - 1),                      # a causal mask one short
    "first missing": without(lambda seen, page: 0),
    "one in the middle missing": without(lambda seen, page: seen // 2 + 3),
    "a page's last missing": without(lambda seen, page: page - 1),
    "newest two swapped": newest_swapped,
    "values one token off": lambda w, V, page: (w, V.roll(1, 0)),
    "first counted twice": first_twice,
}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("layout", range(len(LONG)))
def test_wrong_oracles_are_rejected(layout, bits, dtype):
    """Over the kinds of rows, each is beyond the bound somewhere."""
    wrong = dict(WRONG, **{"weights of few bits": rounded_weights(8 if dtype == "f16" else 5)})
    worst = dict.fromkeys(wrong, 0.0)
    for turn in range(3):
        for q, k, v, past, page in sequences(LONG[layout], bits, dtype, turn):
            want, off, others = attention_bound(q, k, v, past, q.shape[2] ** -0.5, True, bits, dtype,
                                                [lambda w, V, f=f: f(w, V, page) for f in wrong.values()])
            for name, got in zip(wrong, others):
                worst[name] = max(worst[name], (np.abs(got - want) / off).max())
    assert min(worst.values()) > 1, worst


def test_the_bound_is_small():
    """Against the outputs themselves: a hundredth of their mean magnitude, where the weights' rounding and the outputs' are most of it."""
    for layout in LONG:
        for bits in (8, 4):
            for dtype in ("f16", "bf16"):
                for q, k, v, past, _ in sequences(layout, bits, dtype, 0):
                    want, off = attention_bound(q, k, v, past, q.shape[2] ** -0.5, True, bits, dtype)
                    assert np.median(off) < 0.02 * np.abs(want).mean(), (layout, bits, dtype)


def test_the_formula_by_hand():
    q = np.zeros((2, 1, 64), np.float32)
    q[0, 0, 0], q[1, 0, 0] = 8.0, 16.0
    k, v = np.zeros((3, 1, 64), np.float32), np.zeros((3, 1, 64), np.float32)
    k[:, 0, 0] = [0.0, np.log(2), np.log(3)]
    v[:, 0, 0], v[:, 0, 5] = [127.0, 0.0, -127.0], [1.0, 127.0, 3.0]
    want, off = attention_bound(q, stored(k, 8), stored(v, 8), 1, 0.125, True, 8, "f16")
    held = stored(k, 8)[0][:, 0, 0].astype(np.float64)
    w0, w1 = np.exp(held[:2]), np.exp(2 * held)
    assert abs(want[0, 0, 0] - 127 * w0[0] / w0.sum()) < 1e-9 and abs(want[1, 0, 5] - (w1 @ [1, 127, 3]) / w1.sum()) < 1e-9
    assert (off < 0.2).all()


def test_what_telling_queries_tell():
    gen = torch.Generator().manual_seed(0)
    k = torch.randn(700, 2, 64, generator=gen).half()
    q = telling_queries((2 * torch.randn(90, 4, 64, generator=gen)).half(), k, 610, True, 16, 0, 0.125)
    shares, alike = [], []
    for i in range(90):
        for j in range(4):
            w, _ = weights_of(q[i, j][None].double(), k[:, j // 2].double(), torch.arange(700)[None] < 611 + i, 0.125)
            if (i * 4 + j) % 3 == 1:
                shares.append(float(w.max()))
                assert int(w.argmax()) in edges(611 + i, 16)
            if (i * 4 + j) % 3 == 2:
                alike.append(float(w.max() / w[w > 0].min()))
    assert 0.2 < min(shares) and max(shares) < 0.9 and max(alike) < 1.3


@pytest.mark.parametrize("bits", [8, 4])
def test_weights_of_one_binary16_are_rejected_for_binary16_outputs(bits):
    from test_gpu_attention_bound import cancelling
    half = lambda w: w.astype(np.float16).astype(np.float64)  # noqa: E731
    for weights, fine in ((half, False), (lambda w: half(w) + half(w - half(w)), True)):
        *_, want, off, got = cancelling(weights, bits)
        assert ((np.abs(got - want) / off).max() <= 1) == fine
