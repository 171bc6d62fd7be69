"""Microscaled 4-bit floating point, a router and experts, plainly and in 64 bits on the CPU, with what results may be off by."""
import math

import torch

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def nearest_code(a):
    """The code (0 ... 7) nearest to a >= 0: the levels one by one, of two as near the even code."""
    best = 0
    for c in range(1, 8):
        d, b = abs(LEVELS[c] - a), abs(LEVELS[best] - a)
        if d < b or (d == b and c % 2 == 0):
            best = c
    return best


# the borders by that rule: below or at the one, above the other
BORDERS = [(LEVELS[c] + LEVELS[c + 1]) / 2 for c in range(7)]


def quantize(x):
    """[N][K] -> codes uint8 [N][blocks][32] (zeros from K on) and scale bytes uint8 [N][blocks]."""
    N, K = x.shape
    blocks = -(-K // 32)
    y = torch.zeros(N, blocks * 32, dtype=torch.float64)
    y[:, :K] = x.double()
    sign = torch.zeros(N, blocks * 32, dtype=torch.bool)
    sign[:, :K] = torch.signbit(x.float())
    y, sign = y.view(N, blocks, 32), sign.view(N, blocks, 32)
    most = y.abs().amax(2)
    bad = ~torch.isfinite(y).all(2)
    exponent = torch.full_like(most, -127)
    there = (most > 0) & ~bad
    exponent[there] = (torch.frexp(most[there]).exponent - 1 - 2).clamp(-127, 127).double()
    a = y.abs() / torch.exp2(exponent)[..., None]
    codes = torch.zeros_like(a, dtype=torch.uint8)
    for c, border in enumerate(BORDERS):
        codes += (a > border) | ((a == border) & (c % 2 == 1))
    codes = codes + 8 * sign.to(torch.uint8)
    codes[bad] = 0
    return codes, torch.where(bad, 255.0, exponent + 127).to(torch.uint8)


def pack(codes):
    codes = codes.flatten(1)
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def values(packed, scales, K):
    """What codes (uint8 [..., 16 * blocks]) and scales stand for, 64 bits, the first K of each row."""
    codes = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    x = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64)[codes.long()].unflatten(-1, (-1, 32))
    s = torch.exp2(scales.double() - 127)
    s[scales == 255] = math.nan
    return (x * s[..., None]).flatten(-2)[..., :K]


def rounding(y, dtype):
    """Half a step of `dtype` at y, and what lies below its smallest numbers."""
    return y.abs() * (torch.finfo(dtype).eps / 2) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def product(A, W, bias, dtype):
    """[N][K], [M][K] in 64 bits -> the result and how far one of `dtype` may be off: binary32 sums of an instruction's 64 products at least, behind one another and over
    up to 16 wavefronts, each rounded to 2^-24 of what no partial sum exceeds; within an instruction products are cut at 2^-28 of the largest."""
    y = A @ W.t()
    size = A.abs() @ W.abs().t()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    steps = A.shape[1] / 64 + 32
    off = size * (steps * 2.0 ** -24 + 64 * 2.0 ** -28)
    return y, off + rounding(y.abs() + off, dtype)


def route(x, R, top, mode, bias, factor):
    """-> ids, weights (64 bits) by the header's rules, token by token."""
    logits = (x.double() @ R.double().t()).float().double()
    T, E = logits.shape
    ids, weights = torch.full((T, top), -1, dtype=torch.int32), torch.zeros(T, top, dtype=torch.float64)
    for t in range(T):
        l = logits[t]
        chance = 1 / (1 + torch.exp(-l))
        choice = (chance if mode == "sigmoid" else l) + (0 if bias is None else bias.double())
        if torch.isnan(l).any() or torch.isnan(choice).any():
            ids[t], weights[t] = torch.arange(top, dtype=torch.int32), math.nan
            continue
        taken = [e for e in sorted(range(E), key=lambda e: (-choice[e].item(), e)) if choice[e] != -math.inf][:top]
        if not taken:
            continue
        ids[t, :len(taken)] = torch.tensor(taken, dtype=torch.int32)
        if mode == "sigmoid":
            w = chance[taken] / chance[taken].sum()
        else:
            over = l if mode == "softmax_all" else l[taken]
            w = torch.exp(l[taken] - over.max()) / torch.exp(over - over.max()).sum()
        weights[t, :len(taken)] = w * factor
    return ids, weights


def experts(up, down, x, ids, weights, dtype):
    """up [E][2F][K], down [E][K][F], x in 64 bits -> the result and how far one of `dtype` may be off: binary32 sums as in `product`, of at least 32 products a step; h is held to
    2^-17, and comes out of a handful of binary32 operations, exp among them."""
    T, K = x.shape
    E, F = up.shape[0], up.shape[1] // 2
    y, off = torch.zeros(T, K, dtype=torch.float64), torch.zeros(T, K, dtype=torch.float64)
    e24 = 2.0 ** -24
    steps_up, steps_down = K / 16 + 32, F / 16 + 32
    for t in range(T):
        for j in range(ids.shape[1]):
            e, w = int(ids[t, j]), weights[t, j].double()
            if not 0 <= e < E:
                continue
            g, u = (up[e] @ x[t]).split(F)
            og, ou = ((up[e].abs() @ x[t].abs()) * (steps_up * e24 + 64 * 2.0 ** -28)).split(F)
            s = g * torch.sigmoid(g)
            h = s * u
            oh = 1.1 * og * (u.abs() + ou) + s.abs() * ou + h.abs() * (2.0 ** -17 + 16 * e24)
            y[t] += w * (down[e] @ h)
            size = w.abs() * (down[e].abs() @ h.abs())
            off[t] += w.abs() * (down[e].abs() @ oh) + size * ((steps_down + ids.shape[1] + 4) * e24 + 64 * 2.0 ** -28)
    return y, off + rounding(y.abs() + off, dtype)


def assert_within(got, want, off, what=""):
    """Element by element; where the reference is not a number, or is infinite, the result has to be too."""
    got, strange = got.double().cpu(), ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[strange].nan_to_num(7), want[strange].nan_to_num(7)), what
    wrong = ((got - want).abs() > off) & ~strange
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()}, the first at {wrong.nonzero()[0].tolist()}: {got[wrong][0]} for {want[wrong][0]} +- {off[wrong][0]}"
