"""How far attention over the quantised cache may be from its formula in 64 bits, from what the library says it rounds, and inputs that show what is left
out.  The bound is meant to be missed by a wrong kernel: test_attention_bound.py holds it against wrong ones on the CPU."""
import numpy as np
import torch

from decoder_reference import quantize4, quantize8

UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
EPS = 2.0 ** -24                              # binary32's unit roundoff
TIMES = 7.0                                   # Hoeffding: errors bounded by c_i, of mean 0, add up to more than TIMES sqrt(sum c_i^2) once in 2e10


def stored(x, bits):
    """What the cache holds of x [tokens][heads][D] (float32): the values, a token's scale, and the middle that 4-bit codes are counted from (8 scales above z)."""
    if bits == 8:
        c, s = quantize8(x)
        return c.astype(np.float32) * s[..., None], s.astype(np.float64), np.zeros(s.shape)
    c, s, z = quantize4(x)
    return c.astype(np.float32) * s[..., None] + z[..., None], s.astype(np.float64), 8.0 * s + z


def weights_of(q, k, visible, scale):
    """softmax of [rows][tokens] in 64 bits; 0 in a row that sees nothing."""
    s = torch.where(visible, scale * (q @ k.t()), -torch.inf)
    w = torch.exp(s - s.amax(1, keepdim=True).clamp_min(-1e300))
    return w / w.sum(1, keepdim=True).clamp_min(1e-300), torch.where(visible, s, 0.0)


def visible_to(n, ctx, past, causal):
    return torch.arange(ctx)[None] < (past + torch.arange(n)[:, None] + 1 if causal else torch.full((n, 1), ctx))


def attention_bound(q, k, v, past, scale, causal, bits, dtype, wrong=()):
    """One sequence: q float32 [n][Hq][D]; k, v = what `stored` gives of the keys and values.  The outputs in 64 bits [n][Hq][D], and how far the library's may be
    from them.  `wrong`: functions (w [rows][tokens], values) -> (w, values) that make oracles wrong, for the tests of this bound: then the outputs of each besides.

    With w the softmax of a row, s a value's scale, c its code (4 bits: code - 8), o the output, and T the factor of Hoeffding's inequality for roundings of
    mean 0, which are many and independent:
      the output's own rounding            u |o|
      weights to binary16                  T 2^-11 sqrt(sum (w s c)^2), once for bfloat16 outputs; 2^-22 (twice) for binary16 ones; and below 2^-18 of the largest
                                           w s, which is 2^4 at least in binary16, T 2^-29 max(w s) sqrt(sum c^2)
      scores, D additions of (bias + code) times a query's number that begin from the bias' sum, by 32 channels: a token's logit is off by D roundings of at
                                           most EPS M, M = scale ks (bias (largest sum over the blocks left) + (bias + 2^bits) (largest sum of magnitudes of a
                                           block) + most code * sum |q|); in the output T EPS sqrt(D) sqrt(sum (w M (v - o))^2)
      factors of a score, their product, the shift, the exponential (2^-22)
                                           sum w |v - o| (8 EPS (|logit| + |row's largest| + |z sum q|) + 2^-22)
      the sums of weights, and of w * middle  (tokens / 32 + 64) EPS (|o| + sum w |s c| + sum w |middle|)
      outputs, 64 roundings a tile of 32   T EPS 8 sqrt(sum over tiles of ((bias + 2^bits) sum w s + sum of all w s |c|)^2)
    """
    n, Hq, D = q.shape
    (kv, ks, kmid), (vv, vs, vmid) = k, v
    ctx, H = kv.shape[:2]
    out, off, others = np.zeros((n, Hq, D)), np.full((n, Hq, D), 1e-30), np.zeros((len(wrong), n, Hq, D))
    if ctx == 0 or n == 0:
        return (out, off, others) if wrong else (out, off)
    see = visible_to(n, ctx, past, causal)
    bias_k, bias_v, most = (1152.0, 1152.0, 127.0) if bits == 8 else (64.0, 1032.0, 15.0)
    # the order of the first product's blocks: 8 channels of each of 4 pieces of 16
    order = torch.tensor([64 * s + 16 * g + 8 * half + e for s in range(D // 64) for half in range(2) for g in range(4) for e in range(8)])
    for j in range(Hq):
        h = j * H // Hq
        qq = torch.from_numpy(np.ascontiguousarray(q[:, j])).double()
        K, V = (torch.from_numpy(np.ascontiguousarray(x[:, h])).double() for x in (kv, vv))
        sk, sv, mid_v = (torch.from_numpy(np.ascontiguousarray(x[:, h])).double() for x in (ks, vs, vmid))
        z_k = torch.from_numpy(np.ascontiguousarray(kmid[:, h])).double() - (8 * sk if bits == 4 else 0)
        w, logit = weights_of(qq, K, see, scale)
        c = V - mid_v[:, None]                                              # s c
        o = w @ V
        out[:, j] = o.numpy()
        for other, change in zip(others, wrong):
            ww, VV = change(w, V)
            other[:, j] = (ww @ VV).numpy()
        blocks = qq[:, order].view(n, D // 32, 32)
        left = blocks.sum(2).flip(1).cumsum(1).abs().amax(1)
        M = scale * (bias_k * left + (bias_k + 2 ** bits) * blocks.abs().sum(2).amax(1) + most * qq.abs().sum(1))[:, None] * sk
        spread = lambda a: torch.sqrt(torch.clamp(a @ V ** 2 - 2 * (a @ V) * o + a.sum(1, keepdim=True) * o ** 2, min=0))  # noqa: E731   sqrt(sum a (v - o)^2)
        linear = 8 * EPS * (logit.abs() + logit.abs().amax(1, keepdim=True) + scale * (qq.sum(1)[:, None] * z_k).abs()) + 2.0 ** -22
        once = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
        largest = (w * sv).amax(1, keepdim=True)
        codes = torch.where(sv[:, None] > 0, c / sv.clamp_min(1e-300)[:, None], 0.0)
        pad = -ctx % 32
        tiles = torch.nn.functional.pad(w * sv, (0, pad)).view(n, -1, 32).sum(2)
        all_c = w @ c.abs()
        e = UNIT[dtype] * o.abs()
        e += TIMES * once * torch.sqrt(w ** 2 @ c ** 2) + TIMES * 2.0 ** -29 * largest * torch.sqrt((codes ** 2).sum(0))[None]
        e += TIMES * EPS * D ** 0.5 * spread((w * M) ** 2)
        e += torch.sqrt((w * linear ** 2).sum(1, keepdim=True)) * spread(w)                     # (Cauchy: sum w |v - o| e)
        e += (ctx / 32 + 64) * EPS * (o.abs() + all_c + (w @ mid_v.abs())[:, None])
        e += TIMES * EPS * 8 * torch.sqrt((((bias_v + 2 ** bits) * tiles[:, :, None] + all_c[:, None]) ** 2).sum(1))
        off[:, j] += (e * (1 + UNIT[dtype])).numpy()
    return (out, off, others) if wrong else (out, off)


def edges(ctx, page):
    """Tokens at which a kernel begins or ends something, of a context."""
    at = [0, 1, page - 1, page, 31, 32, 63, 64, 127, 128, 255, 256, 511, 512, 1023, 1024, 2048, ctx // 2, ctx - 32, ctx - 17, ctx - 16, ctx - 2, ctx - 1]
    return sorted({t for t in at if 0 <= t < ctx})


def telling_queries(q, k, past, causal, page, turn, scale):
    """Queries [n][Hq][D] for keys [ctx][H][D], every third row of each kind, the kinds changing places with `turn`: as they are; a row whose softmax is
    about half one token's, at an edge (the row's own newest one first); a row that sees all tokens nearly alike, so that any one is missed."""
    n, Hq, D = q.shape
    ctx, H = k.shape[:2]
    q = q.clone()
    for i in range(n):
        seen = max(0, min(ctx, past + i + 1)) if causal else ctx
        at = edges(seen, page)[::-1]
        for j in range(Hq):
            kind = (i * Hq + j + turn) % 3
            if kind == 1 and at:
                key = k[at[(i * Hq + j) // 3 % len(at)], j * H // Hq].float()
                q[i, j] = (key * ((np.log(seen) + 0.5) / (scale * key.square().sum()))).to(q.dtype)
            if kind == 2:
                q[i, j] *= 2.0 ** -7
    return q
