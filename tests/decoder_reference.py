"""Plain implementations of a quantised decoder layer's operators in numpy, for the tests: the quantisers operation by operation in
binary32, the cache's layout from the formulas that the header states, products in whole numbers, attention in 64 bits."""
import numpy as np

f32 = np.float32


def quantize8(x):
    """float32 [..., K] -> int8 codes, float32 scales [...]."""
    x = np.asarray(x, f32)
    with np.errstate(all="ignore"):
        most = np.abs(x).max(-1)
        s = np.where(np.isfinite(x).all(-1), most / f32(127), f32(np.nan)).astype(f32)
        c = np.clip(np.rint(x / s[..., None]), -127, 127)
    return np.where(s[..., None] > 0, c, 0).astype(np.int8), s


def quantize4(x):
    """float32 [..., K] -> uint8 codes, float32 scales and z [...]."""
    x = np.asarray(x, f32)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        s = np.where(np.isfinite(x).all(-1), hi / f32(15) - lo / f32(15), f32(np.nan)).astype(f32)
        c = np.clip(np.rint((x - lo[..., None]) / s[..., None]), 0, 15)
    return np.where(s[..., None] > 0, c, 0).astype(np.uint8), s, lo.astype(f32)


def product(W, A, scale_m, scale_n, bias=None):
    """float32 [N][M] of int8 W [M][K] and A [N][K], before the rounding to the output's type."""
    sums = A.astype(np.float64) @ W.astype(np.float64).T            # (whole numbers below 2^53)
    with np.errstate(all="ignore"):
        y = sums.astype(f32) * scale_m[None, :] * scale_n[:, None]
        return y if bias is None else y + bias[None, :]


class Cache:
    """A paged cache as bytes, by the header's formulas."""

    def __init__(self, pages, page_size, heads, dim, bits, fill=0):
        self.pages, self.page, self.heads, self.dim, self.bits = pages, page_size, heads, dim, bits
        self.part = page_size * dim * bits // 8
        self.head = 2 * self.part + page_size * (8 if bits == 8 else 16)
        self.bytes = np.full(pages * heads * self.head, fill, np.uint8)

    def _places(self, t):
        b, d = self.bits, np.arange(0, self.dim, 8 // self.bits)
        return ((t // 16) * 2 * b * self.dim + (d // 16) * 32 * b + (t % 16) * 2 * b + (d % 16) * b // 8,
                self.part + (t // 4) * (b * self.dim // 2) + (d * b // 8) * 4 + t % 4)

    def _number(self, at, t, which):
        start = at + 2 * self.part + 4 * (which * self.page + t)
        return self.bytes[start:start + 4]

    def write(self, slots, k, v):
        for i, slot in enumerate(slots):
            if not 0 <= slot < self.pages * self.page:
                continue
            page, t = divmod(int(slot), self.page)
            for h in range(self.heads):
                at = (page * self.heads + h) * self.head
                for which, (x, place) in enumerate(zip((k[i, h], v[i, h]), self._places(t))):
                    if self.bits == 8:
                        c, s = quantize8(x)
                        self.bytes[at + place] = (c.astype(np.int32) + 128).astype(np.uint8)
                    else:
                        c, s, z = quantize4(x)
                        self.bytes[at + place] = c[0::2] | c[1::2] << 4
                        self._number(at, t, 2 + which)[:] = np.frombuffer(z.tobytes(), np.uint8)
                    self._number(at, t, which)[:] = np.frombuffer(s.tobytes(), np.uint8)

    def read(self, slots):
        """float32 keys and values [T][heads][dim], before the rounding to the output's type."""
        out = np.zeros((2, len(slots), self.heads, self.dim), f32)
        for i, slot in enumerate(slots):
            if not 0 <= slot < self.pages * self.page:
                continue
            page, t = divmod(int(slot), self.page)
            for h in range(self.heads):
                at = (page * self.heads + h) * self.head
                for which, place in enumerate(self._places(t)):
                    c, s = self.bytes[at + place], self._number(at, t, which).copy().view(f32)[0]
                    if self.bits == 8:
                        out[which, i, h] = (c.astype(np.int32) - 128).astype(f32) * s
                    else:
                        z = self._number(at, t, 2 + which).copy().view(f32)[0]
                        out[which, i, h] = np.stack((c & 15, c >> 4), -1).reshape(-1).astype(f32) * s + z
        return out[0], out[1]


def attention(q, k, v, past, scale, causal, unit):
    """One sequence in 64 bits: q [n][Hq][D]; k, v [ctx][H][D]; new token i sees p <= past + i.  Returns the outputs, and how far the
    library's may be from them: `unit` is the output type's unit roundoff.

    The bound, per output element, with A = sum_p softmax_p |v_p|: a weight is rounded once to binary16 (2^-11), and with it go the errors of
    the score's exponential -- twice the score's own error, a binary32 sum of D products and a few factors ((D + 8) 2^-24 of the sum of its terms'
    magnitudes), and 2^-20 for the exponential -- and those of sums over the context (ctx 2^-24 of A, twice: weights and outputs).  Then the output's
    own rounding.  4-bit values are s c + z: their parts' magnitudes are counted in A apart (at most four times |v| + |z| is taken)."""
    n, Hq, D = q.shape
    ctx, H = k.shape[:2]
    out, off = np.zeros((n, Hq, D)), np.full((n, Hq, D), 1e-30)      # (rows that see nothing: 0)
    for i in range(n):
        seen = max(0, min(ctx, past + i + 1)) if causal else ctx
        if seen == 0:
            continue
        for j in range(Hq):
            kk, vv = k[:seen, j * H // Hq].astype(np.float64), v[:seen, j * H // Hq].astype(np.float64)
            s = scale * (kk @ q[i, j].astype(np.float64))
            w = np.exp(s - s.max())
            w /= w.sum()
            reach = scale * (np.abs(kk).max(1) * np.abs(q[i, j]).sum()).max()
            part = w @ (4 * np.abs(vv).max(1))
            out[i, j] = w @ vv
            e = 2.0 ** -11 + 2 * ((D + 8) * 2.0 ** -24 * 4 * reach + 2.0 ** -20) + 2 * seen * 2.0 ** -24
            off[i, j] = part * e + unit * np.abs(out[i, j]) + 1e-30
    return out, off
