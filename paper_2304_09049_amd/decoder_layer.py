"""A quantised decoder layer out of this library's calls: attention with 8-bit projections over a cache in 8 or 4 bits, and a
feed-forward part by 2-bit table lookup, or of experts in microscaled 4-bit floating point.

The layer serves a batch of sequences whose cached keys and values lie in pages of one buffer.  A step takes any number of new
tokens a sequence -- a prompt, a chunk of one, one decoded token each, mixed -- as the same six calls:

    dg_linear_i8          queries, keys and values of the new tokens (8-bit weights, tokens quantised on the way)
    dg_cache_write        keys and values quantised into their slots
    dg_paged_attention    the new tokens against everything cached
    dg_linear_i8          the attention's output projection
    dg_quantize_pack_activations, dg_gemm_lut   the feed-forward product on 2-bit codes, to float32 with a scale per channel

``ExpertsLayer`` has another feed-forward part, of weights in blocks of 32 with a power of two each (dg_quantize_mx4):

    dg_route_tokens       which experts each token goes to, with what weights
    dg_experts_mx4        those experts' gated feed-forward, added up
    dg_linear_mx4         twice: the gated feed-forward that every token passes

``python -m paper_2304_09049_amd.decoder_layer`` runs a batch through prompts in chunks and some decoded tokens, and prints how far
the attention part is from float32 with nothing quantised (with experts, the feed-forward part too), and what a step of decoded tokens takes with its host work.
"""
from __future__ import annotations

import torch

from . import binding as dg


class PagedSequences:
    """Which pages of a cache belong to which sequence; pages are handed out as tokens come."""

    def __init__(self, desc: dg.CacheDesc, count: int, device):
        self.desc, self.device = desc, device
        self.cache = torch.zeros(dg.dg_cache_bytes(desc), dtype=torch.uint8, device=device)
        self.pages = [[] for _ in range(count)]
        self.lengths = [0] * count
        self.free = list(range(desc.pages))[::-1]

    def extend(self, new):
        """Room for new[b] more tokens of each sequence -> (slots of the new tokens, q_start, ctx_len, table) on the device.  Nothing changes where
        the pages do not suffice (MemoryError)."""
        if len(new) != len(self.pages) or min(new, default=0) < 0:
            raise ValueError(f"new tokens {list(new)} for {len(self.pages)} sequences")
        need = sum(-(-(length + n) // self.desc.page_size) - len(pages) for length, n, pages in zip(self.lengths, new, self.pages))
        if need > len(self.free):
            raise MemoryError(f"{need} more pages are needed, {len(self.free)} of {self.desc.pages} are free")
        slots, starts = [], [0]
        for b, n in enumerate(new):
            while len(self.pages[b]) * self.desc.page_size < self.lengths[b] + n:
                self.pages[b].append(self.free.pop())
            for t in range(self.lengths[b], self.lengths[b] + n):
                slots.append(self.pages[b][t // self.desc.page_size] * self.desc.page_size + t % self.desc.page_size)
            self.lengths[b] += n
            starts.append(starts[-1] + n)
        width = max(1, max(len(p) for p in self.pages))
        table = [p + [-1] * (width - len(p)) for p in self.pages]
        return tuple(torch.tensor(x, dtype=torch.int32, device=self.device) for x in (slots, starts, self.lengths, table))


class DecoderLayer:
    """Weights are float32 [out][in] tensors on the device; the layer keeps their codes.  The feed-forward weight is quantised to four
    levels a channel, its input to four multiples of ``ff_step``."""

    LEVELS_W, LEVELS_A = (-2, -1, 0, 1), (-2, -1, 0, 1)

    def __init__(self, w_qkv, w_out, w_ff, heads: int, kv_heads: int, dim: int, ff_step: float = 1.0):
        self.take_attention(w_qkv, w_out, heads, kv_heads, dim)
        self.ff_step, self.ff_shape = ff_step, w_ff.shape
        codes, self.ff_scale = self.two_bits(w_ff)
        self.ff = dg.dg_pack_weights(codes, *self.ff_shape)
        self.lut = dg.dg_build_lut(self.LEVELS_W, self.LEVELS_A)

    def take_attention(self, w_qkv, w_out, heads, kv_heads, dim):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.qkv, self.qkv_scale = dg.dg_quantize_tokens(w_qkv)
        self.out, self.out_scale = dg.dg_quantize_tokens(w_out)

    @staticmethod
    def two_bits(w):
        """Codes [out][in] and scales [out] of float32 weights: code + level 0 -> -2, so that the four levels -2, -1, 0, 1 times the scale cover a channel; a
        channel of zeros has level 0 and scale 0."""
        scale = w.abs().amax(1) / 2
        codes = torch.clamp(torch.round(w / torch.where(scale > 0, scale, 1.0)[:, None]), -2, 1) + 2
        return codes.to(torch.uint8).contiguous(), scale

    def step(self, x, sequences: PagedSequences, new):
        """x: [sum(new)][hidden] of the new tokens, sequence after sequence, float16 or bfloat16 -> the layer's output, the same shape."""
        h = self.attend(x, sequences, new)
        return h + self.feed_forward(h)

    def attend(self, x, sequences: PagedSequences, new):
        slots, q_start, ctx_len, table = sequences.extend(new)
        tokens = x.shape[0]
        qkv = dg.dg_linear_i8(self.qkv, x, self.qkv_scale).view(tokens, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)          # (views: heads and tokens keep their strides)
        dg.dg_cache_write(sequences.desc, sequences.cache, k, v, slots)
        attended = dg.dg_paged_attention(sequences.desc, sequences.cache, q, q_start, ctx_len, table, max(new), max(sequences.lengths))
        return x + dg.dg_linear_i8(self.out, attended.view(tokens, self.heads * self.dim), self.out_scale)

    def feed_forward(self, h):
        M, K = self.ff_shape
        if not h.shape[0]:                                        # (the calls around the tables take one row at least)
            return torch.empty(0, M, dtype=h.dtype, device=h.device)
        packed = dg.dg_quantize_pack_activations(h.float(), h.shape[0], K, 1 / self.ff_step, 0.0, -2)
        y = torch.empty(h.shape[0], M, dtype=torch.float32, device=h.device)
        dg.dg_gemm_lut(self.lut, self.ff, packed, M, h.shape[0], K, out=y, scale=self.ff_scale * self.ff_step, strides=(1, M))
        return y.to(h.dtype)


class ExpertsLayer(DecoderLayer):
    """A layer whose feed-forward part is ``top`` of some experts a token and one that every token passes.  router: [experts][hidden] (kept in float32);
    up: [experts][2 * inner][hidden], the gates first; down: [experts][hidden][inner]; shared_up, shared_down: the same without experts, of an inner size of
    their own.  bias: [experts] float32 added to what experts are chosen by."""

    def __init__(self, w_qkv, w_out, router, up, down, shared_up, shared_down, heads: int, kv_heads: int, dim: int, top: int, mode="softmax", bias=None):
        experts, hidden = router.shape
        inner = down.shape[2]
        if up.shape != (experts, 2 * inner, hidden) or down.shape != (experts, hidden, inner) or not 0 < top <= experts:
            raise ValueError(f"{top} of {experts} experts on {hidden} with up {list(up.shape)} and down {list(down.shape)}")
        if shared_up.shape != (2 * shared_down.shape[1], hidden) or shared_down.shape[0] != hidden:
            raise ValueError(f"shared up {list(shared_up.shape)} and down {list(shared_down.shape)} on {hidden}")
        self.take_attention(w_qkv, w_out, heads, kv_heads, dim)
        self.router, self.top, self.mode, self.bias = router.float(), top, mode, bias
        self.experts = [t.unflatten(0, w.shape[:2]) for w in (up, down) for t in dg.dg_quantize_mx4(w.flatten(0, 1))]
        self.shared_up, self.shared_down = dg.dg_quantize_mx4(shared_up), dg.dg_quantize_mx4(shared_down)

    def feed_forward(self, h):
        ids, weights = dg.dg_route_tokens(h, self.router, self.top, self.mode, self.bias)
        chosen = dg.dg_experts_mx4(*self.experts, h, ids, weights)
        gate, other = dg.dg_linear_mx4(*self.shared_up, h).chunk(2, 1)
        return chosen + dg.dg_linear_mx4(*self.shared_down, torch.nn.functional.silu(gate) * other)


def plain_experts_part(h, router, up, down, shared_up, shared_down, top):
    """What ``ExpertsLayer.feed_forward`` approximates (mode "softmax", no bias), in float32, nothing quantised: every expert on all tokens."""
    h, weights = h.float(), torch.zeros(h.shape[0], router.shape[0], device=h.device)
    most, ids = (h @ router.t()).topk(top)
    weights.scatter_(1, ids, torch.softmax(most, 1))
    gated = lambda x, up, down: (torch.nn.functional.silu(x @ up[:down.shape[1]].t()) * (x @ up[down.shape[1]:].t())) @ down.t()  # noqa: E731
    return gated(h, shared_up, shared_down) + sum(weights[:, e, None] * gated(h, up[e], down[e]) for e in range(router.shape[0]))


def plain_attention_part(x, w_qkv, w_out, heads, kv_heads, dim):
    """What ``DecoderLayer.attend`` approximates: one sequence from its first token on, in float32, nothing quantised."""
    n = x.shape[0]
    q, k, v = (x.float() @ w_qkv.t()).view(n, -1, dim).split((heads, kv_heads, kv_heads), 1)
    k, v = (t.repeat_interleave(heads // kv_heads, 1) for t in (k, v))
    s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * dim ** -0.5
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), float("-inf"))
    return x.float() + torch.matmul(torch.softmax(s, -1), v.transpose(0, 1)).transpose(0, 1).reshape(n, -1) @ w_out.t()


def main():
    import time
    device, gen = torch.device("cuda:0"), torch.Generator(device="cuda").manual_seed(0)
    hidden, heads, kv_heads, dim, prompt, decoded = 1024, 16, 4, 64, 300, 20
    w_qkv, w_out, w_ff = (torch.randn(n, m, device=device, generator=gen) * m ** -0.5
                          for n, m in (((heads + 2 * kv_heads) * dim, hidden), (hidden, heads * dim), (hidden, hidden)))
    experts, inner, top = 16, 512, 4
    parts = [torch.randn(*size, device=device, generator=gen) * size[-1] ** -0.5
             for size in ((experts, hidden), (experts, 2 * inner, hidden), (experts, hidden, inner), (2 * inner, hidden), (hidden, inner))]
    for kind, bits in (("tables", 8), ("tables", 4), ("experts", 8)):
        if kind == "tables":
            layer = DecoderLayer(w_qkv, w_out, w_ff, heads, kv_heads, dim)
        else:
            layer = ExpertsLayer(w_qkv, w_out, *parts, heads, kv_heads, dim, top)
        sequences = PagedSequences(dg.cache_desc(64, 16, kv_heads, dim, bits), 3, device)
        x = torch.randn(3, prompt + decoded, hidden, device=device, generator=gen).bfloat16()
        done, at, took = [[], [], []], [0, 0, 0], []
        for new in [(100, 300, 1), (200, 1, 150), (1, 1, 149)] + [(1, 1, 1)] * (decoded - 3):
            batch = torch.cat([x[b, at[b]:at[b] + n] for b, n in enumerate(new)])
            torch.cuda.synchronize()
            start = time.perf_counter()
            h = layer.attend(batch, sequences, new)
            y = h + layer.feed_forward(h)
            torch.cuda.synchronize()
            took.append(time.perf_counter() - start)
            assert y.isfinite().all()
            for b, part in enumerate(h.split(new)):
                done[b].append(part)
                at[b] += new[b]
        off = 0.0
        for b in range(3):
            want = plain_attention_part(x[b, :at[b]], w_qkv, w_out, heads, kv_heads, dim) - x[b, :at[b]].float()
            got = torch.cat(done[b]).float() - x[b, :at[b]].float()
            off = max(off, ((got - want).norm() / want.norm()).item())
        told = ""
        if kind == "experts":
            h = torch.cat([t for parts_done in done for t in parts_done])
            want = plain_experts_part(h, *parts, top)
            told = f"feed-forward by {((layer.feed_forward(h).float() - want).norm() / want.norm()).item():.3f}, "
        print(f"{kind}, {bits}-bit cache: sequences of {at} tokens, attention off by {off:.3f} of its norm, {told}"
              f"a step of decoded tokens {sorted(took)[len(took) // 2] * 1e6:.0f} us")


if __name__ == "__main__":
    main()
