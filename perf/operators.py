"""The operators of a quantised decoder layer, as measurable cases: their plain form, and the library's.

A case is one pass through one of these, on operands that the caller holds on the GPU:

  product    matrix product in 8-bit integers with a scale for each token and each channel, from codes
  linear     the same layer from 16- or 32-bit activations: the tokens are quantised within the pass
  cache      new keys and values quantised into a paged cache (8 or 4 bits), and read back as the values that the cache now holds
  attention  a batch's new tokens (one each, or a chunk each) against that cache

The definitions that both forms follow, operation by operation in binary32:

  8 bits     s = max|x| / 127, code = rint(x / s) within -127 ... 127 (0 where s is 0); the value of a code is s * code
  4 bits     z = min x, s = max x / 15 - min x / 15, code = rint((x - z) / s) within 0 ... 15 (0 where s is 0); value s * code + z

over a token's channels for the linear layer, and over a token's channels of one head for the cache.  The cache is one buffer of
pages; page p, head h holds `page` tokens: the keys' codes, the values' codes, the keys' scales, the values' scales and, with 4 bits,
the keys' and the values' z.  8-bit codes are stored plus 128.  Keys lie in units of 16 tokens, in a unit in pieces of 16 channels,
[unit][channel / 16][token][channel % 16]; values in words of 4 tokens, [unit][token / 4][channel][token % 4].  4-bit codes lie two
to a byte, the even channel low: [unit][channel / 16][token][8 bytes] and [unit][token / 4][channel / 2][token % 4].
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
LARGEST = {"bytes": 1.5e9, "flops": 1.2e12}


def listed():
    return [
        # one linear layer for one token: latency, and the weights streamed once
        dict(name="linear_one_token", kind="linear", N=1, M=4096, K=4096, dtype="bf16", bias=False),
        # the benchmark's large layer for a small batch of decoded tokens, with a bias
        dict(name="linear_decode_16", kind="linear", N=16, M=8192, K=8192, dtype="f16", bias=True),
        # an odd prompt through a layer of odd size, in 32 bits
        dict(name="product_ragged", kind="product", N=333, M=1537, K=2000, dtype="f32", bias=True),
        # the benchmark's square product: a long prompt, bound by arithmetic
        dict(name="linear_prompt_8192", kind="linear", N=8192, M=8192, K=8192, dtype="bf16", bias=False),
        # a decode step of 32 sequences written to the cache (and read back): latency
        dict(name="cache_step_32", kind="cache", T=32, H=8, D=128, page=16, bits=8, dtype="bf16"),
        # an odd chunk of a prompt, 4 bits
        dict(name="cache_chunk_4bit", kind="cache", T=2049, H=8, D=64, page=64, bits=4, dtype="f16"),
        # many long prompts at once: bound by memory
        dict(name="cache_prompts", kind="cache", T=65536, H=8, D=128, page=64, bits=8, dtype="bf16"),
        # one sequence's next token over a short context: the smallest attention, latency
        dict(name="decode_one_short", kind="attention", B=1, q=1, ctx=1000, Hq=32, Hkv=8, D=128, page=16, bits=8, dtype="bf16", causal=True),
        # a serving batch's next tokens over contexts of all lengths up to 8192, 4 bits
        dict(name="decode_batch_4bit", kind="attention", B=64, q=1, ctx=8192, Hq=32, Hkv=8, D=128, page=64, bits=4, dtype="bf16", causal=True),
        # one sequence's next token over a long context: few rows, work split over the context
        dict(name="decode_one_long", kind="attention", B=1, q=1, ctx=131071, Hq=32, Hkv=8, D=128, page=64, bits=8, dtype="f16", causal=True),
        # a mixed batch: ragged chunks of a few new tokens to 300 over ragged contexts, narrow heads, each query head with its own keys
        dict(name="chunks_ragged", kind="attention", B=12, q=300, ctx=3000, Hq=16, Hkv=16, D=64, page=16, bits=4, dtype="f16", causal=True),
        # a chunk of a long prompt: bound by arithmetic
        dict(name="chunk_long", kind="attention", B=1, q=2048, ctx=32768, Hq=32, Hkv=8, D=128, page=64, bits=8, dtype="bf16", causal=True),
    ]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: a quarter of the layers' sizes are any integers, the others multiples of 16."""
    while True:
        family = rng.choice(("product", "linear", "linear", "cache", "cache", "decode", "decode", "chunk", "chunk"))
        if family in ("product", "linear"):
            size = (lambda lo, hi: _log(rng, lo, hi)) if rng.random() < 0.25 else (lambda lo, hi: 16 * _log(rng, lo / 16, hi / 16))
            case = dict(kind=family, N=_log(rng, 1, 8192), M=size(256, 16384), K=size(256, 16384), dtype=rng.choice(("bf16", "f16", "f32")),
                        bias=rng.random() < 0.5)
        elif family == "cache":
            case = dict(kind="cache", T=_log(rng, 1, 65536), H=rng.choice((1, 2, 4, 8, 12, 32)), D=rng.choice((64, 128)),
                        page=rng.choice((16, 32, 48, 64, 128)), bits=rng.choice((8, 4)), dtype=rng.choice(("bf16", "f16", "f32")))
        else:
            heads = rng.choice((1, 2, 4, 8, 16))
            case = dict(kind="attention", B=_log(rng, 1, 64), q=1 if family == "decode" else _log(rng, 2, 2048), ctx=_log(rng, 16, 131072),
                        Hq=heads * rng.choice((1, 2, 4, 7, 8)), Hkv=heads, D=rng.choice((64, 128)), page=rng.choice((16, 32, 48, 64, 128)),
                        bits=rng.choice((8, 4)), dtype=rng.choice(("bf16", "f16")), causal=rng.random() < 0.85)
            if case["q"] > case["ctx"] or case["Hq"] > 64 or not 1e6 < _scores(case) < 2.2e9 or case["B"] * case["ctx"] * heads * case["D"] > 6e8:
                continue
        w = work(case)
        if w["bytes"] <= LARGEST["bytes"] and 1e6 < w["flops"] <= LARGEST["flops"]:
            return case


def _lengths(case):
    """The new tokens and the contexts (these included) of a batch: spread evenly up to the largest, in no order."""
    B, q, ctx = case["B"], case["q"], case["ctx"]
    order = [(5 * b + 2) % B if math.gcd(5, B) == 1 else B - 1 - b for b in range(B)]
    new = [max(1, (q * (order[B - 1 - b] + 1)) // B) for b in range(B)]
    return new, [max(new[b], (ctx * (order[b] + 1)) // B) for b in range(B)]


def _scores(case):
    """The scores of a batch with every sequence as long as the longest."""
    return case["B"] * case["q"] * case["ctx"] * case["Hq"]


def _head_bytes(case):
    """What a page holds for one head."""
    return case["page"] * (2 * case["D"] * case["bits"] // 8 + (8 if case["bits"] == 8 else 16))


def work(case):
    if case["kind"] in ("product", "linear"):
        N, M, K, b = case["N"], case["M"], case["K"], SIZE[case["dtype"]]
        x = N * K + 4 * N if case["kind"] == "product" else N * K * b
        return {"bytes": x + M * K + 4 * M + N * M * b + (4 * M if case["bias"] else 0), "flops": 2 * N * M * K}
    token = 2 * case["D"] * case["bits"] / 8 + (8 if case["bits"] == 8 else 16)       # a head's keys, values and scales in the cache
    if case["kind"] == "cache":
        values = 2 * case["T"] * case["H"] * case["D"]
        return {"bytes": 2 * values * SIZE[case["dtype"]] + 2 * case["T"] * case["H"] * token + 4 * case["T"], "flops": 8 * values}
    new, ctx = _lengths(case)
    rows = sum(n * c - (n * (n - 1) // 2 if case["causal"] else 0) for n, c in zip(new, ctx))
    return {"bytes": sum(ctx) * case["Hkv"] * token + 2 * sum(new) * case["Hq"] * case["D"] * SIZE[case["dtype"]],
            "flops": 4 * rows * case["Hq"] * case["D"]}


# ---- the plain form ---------------------------------------------------------------------------------------------------


def _quantize8(x):
    """[..., K] -> codes (as float32) and scale [..., 1].  (Divisors are tensors: by a number, torch multiplies by its inverse.)"""
    s = x.abs().amax(-1, keepdim=True) / torch.full((), 127.0, device=x.device)
    return torch.where(s > 0, torch.round(x / s).clamp(-127, 127), torch.zeros_like(x)), s


def _quantize4(x):
    """[..., K] -> codes (as float32), scale and z [..., 1]."""
    fifteen = torch.full((), 15.0, device=x.device)
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = hi / fifteen - lo / fifteen
    return torch.where(s > 0, torch.round((x - lo) / s).clamp(0, 15), torch.zeros_like(x)), s, lo


def _layer(codes, scale_n, W, scale_m, bias, dtype):
    y = torch.matmul(codes, W.float().t()) * scale_m * scale_n
    return (y if bias is None else y + bias).to(dtype)


def _places(case, slots):
    """Where the tokens of `slots` lie: the first byte of every (token, head)'s page and head, and the token's place in the page."""
    head = _head_bytes(case)
    base = (slots // case["page"]).long() * (head * case["H"])
    return base[:, None] + head * torch.arange(case["H"], device=slots.device), (slots % case["page"]).long()


def _code_bytes(case, base, t, values):
    """The byte of every code [T][H][D] (with 4 bits, of every two [T][H][D / 2])."""
    D, per = case["D"], case["bits"]
    step = D * per // 8                                       # bytes of a token
    c = torch.arange(step, device=t.device)
    if values:
        at = ((t // 4) * (4 * step) + t % 4)[:, None] + c * 4
    else:
        piece = 2 * per                                       # bytes of a token's 16 channels
        at = ((t // 16) * (16 * step) + (t % 16) * piece)[:, None] + (c // piece) * (16 * piece) + c % piece
    return base[:, :, None] + at[:, None, :] + (case["page"] * step if values else 0)


def _word_places(case, base, t, which):
    """The 32-bit word of every (token, head)'s number `which`: key scale, value scale, key z, value z."""
    return (base + 2 * case["page"] * case["D"] * case["bits"] // 8 + 4 * (which * case["page"] + t)[:, None]) // 4


def _plain_write(case, cache, slots, k, v):
    base, t = _places(case, slots)
    flat, words = cache.view(-1), cache.view(-1).view(torch.float32)
    for i, x in enumerate((k.float(), v.float())):
        at = _code_bytes(case, base, t, i == 1)
        if case["bits"] == 8:
            codes, s = _quantize8(x)
            flat[at] = (codes + 128).to(torch.uint8)
        else:
            codes, s, z = _quantize4(x)
            codes = codes.to(torch.uint8)
            flat[at] = codes[..., 0::2] | (codes[..., 1::2] << 4)
            words[_word_places(case, base, t, 2 + i)] = z[..., 0]
        words[_word_places(case, base, t, i)] = s[..., 0]


def _plain_read(case, cache, slots, dtype):
    base, t = _places(case, slots)
    flat, words, out = cache.view(-1), cache.view(-1).view(torch.float32), []
    for i in range(2):
        codes, s = flat[_code_bytes(case, base, t, i == 1)], words[_word_places(case, base, t, i)][..., None]
        if case["bits"] == 8:
            x = (codes.float() - 128) * s
        else:
            z = words[_word_places(case, base, t, 2 + i)][..., None]
            x = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() * s + z
        out.append(x.to(dtype))
    return out


def _plain_context(case, cache, table):
    """The keys and values of every sequence's table, [B][Hkv][tokens][D], in 32 bits."""
    B, pages = table.shape
    H, D, page, step = case["Hkv"], case["D"], case["page"], case["D"] * case["bits"] // 8
    held = cache.view(-1, H, _head_bytes(case))[table.clamp_min(0).long()].transpose(1, 2)        # [B][H][pages][bytes]
    words = held[..., 2 * page * step:].contiguous().view(torch.float32).view(B, H, pages, -1, page)
    out = []
    for i in range(2):
        codes = held[..., i * page * step:(i + 1) * page * step]
        if i == 0:
            codes = codes.reshape(B, H, pages, page // 16, D // 16, 16, 2 * case["bits"]).transpose(4, 5)
        else:
            codes = codes.reshape(B, H, pages, page // 4, step, 4).transpose(4, 5)
        codes = codes.reshape(B, H, pages * page, step)
        s = words[:, :, :, i].reshape(B, H, pages * page, 1)
        if case["bits"] == 8:
            out.append((codes.float() - 128) * s)
        else:
            z = words[:, :, :, 2 + i].reshape(B, H, pages * page, 1)
            out.append(torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() * s + z)
    return out


def _plain_attention(state):
    case, q = state["case"], state["q"]
    B, Hq, H, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    K, V = _plain_context(case, state["cache"], state["table"])
    start, ctx = state["q_start"].long(), state["ctx_len"].long()
    new = start[1:] - start[:-1]
    i, p = torch.arange(state["max_q"], device=q.device), torch.arange(K.shape[2], device=q.device)
    at = (start[:-1, None] + i).clamp_max(q.shape[0] - 1)                                          # [B][max_q]
    rows = q.float()[at].view(B, -1, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)    # [B][H][group * max_q][D]
    last = ctx[:, None] - new[:, None] + i if state["causal"] else (ctx[:, None] - 1).expand(B, i.numel())
    seen = (p <= last[:, :, None]) & (p < ctx[:, None, None])                                      # [B][max_q][tokens]
    s = torch.matmul(rows, K.transpose(2, 3)).view(B, H, Hq // H, i.numel(), -1).mul_(state["scale"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, H, -1, e.shape[-1]), V).view(B, H, Hq // H, i.numel(), D) / total.clamp_min(1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, i.numel(), Hq, D)
    out = torch.zeros_like(q)
    there = i < new[:, None]
    out[at[there]] = o[there].to(q.dtype)
    return out


# ---- cases ------------------------------------------------------------------------------------------------------------


def _layer_inputs(case, gen):
    """Activations of a few large channels among many, as between a network's layers; weights of their own scale per channel."""
    N, M, K, dtype = case["N"], case["M"], case["K"], DTYPES[case["dtype"]]
    x = torch.randn(N, K, device="cuda", generator=gen) * (1 + 9 * (torch.rand(K, device="cuda", generator=gen) < 0.01))
    W = (torch.randn(M, K, device="cuda", generator=gen) * 32).round_().clamp_(-127, 127).to(torch.int8)
    scale_m = (0.5 + torch.rand(M, device="cuda", generator=gen)) / (32 * math.sqrt(K))
    return x.to(dtype), W, scale_m, torch.randn(M, device="cuda", generator=gen) if case["bias"] else None


def _kv(case, gen, count, heads):
    """Keys with some channels away from zero, and values; [tokens][heads][D]."""
    k = torch.randn(count, heads, case["D"], device="cuda", generator=gen)
    k += 3 * torch.randn(heads, case["D"], device="cuda", generator=gen) * (torch.rand(heads, case["D"], device="cuda", generator=gen) < 0.1)
    return k.to(DTYPES[case["dtype"]]), torch.randn(count, heads, case["D"], device="cuda", generator=gen).to(DTYPES[case["dtype"]])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    state = {"case": case, "kind": case["kind"], "dtype": dtype}
    if case["kind"] in ("product", "linear"):
        x, W, scale_m, bias = _layer_inputs(case, gen)
        state.update(W=W, scale_m=scale_m, bias=bias, out=torch.empty(case["N"], case["M"], dtype=dtype, device="cuda"))
        if case["kind"] == "linear":
            pitch = -(-case["K"] // 16) * 16                     # the quantised tokens' buffer: rows of whole 16 bytes, then the scales
            state.update(x=x, work=torch.empty(case["N"] * (pitch + 4), dtype=torch.uint8, device="cuda"))
        else:
            codes, s = _quantize8(x.float())
            state.update(codes=codes.to(torch.int8), scale_n=s[:, 0].contiguous())
        return state
    if case["kind"] == "cache":
        T, H, page = case["T"], case["H"], case["page"]
        pages = -(-T // page) + 3
        k, v = _kv(case, gen, T, H)
        # sequences of whole chunks in scattered pages; with few tokens, each in a page of its own (a decode step's)
        order = torch.randperm(pages, device="cuda", generator=gen)
        if T <= 64:
            pages = T + 3
            slots = torch.randperm(pages, device="cuda", generator=gen)[:T] * page + torch.randint(0, page, (T,), device="cuda", generator=gen)
        else:
            t = torch.arange(T, device="cuda") + page // 3       # (a chunk begins inside a page)
            slots = order[t // page] * page + t % page
        state.update(k=k, v=v, slots=slots.to(torch.int32), cache=torch.zeros(pages * H * _head_bytes(case), dtype=torch.uint8, device="cuda"),
                     pages=pages, k_out=torch.empty_like(k), v_out=torch.empty_like(v))
        return state
    B, H, Hq, D, page = case["B"], case["Hkv"], case["Hq"], case["D"], case["page"]
    new, ctx = _lengths(case)
    need = [-(-c // page) for c in ctx]
    order = torch.randperm(sum(need) + 2, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    there = torch.arange(max(need), device="cuda") < torch.tensor(need, device="cuda")[:, None]
    table[there] = order[:sum(need)]
    cache = torch.zeros((sum(need) + 2) * H * _head_bytes(case), dtype=torch.uint8, device="cuda")
    at = dict(case, H=H)
    for first in range(0, sum(need) * page, 1 << 16):            # (a prompt's chunks, so that the indices stay small)
        slots = torch.arange(first, min(first + (1 << 16), sum(need) * page), device="cuda")
        _plain_write(at, cache, order[slots // page].long() * page + slots % page, *_kv(case, gen, slots.numel(), H))
    start = [sum(new[:b]) for b in range(B + 1)]
    scale = D ** -0.5
    state.update(cache=cache, pages=sum(need) + 2, table=table, q=(2 * torch.randn(start[-1], Hq, D, device="cuda", generator=gen)).to(dtype),
                 q_start=torch.tensor(start, dtype=torch.int32, device="cuda"), ctx_len=torch.tensor(ctx, dtype=torch.int32, device="cuda"),
                 max_q=max(new), max_ctx=max(ctx), scale=scale, causal=case["causal"])
    state["out"] = torch.empty_like(state["q"])
    return state


def _desc(case, pages, heads):
    from paper_2304_09049_amd import binding as dg
    return dg.cache_desc(pages, case["page"], heads, case["D"], case["bits"])


def run(state):
    kind, case = state["kind"], state["case"]
    if not own:
        if kind == "product":
            return _layer(state["codes"].float(), state["scale_n"][:, None], state["W"], state["scale_m"], state["bias"], state["dtype"])
        if kind == "linear":
            codes, s = _quantize8(state["x"].float())
            return _layer(codes, s, state["W"], state["scale_m"], state["bias"], state["dtype"])
        if kind == "cache":
            _plain_write(case, state["cache"], state["slots"], state["k"], state["v"])
            return _plain_read(case, state["cache"], state["slots"], state["dtype"])
        return _plain_attention(state)
    from paper_2304_09049_amd import binding as dg
    if kind == "product":
        return dg.dg_gemm_i8(state["W"], state["codes"], state["scale_m"], state["scale_n"], bias=state["bias"], out=state["out"])
    if kind == "linear":
        return dg.dg_linear_i8(state["W"], state["x"], state["scale_m"], bias=state["bias"], work=state["work"], out=state["out"])
    if "desc" not in state:                                      # (a program builds it once, beside its cache)
        heads = case["H"] if kind == "cache" else case["Hkv"]
        state["desc"] = _desc(case, state["pages"], heads)
        if kind == "attention":
            need = dg.dg_paged_attention_work_bytes(state["desc"], case["B"], case["Hq"], state["max_q"], state["max_ctx"])
            state["work"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    if kind == "cache":
        dg.dg_cache_write(state["desc"], state["cache"], state["k"], state["v"], state["slots"])
        return dg.dg_cache_read(state["desc"], state["cache"], state["slots"], k_out=state["k_out"], v_out=state["v_out"])
    return dg.dg_paged_attention(state["desc"], state["cache"], state["q"], state["q_start"], state["ctx_len"], state["table"], state["max_q"],
                                 state["max_ctx"], scale=state["scale"], causal=state["causal"], out=state["out"], work=state["work"])


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _codes_by_definition(x, bits):
    """What the stored codes of x [..., K] (64 bits) stand for.  A quotient of binary32 numbers taken in 64 bits and rounded to 32 is the
    correctly rounded one."""
    f32 = lambda y: y.float().double()  # noqa: E731
    if bits == 8:
        s = f32(x.abs().amax(-1, keepdim=True) / 127)
        return f32(x / s.where(s > 0, torch.ones_like(s))).round().clamp(-127, 127) * (s > 0), s, torch.zeros_like(s)
    lo = x.amin(-1, keepdim=True)
    s = f32(f32(x.amax(-1, keepdim=True) / 15) - f32(lo / 15))
    return f32(f32(x - lo) / s.where(s > 0, torch.ones_like(s))).round().clamp(0, 15) * (s > 0), s, lo


def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] in ("product", "linear"):
        x, W, scale_m, bias = _layer_inputs(case, gen)
        codes, s, _ = _codes_by_definition(x.double(), 8)
        y = torch.matmul(codes, W.double().t()) * scale_m.double() * s
        return y if bias is None else y + bias.double()
    if case["kind"] == "cache":
        out = []
        for x in _kv(case, gen, case["T"], case["H"]):
            codes, s, z = _codes_by_definition(x.double(), case["bits"])
            out.append(codes * s + z)
        return out
    state = prepare(case, seed)
    Hq, H, D = case["Hq"], case["Hkv"], case["D"]
    new, ctx = _lengths(case)
    out = torch.zeros(sum(new), Hq, D, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, c) in enumerate(zip(new, ctx)):
        K, V = _context_by_definition(case, state["cache"], state["table"][b].tolist(), c)
        for h in range(Hq):
            for lo in range(0, n, 512):
                hi = min(n, lo + 512)
                s = torch.matmul(state["q"][first + lo:first + hi, h].double(), K[h * H // Hq].t()) * state["scale"]
                if case["causal"]:
                    s += torch.where(torch.arange(c, device="cuda") <= c - n + torch.arange(lo, hi, device="cuda")[:, None], 0.0, -math.inf)
                out[first + lo:first + hi, h] = torch.matmul(torch.softmax(s, -1), V[h * H // Hq])
        first += n
    return out


def _context_by_definition(case, cache, table, tokens):
    """One sequence's keys and values [Hkv][tokens][D] in 64 bits, by each code's place as the layout states it."""
    H, D, page, bits = case["Hkv"], case["D"], case["page"], case["bits"]
    head, step = _head_bytes(case), D * bits // 8
    p = torch.arange(tokens, device="cuda")
    t, d, h = (p % page)[None, :, None], torch.arange(D, device="cuda")[None, None, :], torch.arange(H, device="cuda")[:, None, None]
    base = (torch.tensor(table, device="cuda")[p // page][None, :, None] * H + h) * head
    if bits == 8:
        places = ((t // 16) * 16 * D + (d // 16) * 256 + (t % 16) * 16 + d % 16, page * step + (t // 4) * 4 * D + d * 4 + t % 4)
    else:
        places = ((t // 16) * 8 * D + (d // 16) * 128 + (t % 16) * 8 + d % 16 // 2, page * step + (t // 4) * 2 * D + (d // 2) * 4 + t % 4)
    out = []
    for i, place in enumerate(places):
        byte = cache[base + place].long()
        words = [cache.view(torch.float32)[(base + 2 * page * step + 4 * (j * page + t)) // 4].double() for j in ((i,) if bits == 8 else (i, 2 + i))]
        out.append((byte - 128) * words[0] if bits == 8 else torch.where(d % 2 == 1, byte >> 4, byte & 15) * words[0] + words[1])
    return out
