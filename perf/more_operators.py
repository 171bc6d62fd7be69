"""Layers in microscaled 4-bit floating point and layers of experts, as measurable cases: their plain form, and the library's.

A case is one pass through one of these, on operands that the caller holds on the GPU:

  quantize   rows of numbers quantised, and read back as the values that they now stand for
  product    matrix product of two quantised matrices
  linear     the same layer from 16- or 32-bit activations: they are quantised within the pass
  route      a router: which experts each token goes to, and with what weights
  experts    the gated feed-forward of the chosen experts, weights in 4 bits, activations in 16
  layer      route and experts behind one another

The definitions that both forms follow:

  4 bits     blocks of 32 neighbours in a row, the last one shorter; with m = max|x| of a block its scale is s = 2^(floor(log2 m) - 2), within 2^-127 ... 2^127
             (2^-127 for m = 0), and each element the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives to x / s, ties to the even code
  product    out[n][m] = sum_k W[m][k] A[n][k] + bias[m]
  route      l[t][e] = sum_k x[t][k] R[e][k], in 64 bits, rounded to 32; the `top` largest of l, or of sigmoid(l) + bias[e], the lowest expert first among
             equals; weights by softmax over the chosen, by softmax over all, or sigmoids over their sum, times a factor
  experts    out[t] = sum_j w[t][j] D_e (silu(G_e x[t]) * (U_e x[t])) with e = ids[t][j]; silu(g) = g / (1 + exp(-g))

A code is the element's place in the list above, plus 8 for the negatives; two to a byte, the even element low, whole blocks of 16 bytes (filled up with
zeros); a scale is the byte 127 + log2 s.  Rows of scales are whole words of four.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = {"bytes": 7e8, "flops": 1.2e12}


def listed():
    return [
        # one token's activations: latency
        dict(name="quantize_one", kind="quantize", N=1, K=4096, dtype="bf16"),
        # an odd chunk of a prompt with rows of odd length
        dict(name="quantize_ragged", kind="quantize", N=2049, K=5003, dtype="f16"),
        # a long prompt's activations, or a weight matrix: bound by memory
        dict(name="quantize_prompt", kind="quantize", N=16384, K=8192, dtype="bf16"),
        # one linear layer for one token: latency, and the weights streamed once
        dict(name="linear_one_token", kind="linear", N=1, M=4096, K=4096, dtype="bf16", bias=False),
        # a large layer for a small batch of decoded tokens, with a bias
        dict(name="linear_decode_16", kind="linear", N=16, M=8192, K=8192, dtype="f16", bias=True),
        # an odd prompt through a layer of odd size, in 32 bits
        dict(name="product_ragged", kind="product", N=333, M=1537, K=2000, dtype="f32", bias=True),
        # the benchmark's square product: a long prompt, bound by arithmetic
        dict(name="linear_prompt_8192", kind="linear", N=8192, M=8192, K=8192, dtype="bf16", bias=False),
        # one token's experts: latency
        dict(name="route_one", kind="route", T=1, K=4096, E=64, top=4, mode="softmax", bias=False, dtype="bf16", rdtype="bf16"),
        # a long prompt's experts, by sigmoids and a bias, from a router held in 32 bits
        dict(name="route_prompt", kind="route", T=8192, K=2048, E=128, top=8, mode="sigmoid", bias=True, dtype="bf16", rdtype="f32"),
        # one token through its experts: latency
        dict(name="experts_one", kind="experts", T=1, K=2048, F=1024, E=64, top=4, dtype="bf16"),
        # a serving batch's next tokens: nearly every expert's weights are read
        dict(name="experts_batch", kind="experts", T=64, K=4096, F=1024, E=64, top=6, dtype="bf16"),
        # a whole layer for an odd batch, odd sizes
        dict(name="layer_ragged", kind="layer", T=37, K=1444, F=715, E=60, top=5, mode="softmax_all", bias=False, dtype="f16", rdtype="f16"),
    ]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: a quarter of the sizes are any integers, the others multiples of 32."""
    while True:
        kind = rng.choice(("quantize", "product", "linear", "linear", "route", "route", "experts", "experts", "layer"))
        size = (lambda lo, hi: _log(rng, lo, hi)) if rng.random() < 0.25 else (lambda lo, hi: 32 * _log(rng, lo / 32, hi / 32))
        if kind == "quantize":
            case = dict(kind=kind, N=_log(rng, 1, 16384), K=size(64, 16384), dtype=rng.choice(("bf16", "f16", "f32")))
        elif kind in ("product", "linear"):
            case = dict(kind=kind, N=_log(rng, 1, 8192), M=size(256, 16384), K=size(256, 16384), dtype=rng.choice(("bf16", "f16", "f32")),
                        bias=rng.random() < 0.5)
        else:
            E = rng.choice((4, 8, 16, 32, 60, 64, 128, 256))
            case = dict(kind=kind, T=_log(rng, 1, 8192 if kind == "route" else 256), K=size(256, 8192 if kind == "route" else 4096), E=E,
                        top=rng.randint(1, min(E, 8)), dtype=rng.choice(("bf16", "f16")))
            if kind != "experts":
                case.update(mode=rng.choice(("softmax", "softmax_all", "sigmoid")), bias=rng.random() < 0.5, rdtype=rng.choice(("f32", case["dtype"])))
            if kind != "route":
                case["F"] = size(128, 4096)
                if E * case["K"] * case["F"] > 3e8:
                    continue
        w = work(case)
        if w["bytes"] <= LARGEST["bytes"] and 1e4 < w["flops"] <= LARGEST["flops"]:
            return case


def _held(rows, K):
    """The bytes of a quantised matrix's codes and scales."""
    return rows * -(-K // 32) * 17


def _chosen(case):
    """About how many experts a batch goes to: tokens choose by popularities that fall from expert to expert (see _choices)."""
    p = [0.99 ** e for e in range(case["E"])]
    return sum(1 - (1 - min(1.0, case["top"] * x / sum(p))) ** case["T"] for x in p)


def work(case):
    if case["kind"] == "quantize":
        values = case["N"] * case["K"]
        return {"bytes": 2 * values * SIZE[case["dtype"]] + 2 * _held(case["N"], case["K"]), "flops": 4 * values}
    if case["kind"] in ("product", "linear"):
        N, M, K, b = case["N"], case["M"], case["K"], SIZE[case["dtype"]]
        x = _held(N, K) if case["kind"] == "product" else N * K * b
        return {"bytes": x + _held(M, K) + N * M * b + (4 * M if case["bias"] else 0), "flops": 2 * N * M * K}
    T, K, E, top = case["T"], case["K"], case["E"], case["top"]
    bytes_, flops = T * K * SIZE[case["dtype"]] + 8 * T * top, 0
    if case["kind"] != "experts":
        bytes_ += E * K * SIZE[case["rdtype"]] + (4 * E if case["bias"] else 0)
        flops += 2 * T * E * K
    if case["kind"] != "route":
        bytes_ += int(_chosen(case) * (_held(2 * case["F"], K) + _held(K, case["F"]))) + T * K * SIZE[case["dtype"]]
        flops += 6 * T * top * K * case["F"]
    return {"bytes": bytes_, "flops": flops}


# ---- the plain form ---------------------------------------------------------------------------------------------------


def _levels(device, dtype=torch.float32):
    return torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=device, dtype=dtype)


def _quantize(x):
    """[..., K] in 32 bits -> codes (a byte each) and scales' bytes, [..., blocks, 32] and [..., blocks]; elements past K are 0."""
    K = x.shape[-1]
    if K % 32:
        x = torch.cat((x, torch.zeros(*x.shape[:-1], 32 - K % 32, device=x.device)), -1)
    x = x.unflatten(-1, (-1, 32))
    exponent = torch.frexp(x.abs().amax(-1)).exponent.clamp(-124, 130) - 3       # (2^exponent / 8 <= max / 4 < 2^exponent / 4; 0 is 0 * 2^0)
    exponent = torch.where((x == 0).all(-1), -127, exponent)
    a = torch.ldexp(x, -exponent[..., None]).abs()
    codes = torch.zeros_like(a, dtype=torch.uint8)
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        codes += (a > border) if i % 2 == 0 else (a >= border)
    return codes + 8 * (x < 0), (exponent + 127).to(torch.uint8)


def _pack(codes, scales):
    """What a program holds of them: two codes to a byte, [rows][16 * blocks], and rows of scales of whole words."""
    codes = codes.flatten(-2)
    packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
    room = torch.zeros(*scales.shape[:-1], -(-scales.shape[-1] // 4) * 4, dtype=torch.uint8, device=scales.device)
    room[..., :scales.shape[-1]] = scales
    return packed, room[..., :scales.shape[-1]]


def _values(packed, scales, K, dtype=torch.float32):
    """The values [..., K] of codes and scales as _pack gives them."""
    codes = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    x = _levels(packed.device, dtype)[codes.long()].unflatten(-1, (-1, 32))
    return torch.ldexp(x, scales[..., None].to(torch.int32) - 127).flatten(-2)[..., :K]


def _product(A, W, bias, dtype):
    y = torch.matmul(A, W.t())
    return (y if bias is None else y + bias).to(dtype)


def _route(x, R, top, mode, bias, factor):
    logits = torch.matmul(x.double(), R.double().t()).float()
    choice = torch.sigmoid(logits.double()) if mode == "sigmoid" else logits.double()
    if bias is not None:
        choice = choice + bias.double()
    ids = torch.sort(choice, dim=-1, descending=True, stable=True).indices[:, :top]
    if mode == "sigmoid":
        w = torch.sigmoid(logits).gather(1, ids)
        w = w / w.sum(-1, keepdim=True)
    else:
        chosen = logits.gather(1, ids)
        over = chosen if mode == "softmax" else logits
        most = over.amax(-1, keepdim=True)
        w = torch.exp(chosen - most) / torch.exp(over - most).sum(-1, keepdim=True)
    return ids.to(torch.int32), w * factor


def _gated(x, up, down):
    """x [..., K], up [..., 2 F, K], down [..., K, F] -> [..., K], all in one width."""
    g, u = torch.matmul(x, up.transpose(-1, -2)).chunk(2, -1)
    return torch.matmul(g / (1 + torch.exp(-g)) * u, down.transpose(-1, -2))


def _experts(state, x, ids, weights):
    """Few choices: each with its expert's weights; more than there are experts: every expert for all tokens."""
    case = state["case"]
    K, F, E, top = case["K"], case["F"], case["E"], case["top"]
    x, out = x.float(), 0.0
    if case["T"] * top <= E:
        up, down = (_values(state[n][ids.long()], state[n + "_scales"][ids.long()], size) for n, size in (("up", K), ("down", F)))
        y = _gated(x[:, None, None], up, down)[:, :, 0]
        return (y * weights[..., None]).sum(1).to(state["dtype"])
    for e in range(E):
        y = _gated(x, _values(state["up"][e], state["up_scales"][e], K), _values(state["down"][e], state["down_scales"][e], F))
        out = out + y * torch.where(ids == e, weights, 0.0).sum(1, keepdim=True)
    return out.to(state["dtype"])


# ---- cases ------------------------------------------------------------------------------------------------------------


def _activations(gen, rows, K, dtype):
    """A few large channels among many, as between a network's layers."""
    x = torch.randn(rows, K, device="cuda", generator=gen) * (1 + 9 * (torch.rand(K, device="cuda", generator=gen) < 0.01))
    return x.to(DTYPES[dtype])


def _weights(gen, rows, K):
    """A layer's weights, each row of its own size, quantised and packed."""
    W = torch.randn(rows, K, device="cuda", generator=gen) * ((0.5 + torch.rand(rows, 1, device="cuda", generator=gen)) / math.sqrt(K))
    return _pack(*_quantize(W))


def _router(case, gen):
    x = _activations(gen, case["T"], case["K"], case["dtype"])
    R = (torch.randn(case["E"], case["K"], device="cuda", generator=gen) / math.sqrt(case["K"])).to(DTYPES[case["rdtype"]])
    return x, R, 0.05 * torch.randn(case["E"], device="cuda", generator=gen) if case["bias"] else None


def _choices(case, gen):
    """Experts of popularities that fall from one to the next, in no order, different ones for a token; and weights that add up to 1."""
    T, E, top = case["T"], case["E"], case["top"]
    score = torch.rand(T, E, device="cuda", generator=gen).log_() / (0.99 ** torch.arange(E, device="cuda"))
    ids = torch.randperm(E, device="cuda", generator=gen)[score.topk(top, -1).indices].to(torch.int32)
    return ids, torch.softmax(torch.randn(T, top, device="cuda", generator=gen), -1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    state = {"case": case, "kind": kind, "dtype": dtype, "factor": 1.0}
    if kind == "quantize":
        N, K = case["N"], case["K"]
        x = _activations(gen, N, K, case["dtype"])
        codes, scales = _pack(torch.zeros(N, -(-K // 32), 32, dtype=torch.uint8, device="cuda"), torch.zeros(N, -(-K // 32), dtype=torch.uint8, device="cuda"))
        state.update(x=x, codes=codes, scales=scales, out=torch.empty_like(x))
        return state
    if kind in ("product", "linear"):
        N, M, K = case["N"], case["M"], case["K"]
        x = _activations(gen, N, K, case["dtype"])
        W, W_scales = _weights(gen, M, K)
        state.update(W=W, W_scales=W_scales, bias=torch.randn(M, device="cuda", generator=gen) if case["bias"] else None,
                     out=torch.empty(N, M, dtype=dtype, device="cuda"))
        if kind == "linear":
            state["x"] = x
        else:
            state["A"], state["A_scales"] = _pack(*_quantize(x.float()))
        return state
    if kind == "experts":
        x = _activations(gen, case["T"], case["K"], case["dtype"])
        state["ids"], state["weights"] = _choices(case, gen)
    else:
        x, state["R"], state["bias"] = _router(case, gen)
        state["ids"] = torch.empty(case["T"], case["top"], dtype=torch.int32, device="cuda")
        state["weights"] = torch.empty(case["T"], case["top"], device="cuda")
        state["factor"] = 2.5 if case["mode"] == "sigmoid" else 1.0
    state["x"] = x
    if kind != "route":
        E, K, F = case["E"], case["K"], case["F"]
        for name, rows, size in (("up", 2 * F, K), ("down", K, F)):
            blocks = -(-size // 32)
            codes = torch.empty(E, rows, 16 * blocks, dtype=torch.uint8, device="cuda")
            scales = torch.zeros(E, rows, -(-blocks // 4) * 4, dtype=torch.uint8, device="cuda")
            for e in range(E):
                codes[e], scales[e, :, :blocks] = _weights(gen, rows, size)
            state[name], state[name + "_scales"] = codes, scales[..., :blocks]
        state["out"] = torch.empty_like(x)
    return state


def run(state):
    kind, case = state["kind"], state["case"]
    if not own:
        if kind == "quantize":
            codes, scales = _quantize(state["x"].float())
            return _values(*_pack(codes, scales), case["K"]).to(state["dtype"])
        if kind == "product":
            K = case["K"]
            return _product(_values(state["A"], state["A_scales"], K), _values(state["W"], state["W_scales"], K), state["bias"], state["dtype"])
        if kind == "linear":
            K = case["K"]
            A = _values(*_pack(*_quantize(state["x"].float())), K)
            return _product(A, _values(state["W"], state["W_scales"], K), state["bias"], state["dtype"])
        if kind == "experts":
            return _experts(state, state["x"], state["ids"], state["weights"])
        ids, weights = _route(state["x"], state["R"], case["top"], case["mode"], state["bias"], state["factor"])
        return (ids, weights) if kind == "route" else (ids, weights, _experts(state, state["x"], ids, weights))
    else:
        for name in ("W", "A"):                                  # (a program holds codes as bytes: the library's calls take nothing else)
            if name in state and state[name].dtype != torch.uint8:
                state[name] = state[name].to(torch.uint8)
    from paper_2304_09049_amd import binding as dg
    if kind == "quantize":
        dg.dg_quantize_mx4(state["x"], codes=state["codes"], scales=state["scales"])
        return dg.dg_dequantize_mx4(state["codes"], state["scales"], case["K"], out=state["out"])
    if kind == "product":
        return dg.dg_gemm_mx4(state["W"], state["W_scales"], state["A"], state["A_scales"], bias=state["bias"], out=state["out"])
    if "work" not in state:                                      # (a program keeps them beside its weights)
        need = 0
        if kind == "linear":
            need = dg.dg_linear_mx4_work_bytes(case["N"], case["K"])
        if kind in ("route", "layer"):
            state["route_work"] = torch.empty(dg.dg_route_tokens_work_bytes(case["T"], case["E"]), dtype=torch.uint8, device="cuda")
        if kind in ("experts", "layer"):
            need = dg.dg_experts_mx4_work_bytes(case["T"], case["top"], case["K"], case["F"])
        state["work"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    if kind == "linear":
        return dg.dg_linear_mx4(state["W"], state["W_scales"], state["x"], bias=state["bias"], work=state["work"], out=state["out"])
    if kind != "experts":
        dg.dg_route_tokens(state["x"], state["R"], case["top"], mode=case["mode"], bias=state["bias"], factor=state["factor"], ids=state["ids"],
                           weights=state["weights"], work=state["route_work"])
        if kind == "route":
            return state["ids"], state["weights"]
    out = dg.dg_experts_mx4(state["up"], state["up_scales"], state["down"], state["down_scales"], state["x"], state["ids"], state["weights"],
                            work=state["work"], out=state["out"])
    return out if kind == "experts" else (state["ids"], state["weights"], out)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _nearest(x):
    """The values that rows of x [N][K], 64 bits holding 32 or fewer, stand for once quantised: whole steps of 1/2, 1 or 2 scales."""
    N, K = x.shape
    y = torch.zeros(N, -(-K // 32) * 32, dtype=torch.float64, device=x.device)
    y[:, :K] = x
    y = y.view(N, -1, 32)
    most = y.abs().amax(2, keepdim=True)
    power = (most.view(torch.int64) >> 52) - 1023 - 2            # floor(log2), by the number's own bits
    scale = (power.clamp(-127, 127) + 1023 << 52).view(torch.float64)
    q = y / scale
    step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0))
    return ((q / step).round() * step).clamp(-6, 6).mul_(scale).view(N, -1)[:, :K]


def _decoded(codes, scales, K):
    """Values by each element's place in its row's bytes, 64 bits."""
    k = torch.arange(K, device=codes.device)
    code = (codes[..., k // 2] >> (4 * (k % 2)).to(torch.uint8)) & 15
    size, sign = (code & 7).double(), 1 - 2 * (code >> 3).double()
    value = torch.where(size < 4, size / 2, torch.where(size < 6, size - 2, 2 * size - 8))
    return sign * value * torch.exp2(scales[..., k // 32].double() - 127)


def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "quantize":
        return _nearest(_activations(gen, case["N"], case["K"], case["dtype"]).double())
    if case["kind"] in ("product", "linear"):
        state = prepare(case, seed)
        A = _nearest(_activations(gen, case["N"], case["K"], case["dtype"]).double())
        y = torch.matmul(A, _decoded(state["W"], state["W_scales"], case["K"]).t())
        return y if state["bias"] is None else y + state["bias"].double()
    state = prepare(case, seed)
    x, ids, weights = state["x"].double(), state["ids"].long(), state["weights"].double()
    if case["kind"] != "experts":
        logits = (x @ state["R"].double().t()).float().double()
        bias = 0.0 if state["bias"] is None else state["bias"].double()
        chance = 1 / (1 + torch.exp(-logits)) if case["mode"] == "sigmoid" else torch.exp(logits)
        ids = ((chance if case["mode"] == "sigmoid" else logits) + bias).sort(dim=-1, descending=True, stable=True)[1][:, :case["top"]]
        weights = chance.gather(1, ids)
        weights = weights * state["factor"] / (chance if case["mode"] == "softmax_all" else weights).sum(1, keepdim=True)
        if case["kind"] == "route":
            return ids.int(), weights
    out = torch.zeros_like(x)
    for e in range(case["E"]):
        t, j = (ids == e).nonzero(as_tuple=True)
        if t.numel():
            up, down = _decoded(state["up"][e], state["up_scales"][e], case["K"]), _decoded(state["down"][e], state["down_scales"][e], case["F"])
            h = x[t] @ up.t()
            g, u = h[:, :case["F"]], h[:, case["F"]:]
            out.index_add_(0, t, weights[t, j, None] * ((g * torch.sigmoid(g) * u) @ down.t()))
    return out if case["kind"] == "experts" else (ids.int(), weights, out)
