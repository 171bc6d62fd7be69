"""The measured cases of products and linear layers, small: what the library's calls give for their inputs is within what the roundings allow."""
import importlib.util
import os

import pytest
import torch

import mx4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cases():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "more_operators.py")
    spec = importlib.util.spec_from_file_location("more_operators", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind,N,M,K,bias", [("product", 1, 64, 96, False), ("product", 37, 65, 300, True), ("linear", 1, 64, 96, True), ("linear", 40, 33, 1024, False)])
def test_products(cases, kind, N, M, K, bias, dtype):
    case = dict(kind=kind, N=N, M=M, K=K, dtype=dtype, bias=bias)
    state = cases.prepare(case, 3)
    W = ref.values(state["W"].cpu().to(torch.uint8), state["W_scales"].cpu(), K)
    if kind == "linear":
        codes, scales = ref.quantize(state["x"].cpu())
        A = ref.pack(codes), scales
    else:
        A = state["A"].cpu().to(torch.uint8), state["A_scales"].cpu()
    want, off = ref.product(ref.values(*A, K), W, state["bias"].cpu() if bias else None, ref.TYPES[dtype])
    cases.own = True
    for _ in range(2):                                               # (the second pass finds what the first has made)
        ref.assert_within(cases.run(state), want, off)
