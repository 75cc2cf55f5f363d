"""Weights written by a product of this library, one other call, then a few-token forward that reads them: the header's
rule for weights (any later work between their writer and the call) without a synchronisation."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("between", ["quantise", "product", "dense"])
@pytest.mark.parametrize("T", [1, 20])
def test_fc1_and_experts_see_them(between, T):
    d, H, E = 768, 3072, 2
    L = Layer("bf16", d, H, E, seed=T)
    x, out = L.tokens(T), torch.zeros(T, d, device="cuda", dtype=torch.bfloat16)
    K = 256
    ops = []
    for rows, cols in ((H, d), (d, H), (d, H)):  # W1 and both experts as products
        A, B = cm.fp8_rows(rows, K), cm.fp8_weight(cols, K)
        cm.clearmoe_fp8_quantize_rows(torch.randn(rows, K, device="cuda", generator=L.g), A)
        cm.clearmoe_fp8_quantize_weight(0.01 * torch.randn(cols, K, device="cuda", generator=L.g), B)
        ops.append((A, B))
    xs, rows = torch.randn(3, 128, device="cuda", dtype=torch.bfloat16), cm.fp8_rows(3, 128)
    W8, small = cm.fp8_weight(16, 128), torch.empty(3, 16, device="cuda")
    cm.clearmoe_fp8_quantize_weight(torch.randn(16, 128, device="cuda"), W8)
    cm.clearmoe_fp8_quantize_rows(xs, rows)
    L2 = Layer("bf16", 64, 64, 1, seed=1)
    x2, o2 = L2.tokens(2), torch.empty(2, 64, device="cuda", dtype=torch.bfloat16)
    for r in range(4):
        for m in L.m[:3]:
            m.zero_()
        torch.cuda.synchronize()
        for (A, B), m in zip(ops, L.m):
            cm.clearmoe_fp8_gemm(A, B, m)
        if between == "quantise":
            cm.clearmoe_fp8_quantize_rows(xs, rows)
        elif between == "product":
            cm.clearmoe_fp8_gemm(rows, W8, small)
        else:
            cm.clearmoe_dense_ffn_forward(L2.h, x2, L2.m[0], L2.b1, L2.m[1], o2)
        cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
        first = out.clone()
        torch.cuda.synchronize()
        cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
        assert torch.equal(first, out) and bool(out.abs().sum() > 0)
    L.close()
    L2.close()
