"""NaN and infinities through the few-token forward: what a token's output depends on makes it NaN or infinite, as the
formula's float64 value is, and no other token's. NaN comes in several bit patterns, that of GPU arithmetic (all bits set)
among them; an infinity in an fp32 layer may come out as NaN."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu

BITS = [0x7FFFFFFF, 0xFFFFFFFF, 0x7FC00000, 0x7F810000, 0x7F800000, 0xFF800000]  # NaNs, then the infinities
D, H, E = 64, 256, 4


def put(t, at, bits):
    """t[at] = the value of these fp32 bits (their upper half in bf16), without arithmetic."""
    v, n = (t.view(torch.int16), 16) if t.dtype == torch.bfloat16 else (t.view(torch.int32), 32)
    b = bits >> 16 if n == 16 else bits
    v[at] = b - (1 << n) if b >> (n - 1) else b


def run(L, x):
    out = torch.zeros(len(x), D, device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    return out.isfinite()


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("T", [1, 7, 12, 30, 64])
@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("bits", BITS)
def test_in_a_token(kind, T, ln, bits):
    L = Layer(kind, D, H, E, seed=T, ln=ln)
    x = L.tokens(T)
    t = T // 2
    put(x, (t, 5), bits)
    ok = run(L, x)
    assert not bool(ok[t].any())
    ok[t] = True
    assert bool(ok.all())
    L.close()


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("T", [1, 12, 64])
@pytest.mark.parametrize("bits", BITS)
def test_in_a_weight_of_fc1(kind, T, bits):
    for where in ("W1", "b1"):
        L = Layer(kind, D, H, E, seed=T)
        if where == "b1":
            put(L.b1, 37, bits)
        elif kind == "fp8":
            W = 0.05 * torch.randn(H, D, device="cuda")
            put(W, (37, 11), bits)
            cm.clearmoe_fp8_quantize_weight(W, L.m[0])
        else:
            put(L.m[0], (37, 11), bits)
        assert not bool(run(L, L.tokens(T)).any()), where  # every output sums over hidden unit 37
        L.close()


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("T", [4, 12, 64])
@pytest.mark.parametrize("bits", BITS)
def test_in_a_weight_of_an_expert(kind, T, bits):
    L = Layer(kind, D, H, E, seed=T)
    if kind == "fp8":
        W = 0.05 * torch.randn(D, H, device="cuda")
        put(W, (3, 100), bits)
        cm.clearmoe_fp8_quantize_weight(W, L.m[1 + 2])
    else:
        put(L.m[1 + 2], (3, 100), bits)
    experts = [t % E for t in range(T)]
    ok = run(L, L.tokens(T, experts))
    hit = torch.tensor([e == 2 for e in experts], device="cuda")
    assert not bool(ok[hit][:, 3].any())
    assert bool(ok[~hit].all())
    if kind != "fp8":  # of 8-bit weights the whole block is NaN
        ok[:, 3] = True
        assert bool(ok.all())
    L.close()
