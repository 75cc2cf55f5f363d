"""The LayerNorm of the few-token forward on tokens whose mean is many times their deviation. fp32 layers: relative L2 <= 1e-5
as without one, whatever the ratio (the mean is taken off each token, exactly but for roundings of the deviation, before the
products). bf16 layers: their 2e-2, at ratios at which bf16 tokens still have a deviation (a step of 2^-8 of the mean)."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,ratio", [("f32", 0.0), ("f32", 30.0), ("f32", -300.0), ("f32", 3000.0), ("bf16", 8.0), ("fp8", -8.0)])
@pytest.mark.parametrize("d,H,T,E", [(192, 768, 1, 4), (192, 768, 12, 3), (384, 1536, 30, 6), (512, 256, 64, 8), (64, 128, 5, 1)])
def test_large_means(kind, ratio, d, H, T, E):
    L = Layer(kind, d, H, E, seed=T + d, b2=True, ln=True)
    x = (0.7 * (L.cent[torch.arange(T, device="cuda") % E] + 0.3 * torch.randn(T, d, generator=L.g, device="cuda") + ratio)).to(L.tdt)
    out = torch.full((T, d), float("nan"), device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    L.check(out, x)
    L.close()
