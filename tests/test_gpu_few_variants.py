"""Every variant of the few-token kernels: the token counts on both sides of each of their rules, with more experts' CTAs than
SMs (two or three an SM) and with fewer (one), for each weight type. Tolerances as in test_gpu_few."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm
from test_gpu_few import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d,H,E", [(512, 1024, 8), (64, 192, 2)])
@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("T", [1, 2, 4, 5, 7, 8, 9, 16, 17, 32, 33, 64])
def test_token_counts(kind, d, H, E, ln, T):
    L = Layer(kind, d, H, E, seed=T + d, b2=True, ln=ln)
    x = L.tokens(T, [t % E for t in range(T)])
    out = torch.full((T, d), float("nan"), device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    L.check(out, x)
    L.close()
