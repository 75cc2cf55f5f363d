"""RMS norms of rows whose squares, or the sum of their squares, leave fp32's range while the rows and their mean squares do not,
against float64; beside rows of ordinary size, zeros, infinities and NaN in the same call, with eps from 0 on.

Error bound: test_gpu_norm.py's 48 roundings of 2^-24; squares below fp32's normal numbers are off by up to 2^-134 each where eps
is at least 2^-108, another 2^-27 of the result. 1e-38 absolute, for results and products below the normal numbers."""
import math

import numpy as np
import pytest
import torch

import fp4_ref as R4
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu

MAGNITUDES = [0.0, 1e-44, 3e-40, 1e-38, 1e-30, 1e-25, 1e-22, 1e-19, 1e-16, 1e-8, 1.0, 1e4, 1e15, 3e17, 1e18, 1e19, 1e25, 1e38, math.inf,
              math.nan]
FLT_MAX = float(np.finfo(np.float32).max)


def rows(d, pad, dtype):
    """Two rows of each size in random order, of values between half of it and it; in the last two one infinite, one NaN."""
    rng = np.random.default_rng(d)
    m = rng.permutation(np.repeat(np.arange(len(MAGNITUDES)), 2))
    x = rng.uniform(0.5, 1.0, (len(m), d + pad)) * rng.choice([-1.0, 1.0], (len(m), d + pad))
    for i, k in enumerate(m):
        if math.isfinite(MAGNITUDES[k]):
            x[i] *= MAGNITUDES[k]
        else:
            x[i, d // 2] = MAGNITUDES[k]
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)[:, :d]


def reference(s, w, eps):
    """float64 norm, zeros where the mean square is past fp32; the rows whose mean is nearer to the border than its error are not
    made."""
    v = s.double()
    mean = v.square().mean(1, keepdim=True)
    y = v / (mean + float(np.float32(eps))).sqrt() * w.double()
    assert bool(((mean < 0.99 * FLT_MAX) | (mean > 1.01 * FLT_MAX) | mean.isnan()).all())
    return torch.where(mean > FLT_MAX, v * 0.0, y)


def same(out, y, half_step):
    out = out.double()
    if not torch.equal(out.isnan(), y.isnan()):
        return False
    y = torch.where(y.isnan(), 0.0, y)
    out = torch.where(out.isnan(), 0.0, out)
    return bool(((out - y).abs() <= (48 * 2.0 ** -24 + 2.0 ** -27 + half_step) * y.abs() + 1e-38).all())


WIDTHS = [1, 33, 64, 512, 776, 1536, 2048, 4096, 8192, 8200, 32768]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("d", WIDTHS)
def test_far_rows(d, pad, dtype):
    x = rows(d, pad, dtype)
    w = torch.from_numpy(np.random.default_rng(1).uniform(0.5, 2.0, d).astype(np.float32)).cuda()
    for eps in (0.0, 1e-44, 1e-37, 1e-32, 1e-6, 1e30):
        y = reference(x, w, eps)
        for out_dtype in (torch.float32, torch.bfloat16):
            out, total = torch.empty(x.shape, device="cuda", dtype=out_dtype), torch.empty(x.shape, device="cuda", dtype=dtype)
            cm.clearmoe_rms_norm(x, out, sum_out=total, weight=w, eps=eps)
            assert same(out, y, 2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0), (eps, out_dtype)
            assert torch.equal(total[~total.isnan()], x[~x.isnan()])
        place = x.contiguous()
        cm.clearmoe_rms_norm(place, place, weight=w, eps=eps)
        assert same(place, y, 2.0 ** -8 if dtype == torch.bfloat16 else 0.0), eps


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("d", WIDTHS)
def test_far_rows_to_blocks(d, pad, dtype):
    """The blocks that quantising the fp32 norm gives, bit for bit."""
    x = rows(d, pad, dtype)
    T = x.shape[0]
    r = torch.zeros_like(x)
    for eps in (0.0, 1e-6):
        y = torch.empty(T, d, device="cuda")
        cm.clearmoe_rms_norm(x, y, residual=r, eps=eps)
        finite = y.isfinite().all(1)
        a, b, n = cm.fp8_rows(T, d), cm.fp8_rows(T, d), -(-d // 128)
        cm.clearmoe_rms_norm(x, a, residual=r, eps=eps)
        cm.clearmoe_fp8_quantize_rows(y, b)
        assert torch.equal(a.scale[:, :n], b.scale[:, :n])
        assert torch.equal(a.q.view(torch.uint8)[finite], b.q.view(torch.uint8)[finite])
        a, b = cm.fp4_matrix(T, d), cm.fp4_matrix(T, d)
        cm.clearmoe_rms_norm(x, a, residual=r, eps=eps)
        cm.clearmoe_fp4_quantize(y, b)
        assert np.array_equal(R4.scale_bytes(a.scale.cpu().numpy(), T, d), R4.scale_bytes(b.scale.cpu().numpy(), T, d))
        assert torch.equal(a.q[finite], b.q[finite])
