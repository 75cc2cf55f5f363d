"""The activations of products in 4-bit blocks do not depend on the kernel: operands whose sums are multiples of 1/8
that fp32 holds exactly in any order, so that every kernel has the same value before its activation, give the same
value after it, in each kind of output. Special values come by the bias: NaN and -inf give NaN under GELU, inf gives inf."""
import math

import numpy as np
import pytest
import torch

import fp4_ref as R
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu

KERNELS = [(256, 1), (128, 1), (128, 0), (64, 0), (16, 0)]
N, K = 352, 1024
SPECIAL = [-math.inf, math.inf, math.nan, -5.0, -4.5, -30.0, -3e38, 3e38, -0.0, 2.0 ** -149]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def operands(M):
    """Rows of -1, 0 and 1 and weights of eighths: sums are multiples of 1/8 below 128."""
    rng = np.random.default_rng(M)
    a, w = rng.integers(-1, 2, (M, K)), rng.integers(-1, 2, (N, K)) / 8.0
    a[0] = 0  # a row that is its bias alone
    A, W = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K)
    cm.clearmoe_fp4_quantize(dev(a), A)
    cm.clearmoe_fp4_quantize(dev(w), W)
    bias = np.zeros(N, np.float32)
    for i, v in enumerate(SPECIAL):
        bias[40 * (i % 8) + i] = v  # the first eight blocks have one or two each, the others none
    return A, W, dev(bias), a.astype(np.float64) @ w.T + bias.astype(np.float64)


def outputs(A, W, bias, act, M):
    """fp32 and bf16 values, and codes and scale bytes."""
    r = []
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.empty(M, N, device="cuda", dtype=dtype)
        cm.clearmoe_fp4_gemm(A, W, out, bias=bias, act=act)
        r.append(out)
    q = cm.fp4_matrix(M, N)
    q.q.fill_(0x33)
    cm.clearmoe_fp4_gemm(A, W, q, bias=bias, act=act)
    return [*r, q]


def blocks(q):
    """Codes outside blocks that are NaN (their codes may be anything), -0 as 0, and scale bytes."""
    s = R.scale_bytes(q.scale.cpu().numpy(), q.rows, q.cols)
    code = R.unpack(q.q.cpu().numpy(), q.cols)[0]
    return np.where(np.repeat(s == 255, 32, 1)[:, :q.cols] | (code == 8), 0, code), s


@pytest.mark.parametrize("act", [cm.ACT_NONE, cm.ACT_RELU, cm.ACT_GELU])
@pytest.mark.parametrize("M", [1, 30, 128])
def test_every_kernel_gives_the_same_values(M, act):
    A, W, bias, u = operands(M)
    got = {}
    try:
        for k in KERNELS:
            cm.clearmoe_debug_fp4_kernel(*k)
            got[k] = outputs(A, W, bias, act, M)
    finally:
        cm.clearmoe_debug_fp4_kernel()
    got["by size"] = outputs(A, W, bias, act, M)
    first = got[KERNELS[0]]
    for k, (f, b, q) in got.items():
        assert torch.equal(f[~f.isnan()], first[0][~first[0].isnan()]), k
        assert torch.equal(b[~b.isnan()], first[1][~first[1].isnan()]), k
        assert torch.equal(f.isnan(), first[0].isnan()) and torch.equal(b.isnan(), first[0].isnan()), k
        for mine, theirs in zip(blocks(q), blocks(first[2])):
            assert np.array_equal(mine, theirs), k
    if act != cm.ACT_GELU:
        return
    # fp32 against float64: u (1 + erf) / 2, NaN where u is NaN or -inf. u is exact but where 3e38 takes the sum in, half a step
    from scipy.special import ndtr
    with np.errstate(invalid="ignore"):
        want = u * ndtr(u)
    f, b = (t.float().cpu().numpy().astype(np.float64) for t in first[:2])
    assert np.array_equal(np.isnan(f), np.isnan(want)) and np.array_equal(f == np.inf, want == np.inf)
    fine = np.isfinite(want)
    f, b, want = f[fine], b[fine], want[fine]
    assert (np.abs(f - want) <= 2.5e-7 + 2.0 ** -23 * np.abs(want)).all()
    assert (np.abs(b - want) <= 1.01 * 3.2e-7 + 2.0 ** -8 * 1.001 * np.abs(want)).all()


@pytest.mark.parametrize("M,kernel", [(M, k) for k in KERNELS for M in (5, 128, 700) if k != (16, 0) or M <= 128])
@pytest.mark.parametrize("act", [cm.ACT_NONE, cm.ACT_RELU])
def test_blocks_are_the_fp32_result_quantised(M, act, kernel):
    """Bit for bit, of sums that round: the same kernel to fp32, then the quantiser."""
    rng = np.random.default_rng(M)
    A, W = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K)
    cm.clearmoe_fp4_quantize(dev(rng.standard_normal((M, K))), A)
    cm.clearmoe_fp4_quantize(dev(0.1 * rng.standard_normal((N, K))), W)
    bias = dev(rng.standard_normal(N))
    bias[[3, 70]] = torch.tensor([math.inf, math.nan], device="cuda")
    cm.clearmoe_debug_fp4_kernel(*kernel)
    try:
        f, _, q = outputs(A, W, bias, act, M)
    finally:
        cm.clearmoe_debug_fp4_kernel()
    want = cm.fp4_matrix(M, N)
    cm.clearmoe_fp4_quantize(f, want)
    for mine, theirs in zip(blocks(q), blocks(want)):
        assert np.array_equal(mine, theirs)
