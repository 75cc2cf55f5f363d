"""8-bit blocks on the GPU: quantisation against numpy bit for bit, products against float64.

Error bounds, per element: products of e4m3 values and their scales are exact, so the fp32 sum over K terms is off
by at most (K + 8) 2^-23 sum |a| |w| (2^-23: the tensor cores may cut instead of round); bias and activation add a
few fp32 roundings and the GELU's own 4e-7; bf16 outputs half a bf16 step (2^-9 relative, 2^-8 with what is before
it); 8-bit outputs half an e4m3 step (2^-4 relative, or 2^-10 of the block's scale near zero), the scale at most
twice amax / 448."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_ref as R
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda").to(dtype)


def rows_of(rng, M, K, spread=4.0):
    x = rng.standard_normal((M, K)) * np.exp(spread * rng.standard_normal((M, 1)))
    x[:, rng.random(K) < 0.02] *= 50.0
    return x.astype(np.float32)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def codes(m):
    return m.q.view(torch.uint8).cpu().numpy()


def check_quantized(m, x, block_rows):
    q, s, val = R.quantize(x, block_rows)
    kb = s.shape[1]
    assert np.array_equal(m.scale.cpu().numpy()[:, :kb], s)
    fine = np.repeat(np.repeat(s != 255, block_rows, 0)[:x.shape[0]], 128, 1)
    assert np.array_equal(np.where(fine, codes(m), 0), np.where(fine, q, 0))
    return val


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,pad", [(1, 1, 0), (1, 128, 0), (3, 127, 0), (5, 129, 0), (17, 512, 8), (33, 768, 0), (2, 1131, 3),
                                     (300, 64, 0)])
def test_quantize_rows(M, K, pad, dtype):
    rng = np.random.default_rng(M * 1000 + K)
    wide = dev(rows_of(rng, M, K + pad), dtype)
    x = wide[:, :K]
    m = cm.fp8_rows(M, K)
    m.q.view(torch.uint8).fill_(0x5A)
    cm.clearmoe_fp8_quantize_rows(x, m)
    val = check_quantized(m, f64(x), 1)
    out = torch.full((M, K), float("nan"), device="cuda")
    cm.clearmoe_fp8_dequantize(m, out)
    assert np.array_equal(f64(out), val)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,K", [(1, 1), (128, 128), (129, 127), (200, 384), (77, 650)])
def test_quantize_weight(N, K, dtype):
    W = dev(rows_of(np.random.default_rng(N + K), N, K, 0.5), dtype)
    m = cm.fp8_weight(N, K)
    cm.clearmoe_fp8_quantize_weight(W, m)
    val = check_quantized(m, f64(W), 128)
    out = torch.empty(N, K, device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_fp8_dequantize(m, out)
    assert np.array_equal(f64(out), val)  # four significant bits: exact in bf16


def test_quantize_extremes_and_gather():
    x = np.zeros((9, 256), np.float32)
    x[1, 3] = np.inf
    x[2, 200] = np.nan
    x[3] = 1e-45
    x[4] = 3.4e38
    x[5, :128] = np.float32(448.0)
    x[6, :128] = np.nextafter(np.float32(448.0), np.float32(500))
    x[7] = -(2.0 ** -130)
    x[8, 5] = 1.0
    m = cm.fp8_rows(9, 256)
    cm.clearmoe_fp8_quantize_rows(dev(x), m)
    val = check_quantized(m, x.astype(np.float64), 1)
    out = torch.empty(9, 256, device="cuda")
    cm.clearmoe_fp8_dequantize(m, out)
    with np.errstate(over="ignore"):  # 3.4e38 rounds to 2^128, past fp32
        assert np.array_equal(f64(out), val.astype(np.float32), equal_nan=True)
    at = torch.tensor([8, 0, 8, 4, 5], dtype=torch.int32, device="cuda")
    g = cm.fp8_rows(5, 256)
    cm.clearmoe_fp8_quantize_rows(dev(x), g, gather=at)
    check_quantized(g, x.astype(np.float64)[at.cpu().numpy()], 1)


def make(rng, M, N, K, wscale=0.02):
    A, W = cm.fp8_rows(M, K), cm.fp8_weight(N, K)
    cm.clearmoe_fp8_quantize_rows(dev(rows_of(rng, M, K, 1.0)), A)
    cm.clearmoe_fp8_quantize_weight(dev(rows_of(rng, N, K, 0.5) * wscale), W)
    av, wv = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    cm.clearmoe_fp8_dequantize(A, av)
    cm.clearmoe_fp8_dequantize(W, wv)
    return A, W, av.double(), wv.double()


def reference(av, wv, bias, act):
    """float64 result and the bound on the fp32 one's error."""
    y, mag = av @ wv.T, av.abs() @ wv.abs().T
    err = (av.shape[1] + 8) * 2.0 ** -23 * mag
    if bias is not None:
        y = y + bias.double()
        err = err + 2.0 ** -23 * (y.abs() + bias.double().abs())
    if act == cm.ACT_GELU:
        y = 0.5 * y * torch.erfc(-y / np.sqrt(2.0))
        err = 1.13 * err + 4e-7 + 4e-7 * y.abs()  # |GELU'| <= 1.13
    elif act == cm.ACT_RELU:
        y = y.clamp(min=0)
    return y, err


SHAPES = [(1, 1, 1), (1, 96, 16), (3, 130, 128), (128, 128, 128), (129, 200, 511), (197, 768, 192), (64, 33, 4099),
          (1000, 777, 640), (5000, 512, 384), (20000, 192, 1024), (260, 3072, 768)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm(M, N, K, dtype):
    rng = np.random.default_rng(M + 7 * N + 13 * K)
    A, W, av, wv = make(rng, M, N, K)
    act = (cm.ACT_NONE, cm.ACT_GELU, cm.ACT_RELU)[(M + N + K) % 3]
    bias = dev(rng.standard_normal(N), dtype) if (M + N) % 2 else None
    out = torch.full((M + 1, N + 3), float("nan"), device="cuda", dtype=dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cm.clearmoe_fp8_gemm(A, W, out[:M, :N], bias=bias, act=act, status=status)
    y, err = reference(av, wv, bias, act)
    if dtype == torch.bfloat16:
        err = err + 2.0 ** -8 * y.abs() + 1e-38
    assert status.item() == 0
    assert bool(((out[:M, :N].double() - y).abs() <= err + 1e-38).all())
    assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())  # nothing past the output
    dense = torch.empty(M, N, device="cuda", dtype=dtype)
    cm.clearmoe_fp8_gemm(A, W, dense, bias=bias, act=act)
    assert torch.equal(dense, out[:M, :N])  # every store width gives the same values


KERNELS = [(256, 1), (192, 1), (128, 1), (192, 0), (128, 0), (64, 0), (32, 0)]


@pytest.fixture
def kernel(request):
    cm.clearmoe_debug_fp8_kernel(*request.param)
    yield request.param
    cm.clearmoe_debug_fp8_kernel()


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("M,N,K,act", [(700, 700, 1300, cm.ACT_GELU), (5, 40, 130, cm.ACT_NONE), (257, 300, 512, cm.ACT_RELU),
                                       (40000, 200, 100, cm.ACT_NONE)])
def test_every_kernel(kernel, M, N, K, act):
    """Each tile width on one SM and on pairs: sums, both stores, 8-bit outputs where the kernel has them."""
    rng = np.random.default_rng(M + N)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1)
    y, err = reference(av, wv, bias, act)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M, N), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp8_gemm(A, W, out, bias=bias, act=act)
        assert bool(((out.double() - y).abs() <= err + (2.0 ** -8 * y.abs() if dtype == torch.bfloat16 else 0)).all())
    if kernel[0] % 128 == 0:
        q, got = cm.fp8_rows(M, N), torch.empty(M, N, device="cuda")
        cm.clearmoe_fp8_gemm(A, W, q, bias=bias, act=act)
        cm.clearmoe_fp8_dequantize(q, got)
        amax = torch.nn.functional.pad(y.abs(), (0, -N % 128)).view(M, -1, 128).amax(2).repeat_interleave(128, 1)[:, :N]
        assert bool(((got.double() - y).abs() <= 1.07 * err + 2.0 ** -4 * y.abs() + 2.0 ** -10 * 2 * amax / 448 * 1.01).all())


@pytest.mark.parametrize("kernel", [(16, 0)], indirect=True)
@pytest.mark.parametrize("M,N,K,act", [(1, 1, 1, cm.ACT_NONE), (16, 40, 130, cm.ACT_GELU), (9, 5003, 257, cm.ACT_RELU),
                                       (7, 12000, 512, cm.ACT_NONE), (3, 77, 9000, cm.ACT_GELU)])
def test_kernel_for_few_rows(kernel, M, N, K, act):
    """The kernel for up to 16 rows at widths that the library gives to the tiled ones, too; a call of more rows than it
    takes is the tiled kernels' whatever was asked for."""
    rng = np.random.default_rng(M + N + K)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1)
    y, err = reference(av, wv, bias, act)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M, N + 3), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp8_gemm(A, W, out[:, :N], bias=bias, act=act)
        assert bool(((out[:, :N].double() - y).abs() <= err + (2.0 ** -8 * y.abs() if dtype == torch.bfloat16 else 0)).all())
        assert bool(out[:, N:].isnan().all())


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
def test_every_kernel_grouped(kernel):
    rng = np.random.default_rng(77)
    counts, N, K = [0, 300, 1, 0, 129, 700], 320, 640
    M, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    A, _, av, _ = make(rng, M, N, K)
    pairs = [make(rng, 1, N, K)[1::2] for _ in counts]
    perm = rng.permutation(M)
    out = torch.full((M, N), float("nan"), device="cuda")
    cm.clearmoe_fp8_grouped_gemm(A, [p[0] for p in pairs], torch.tensor(off, dtype=torch.int32, device="cuda"), out,
                                 perm=torch.tensor(perm, dtype=torch.int32, device="cuda"))
    for e in range(len(counts)):
        sl = slice(int(off[e]), int(off[e + 1]))
        y, err = reference(av[sl], pairs[e][1], None, cm.ACT_NONE)
        assert bool(((out[torch.tensor(perm[sl], device="cuda", dtype=torch.long)].double() - y).abs() <= err).all())


@pytest.mark.parametrize("M,N,K", [(1, 128, 128), (130, 768, 192), (77, 200, 300), (4000, 1536, 384), (9, 1, 5)])
def test_gemm_to_blocks(M, N, K):
    rng = np.random.default_rng(M + N + K)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1, torch.bfloat16)
    out = cm.fp8_rows(M, N)
    out.q.view(torch.uint8).fill_(0x33)
    cm.clearmoe_fp8_gemm(A, W, out, bias=bias, act=cm.ACT_GELU)
    got = torch.empty(M, N, device="cuda")
    cm.clearmoe_fp8_dequantize(out, got)
    y, err = reference(av, wv, bias, cm.ACT_GELU)
    pad = -N % 128
    amax = torch.nn.functional.pad(y.abs(), (0, pad)).view(M, -1, 128).amax(2).repeat_interleave(128, 1)[:, :N]
    assert bool(((got.double() - y).abs() <= 1.07 * err + 2.0 ** -4 * y.abs() + 2.0 ** -10 * 2 * amax / 448 * 1.01).all())
    assert not out.q.view(torch.uint8)[:, N:].any()
    # the scale is the least that holds the block
    kb = -(-N // 128)
    s = out.scale[:, :kb].double()
    top = torch.nn.functional.pad(got.double().abs(), (0, pad)).view(M, kb, 128).amax(2)
    live = top > 0
    assert bool((top[live] <= 448 * torch.exp2(s - 127)[live]).all())
    assert bool((top[live] * (1 + 2.0 ** -4) >= 224 * torch.exp2(s - 127)[live]).all())


def test_k_blocks_keep_their_scales():
    """Every K block of A and W in a scale of its own, over more than one word of scales and on both sides of a
    128-column border of W: one byte read from the wrong place is off by a power of two."""
    M, N, K = 257, 320, 1536
    rng = np.random.default_rng(5)
    a = rng.standard_normal((M, K)) * np.repeat(2.0 ** rng.integers(-20, 20, (M, K // 128)), 128, 1)
    w = rng.standard_normal((N, K)) * np.repeat(np.repeat(2.0 ** rng.integers(-20, 20, (3, K // 128)), 128, 1), 128, 0)[:N]
    A, W = cm.fp8_rows(M, K), cm.fp8_weight(N, K)
    cm.clearmoe_fp8_quantize_rows(dev(a), A)
    cm.clearmoe_fp8_quantize_weight(dev(w), W)
    av, wv = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    cm.clearmoe_fp8_dequantize(A, av)
    cm.clearmoe_fp8_dequantize(W, wv)
    out = torch.empty(M, N, device="cuda")
    cm.clearmoe_fp8_gemm(A, W, out)
    y, err = reference(av.double(), wv.double(), None, cm.ACT_NONE)
    assert bool(((out.double() - y).abs() <= err).all())
    for kb in range(K // 128):  # each block alone
        one = torch.zeros_like(av)
        one[:, kb * 128:(kb + 1) * 128] = av[:, kb * 128:(kb + 1) * 128]
        B = cm.fp8_rows(M, K)
        cm.clearmoe_fp8_quantize_rows(one, B)
        cm.clearmoe_fp8_gemm(B, W, out)
        y, err = reference(one.double(), wv.double(), None, cm.ACT_NONE)
        assert bool(((out.double() - y).abs() <= err).all()), kb


def test_nan_and_inf_stay_in_their_rows():
    rng = np.random.default_rng(9)
    M, N, K = 140, 256, 384
    x = rows_of(rng, M, K, 1.0)
    x[3, 200] = np.inf
    x[131, 5] = np.nan
    A, W = cm.fp8_rows(M, K), cm.fp8_weight(N, K)
    cm.clearmoe_fp8_quantize_rows(dev(x), A)
    cm.clearmoe_fp8_quantize_weight(dev(rows_of(rng, N, K, 0.5)), W)
    for act in (cm.ACT_NONE, cm.ACT_RELU, cm.ACT_GELU):
        out = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
        cm.clearmoe_fp8_gemm(A, W, out, act=act)
        bad = torch.zeros(M, dtype=torch.bool, device="cuda")
        bad[[3, 131]] = True
        assert bool(out[bad].isnan().all()) and bool(out[~bad].isfinite().all())
        q = cm.fp8_rows(M, N)
        cm.clearmoe_fp8_gemm(A, W, q, act=act)
        assert bool((q.scale[bad][:, :2] == 255).all()) and bool((q.scale[~bad][:, :2] < 255).all())


@pytest.mark.parametrize("counts", [[5], [0, 130, 0, 1], [128, 256, 3, 0, 77], [0, 0, 7], [1] * 16])
@pytest.mark.parametrize("N,K,dtype", [(192, 768, torch.bfloat16), (100, 200, torch.float32)])
def test_grouped(counts, N, K, dtype):
    rng = np.random.default_rng(sum(counts) + N)
    M, E = sum(counts), len(counts)
    A, _, av, _ = make(rng, M, N, K)
    Ws, wv = [], []
    for e in range(E):
        _, W, _, v = make(rng, 1, N, K)
        Ws.append(W)
        wv.append(v)
    off = np.concatenate([[0], np.cumsum(counts)])
    perm = rng.permutation(M)
    bias = dev(rng.standard_normal(N), dtype)
    out = torch.full((M, N), float("nan"), device="cuda", dtype=dtype)
    cm.clearmoe_fp8_grouped_gemm(A, Ws, torch.tensor(off, dtype=torch.int32, device="cuda"), out,
                                 perm=torch.tensor(perm, dtype=torch.int32, device="cuda"), bias=bias)
    for e in range(E):
        sl = slice(int(off[e]), int(off[e + 1]))
        y, err = reference(av[sl], wv[e], bias, cm.ACT_NONE)
        if dtype == torch.bfloat16:
            err = err + 2.0 ** -8 * y.abs()
        got = out[torch.tensor(perm[sl], device="cuda", dtype=torch.long)].double()
        assert bool(((got - y).abs() <= err).all())


def test_another_stream_and_twice():
    rng = np.random.default_rng(1)
    x = dev(rows_of(rng, 300, 768), torch.bfloat16)
    W = cm.fp8_weight(256, 768)
    cm.clearmoe_fp8_quantize_weight(dev(rows_of(rng, 256, 768, 0.5)), W)
    A, out = cm.fp8_rows(300, 768), torch.empty(300, 256, device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_fp8_quantize_rows(x, A)
    cm.clearmoe_fp8_gemm(A, W, out)
    first = out.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            cm.clearmoe_fp8_quantize_rows(x, A)
            cm.clearmoe_fp8_gemm(A, W, out)
    s.synchronize()
    assert torch.equal(out, first)


def test_refusals():
    L, A, W = cm.lib(), cm.fp8_rows(4, 256), cm.fp8_weight(8, 256)
    x = torch.zeros(4, 256, device="cuda")
    out = torch.zeros(4, 8, device="cuda")
    p, o = x.data_ptr(), out.data_ptr()
    qr = L.clearmoe_fp8_quantize_rows
    assert qr(None, cm.F32, 256, None, A.ref, None) == cm.EINVAL
    assert qr(p, 7, 256, None, A.ref, None) == cm.EINVAL
    assert qr(p, cm.F32, 255, None, A.ref, None) == cm.EINVAL
    assert qr(p + 1, cm.F32, 256, None, A.ref, None) == cm.EINVAL
    assert qr(p, cm.F32, 256, None, None, None) == cm.EINVAL

    def bad(m, **kw):
        c = cm.clearmoe_fp8(m.c.q, m.c.scale, m.rows, m.cols)
        for k, v in kw.items():
            setattr(c, k, v)
        return ctypes.byref(c)

    for kw in (dict(q=None), dict(scale=None), dict(rows=0), dict(cols=0), dict(rows=(1 << 30) + 1), dict(cols=(1 << 24) + 1),
               dict(q=A.c.q + 16), dict(scale=A.c.scale + 1)):
        assert qr(p, cm.F32, 1 << 25, None, bad(A, **kw), None) == cm.EINVAL, kw
        assert L.clearmoe_fp8_gemm(bad(A, **kw), W.ref, None, o, cm.F32, 8, None) == cm.EINVAL, kw
    gemm = L.clearmoe_fp8_gemm
    assert gemm(A.ref, bad(W, cols=128), None, o, cm.F32, 8, None) == cm.EINVAL
    assert gemm(A.ref, W.ref, None, None, cm.F32, 8, None) == cm.EINVAL
    assert gemm(A.ref, W.ref, None, o, cm.FP8, 8, None) == cm.EINVAL
    assert gemm(A.ref, W.ref, None, o, cm.F32, 7, None) == cm.EINVAL
    assert gemm(A.ref, W.ref, None, o + 2, cm.F32, 8, None) == cm.EINVAL
    for epi in (cm.clearmoe_fp8_epilogue(None, 0, 5, None), cm.clearmoe_fp8_epilogue(o, 9, -1, None),
                cm.clearmoe_fp8_epilogue(o + 1, cm.BF16, -1, None)):
        assert gemm(A.ref, W.ref, ctypes.byref(epi), o, cm.F32, 8, None) == cm.EINVAL
    assert L.clearmoe_fp8_gemm_fp8(A.ref, W.ref, None, cm.fp8_rows(4, 9).ref, None) == cm.EINVAL
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    arr = (cm.clearmoe_fp8 * 1)(W.c)
    grp = L.clearmoe_fp8_grouped_gemm
    assert grp(A.ref, arr, 0, off.data_ptr(), None, None, o, cm.F32, 8, None) == cm.EINVAL
    assert grp(A.ref, arr, 17, off.data_ptr(), None, None, o, cm.F32, 8, None) == cm.EINVAL
    assert grp(A.ref, arr, 1, None, None, None, o, cm.F32, 8, None) == cm.EINVAL
    for k in ((256, 0), (64, 1), (100, 0), (0, 1), (128, 2)):
        assert L.clearmoe_debug_fp8_kernel(*k) == cm.EINVAL
    with pytest.raises(ValueError):
        cm.clearmoe_fp8_quantize_rows(x[:, ::2], cm.fp8_rows(4, 128))
    with pytest.raises(ValueError):
        cm.clearmoe_fp8_gemm(A, W, torch.zeros(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        cm.Fp8Matrix(A.q, A.scale, 4, 300)
    torch.cuda.synchronize()
    assert not out.any()
