"""4-bit blocks on the GPU: quantisation against numpy bit for bit, products against float64.

Error bounds, per element: products of e2m1 values and their scales are exact, so the fp32 sum over K terms is off by at
most (K + 8) 2^-23 sum |a| |w| (2^-23: the tensor cores may cut instead of round); bias and activation add a few fp32
roundings and the GELU's own 4e-7 (times 1.13, the largest slope, what came before); bf16 outputs half a bf16 step (2^-8
relative, with what is before it); 4-bit outputs half an e2m1 step: at most 1/5 of the value (1.25, 2.5 and 5 lie half way)
or, below 0.5, a quarter of the block's scale, which is less than a third of its largest magnitude."""
import numpy as np
import pytest
import torch

import fp4_ref as R
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.float32):
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda").to(dtype)


def rows_of(rng, M, K, spread=4.0):
    x = rng.standard_normal((M, K)) * np.exp(spread * rng.standard_normal((M, 1)))
    x[:, rng.random(K) < 0.02] *= 50.0
    return x.astype(np.float32)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def check_quantized(m, x):
    """Codes, their padding and scale bytes of m against numpy's of x; numpy's values."""
    code, s, val = R.quantize(x)
    assert np.array_equal(R.scale_bytes(m.scale.cpu().numpy(), m.rows, m.cols), s)
    got, rest = R.unpack(m.q.cpu().numpy(), m.cols)
    fine = np.repeat(s != 255, 32, 1)[:, :m.cols]
    assert np.array_equal(np.where(fine, got, 0), np.where(fine, code, 0))
    last = s[:, -1] != 255
    assert not rest[last].any()
    return val


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,pad", [(1, 1, 0), (1, 32, 0), (3, 31, 0), (5, 33, 0), (17, 512, 8), (130, 96, 0), (2, 1131, 3),
                                     (300, 72, 0), (129, 200, 8)])
def test_quantize(M, K, pad, dtype):
    rng = np.random.default_rng(M * 1000 + K)
    x = dev(rows_of(rng, M, K + pad), dtype)[:, :K]
    m = cm.fp4_matrix(M, K)
    m.q.fill_(0x5A)
    m.scale.fill_(0x5A)
    cm.clearmoe_fp4_quantize(x, m)
    val = check_quantized(m, f64(x))
    tiles = m.scale.cpu().numpy()  # rows past the last are left as they were
    rest = np.concatenate([R.scale_bytes(tiles, tiles.shape[0] * 128, tiles.shape[1] * 128)[M:].ravel(), [0x5A]])
    assert (rest == 0x5A).all()
    out = torch.full((M, K), float("nan"), device="cuda")
    cm.clearmoe_fp4_dequantize(m, out)
    assert np.array_equal(f64(out), val)
    wide = torch.full((M, K + 3), float("nan"), device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_fp4_dequantize(m, wide[:, :K])
    assert np.array_equal(f64(wide[:, :K]), val) and bool(wide[:, K:].isnan().all())  # two significant bits: exact


def test_quantize_ties_and_extremes():
    x = np.zeros((12, 64), np.float32)
    x[1, 3] = np.inf
    x[2, 40] = np.nan
    x[3] = 1e-45
    x[4] = 3.4e38
    x[5, :32] = 6.0
    x[6, :32] = np.nextafter(np.float32(6.0), np.float32(7))
    x[7] = -(2.0 ** -130)
    x[8, 5] = 1.0
    x[9, :17] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -0.0, -6]
    x[10, :17] = np.nextafter(x[9, :17], np.float32(0))
    x[11, 32:49] = x[9, :17]
    for dtype in (torch.float32, torch.bfloat16):
        t = dev(x, dtype)
        m = cm.fp4_matrix(12, 64)
        cm.clearmoe_fp4_quantize(t, m)
        val = check_quantized(m, f64(t))
        out = torch.empty(12, 64, device="cuda")
        cm.clearmoe_fp4_dequantize(m, out)
        with np.errstate(over="ignore"):  # 3.4e38 rounds to 2^128, past fp32
            assert np.array_equal(f64(out), val.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("K", [256, 250])
def test_quantize_gathered(K):
    x = rows_of(np.random.default_rng(1), 9, K)
    t = dev(x)
    at = torch.tensor([8, 0, 8, 4, 5, -1, 9, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    m = cm.fp4_matrix(8, K)
    cm.clearmoe_fp4_quantize(t, m, gather=at)
    val = np.full((8, K), np.nan)
    val[:5] = x[at.cpu().numpy()[:5]]
    check_quantized(m, val)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("start,pad", [(0, 1), (1, 0), (1, 1), (2, 2)])
@pytest.mark.parametrize("K", [1, 2, 31, 127, 128, 129, 255, 256, 301, 1131])
def test_quantize_rows_that_start_anywhere(K, start, pad, gather):
    """bf16 rows at whole words, between them and by turns, NaN around each."""
    rng, M = np.random.default_rng(K), 37
    pitch = K + pad + 1
    flat = torch.full((start + M * pitch,), float("nan"), device="cuda", dtype=torch.bfloat16)
    x = flat[start:].view(M, pitch)[:, :K]
    x.copy_(dev(rows_of(rng, M, K), torch.bfloat16))
    m = cm.fp4_matrix(M, K)
    at = rng.permutation(M) if gather else np.arange(M)
    cm.clearmoe_fp4_quantize(x, m, gather=torch.tensor(at, dtype=torch.int32, device="cuda") if gather else None)
    check_quantized(m, f64(x)[at])


def test_quantize_far_rows():
    """Rows whose offsets pass 32 bits: two of a wide pitch."""
    ld = 1 << 29
    x = torch.zeros(5, ld, dtype=torch.bfloat16, device="cuda")
    v = dev(rows_of(np.random.default_rng(2), 5, 100), torch.bfloat16)
    x[:, 7:107] = v
    m = cm.fp4_matrix(5, 100)
    cm.clearmoe_fp4_quantize(x[:, 7:107], m)
    check_quantized(m, f64(v))


def make(rng, M, N, K, wscale=0.02):
    A, W = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K)
    for m in (A, W):  # bytes of rows past the last may be anything
        m.scale.fill_(255)
    cm.clearmoe_fp4_quantize(dev(rows_of(rng, M, K, 1.0)), A)
    cm.clearmoe_fp4_quantize(dev(rows_of(rng, N, K, 0.5) * wscale), W)
    return A, W, values(A), values(W)


def values(m):
    out = torch.empty(m.rows, m.cols, device="cuda")
    cm.clearmoe_fp4_dequantize(m, out)
    return out.double()


def reference(av, wv, bias, act):
    """float64 result and the bound on the fp32 one's error."""
    y, mag = av @ wv.T, av.abs() @ wv.abs().T
    err = (av.shape[1] + 8) * 2.0 ** -23 * mag
    if bias is not None:
        y = y + bias.double()
        err = err + 2.0 ** -23 * (y.abs() + bias.double().abs())
    if act == cm.ACT_GELU:
        y = 0.5 * y * torch.erfc(-y / np.sqrt(2.0))
        err = 1.13 * err + 4e-7 + 4e-7 * y.abs()
    elif act == cm.ACT_RELU:
        y = y.clamp(min=0)
    return y, err


def within(out, y, err):
    return bool(((out.double() - y).abs() <= err + (2.0 ** -8 * y.abs() if out.dtype == torch.bfloat16 else 0) + 1e-38).all())


SHAPES = [(1, 1, 1), (1, 96, 16), (3, 130, 64), (128, 128, 128), (129, 200, 511), (197, 768, 192), (64, 33, 4099),
          (1000, 777, 640), (5000, 512, 384), (20000, 192, 1024), (260, 2048, 768), (7, 5000, 65), (16, 64, 8192)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm(M, N, K, dtype):
    rng = np.random.default_rng(M + 7 * N + 13 * K)
    A, W, av, wv = make(rng, M, N, K)
    act = (cm.ACT_NONE, cm.ACT_GELU, cm.ACT_RELU)[(M + N + K) % 3]
    bias = dev(rng.standard_normal(N), dtype) if (M + N) % 2 else None
    out = torch.full((M + 1, N + 3), float("nan"), device="cuda", dtype=dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cm.clearmoe_fp4_gemm(A, W, out[:M, :N], bias=bias, act=act, status=status)
    y, err = reference(av, wv, bias, act)
    assert status.item() == 0
    assert within(out[:M, :N], y, err)
    assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())  # nothing past the output
    dense = torch.empty(M, N, device="cuda", dtype=dtype)
    cm.clearmoe_fp4_gemm(A, W, dense, bias=bias, act=act)
    assert torch.equal(dense, out[:M, :N])  # every store width gives the same values


KERNELS = [(256, 1), (128, 1), (128, 0), (64, 0), (16, 0)]


@pytest.fixture
def kernel(request):
    cm.clearmoe_debug_fp4_kernel(*request.param)
    yield request.param
    cm.clearmoe_debug_fp4_kernel()


def check_blocks(q, y, err):
    """A matrix in 4-bit blocks against the float64 values that it was rounded from."""
    M, N = y.shape
    amax = torch.nn.functional.pad(y.abs(), (0, -N % 32)).view(M, -1, 32).amax(2).repeat_interleave(32, 1)[:, :N]
    got = values(q)
    assert bool(((got - y).abs() <= 1.2 * err + 0.2 * y.abs() + 0.25 * 1.01 * amax / 3 + 1e-38).all())
    assert not R.unpack(q.q.cpu().numpy(), N)[1].any()
    # the scale is the least that holds the block, to the error
    s = R.scale_bytes(q.scale.cpu().numpy(), M, N).astype(np.float64)
    s = torch.from_numpy(np.repeat(s, 32, 1)[:, :N]).cuda()
    top = torch.nn.functional.pad(err, (0, -N % 32)).view(M, -1, 32).amax(2).repeat_interleave(32, 1)[:, :N]
    assert bool(((amax <= 6 * torch.exp2(s - 127) + top) & ((amax > 3 * torch.exp2(s - 127) - top) | (s == 0))).all())


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("M,N,K,act", [(700, 700, 1300, cm.ACT_GELU), (5, 40, 130, cm.ACT_NONE), (257, 300, 512, cm.ACT_RELU),
                                       (40000, 200, 100, cm.ACT_NONE), (130, 129, 2000, cm.ACT_NONE)])
def test_every_kernel(kernel, M, N, K, act):
    """Each tile width on one SM and on pairs: sums, every kind of store, 4-bit outputs."""
    rng = np.random.default_rng(M + N)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1)
    y, err = reference(av, wv, bias, act)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M, N), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp4_gemm(A, W, out, bias=bias, act=act)
        assert within(out, y, err)
    q = cm.fp4_matrix(M, N)
    q.q.fill_(0x33)
    cm.clearmoe_fp4_gemm(A, W, q, bias=bias, act=act)
    check_blocks(q, y, err)


@pytest.mark.parametrize("kernel", [(256, 1), (128, 1)], indirect=True)
@pytest.mark.parametrize("M,N,K,act", [(2500, 2000, 300, cm.ACT_GELU), (2500, 1900, 700, cm.ACT_NONE), (20000, 256, 100, cm.ACT_RELU),
                                       (4864, 1536, 1100, cm.ACT_NONE), (5120, 1290, 257, cm.ACT_GELU), (300, 20000, 64, cm.ACT_NONE)])
def test_rounds_that_end_in_few_tiles(kernel, M, N, K, act):
    """Last rounds of two to 38 tiles for 76 pairs, each of them in halves; those past the matrix among them."""
    rng = np.random.default_rng(M + N)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1)
    y, err = reference(av, wv, bias, act)
    for pad, dtype in ((0, torch.float32), (-N % 8, torch.bfloat16), (-N % 8 + 1, torch.bfloat16), (1, torch.float32)):
        out = torch.full((M + 1, N + pad), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp4_gemm(A, W, out[:M, :N], bias=bias, act=act)
        assert within(out[:M, :N], y, err)
        assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())
    q = cm.fp4_matrix(M, N)
    q.q.fill_(0x33)
    cm.clearmoe_fp4_gemm(A, W, q, bias=bias, act=act)
    check_blocks(q, y, err)


@pytest.mark.parametrize("kernel", [(256, 1)], indirect=True)
@pytest.mark.parametrize("counts", [[200, 0, 0, 0], [0, 0, 0, 0, 300], [3000, 1, 0, 5000, 2500, 777], [0, 9000, 0, 1300]])
def test_grouped_rounds_that_end_in_few_tiles(kernel, counts):
    """Halves of tiles in the first round, for half of the pairs that the grid has at the most, and in the second."""
    rng = np.random.default_rng(78)
    N, K = 500, 320
    M, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    A, _, av, _ = make(rng, M, N, K)
    pairs = [make(rng, 1, N, K)[1::2] for _ in counts]
    at = rng.permutation(M)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M + 1, N + 4), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp4_grouped_gemm(A, [p[0] for p in pairs], torch.tensor(off, dtype=torch.int32, device="cuda"), out[:M, :N],
                                     perm=torch.tensor(at, dtype=torch.int32, device="cuda"))
        for e in range(len(counts)):
            sl = slice(int(off[e]), int(off[e + 1]))
            y, err = reference(av[sl], pairs[e][1], None, cm.ACT_NONE)
            assert within(out[torch.tensor(at[sl], device="cuda", dtype=torch.long), :N], y, err)
        assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())


@pytest.mark.parametrize("M,N,K,act", [(1, 1, 1, cm.ACT_NONE), (16, 40, 130, cm.ACT_GELU), (17, 5003, 257, cm.ACT_RELU),
                                       (32, 700, 2048, cm.ACT_GELU), (32, 96, 9000, cm.ACT_NONE), (7, 40000, 512, cm.ACT_NONE),
                                       (3, 128, 1792, cm.ACT_GELU), (29, 20000, 64, cm.ACT_RELU), (33, 300, 300, cm.ACT_NONE),
                                       (64, 1024, 4096, cm.ACT_GELU), (128, 130, 2048, cm.ACT_RELU), (99, 515, 9000, cm.ACT_NONE),
                                       (129, 64, 512, cm.ACT_NONE)])
def test_kernel_for_few_rows(M, N, K, act):
    """K split over one to eight CTAs, one to many tiles, each number of rows; the same bits each time."""
    rng = np.random.default_rng(M + N + K)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1)
    y, err = reference(av, wv, bias, act)
    cm.clearmoe_debug_fp4_kernel(16, 0)
    try:
        for dtype in (torch.float32, torch.bfloat16):
            out = torch.full((M + 1, N + 3), float("nan"), device="cuda", dtype=dtype)
            cm.clearmoe_fp4_gemm(A, W, out[:M, :N], bias=bias, act=act)
            assert within(out[:M, :N], y, err)
            assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())
            again = torch.empty(M, N, device="cuda", dtype=dtype)
            cm.clearmoe_fp4_gemm(A, W, again, bias=bias, act=act)
            assert torch.equal(again, out[:M, :N])
        q = cm.fp4_matrix(M, N)
        q.q.fill_(0x33)
        cm.clearmoe_fp4_gemm(A, W, q, bias=bias, act=act)
        check_blocks(q, y, err)
    finally:
        cm.clearmoe_debug_fp4_kernel()


@pytest.mark.parametrize("kernel", [(256, 1), (128, 1)], indirect=True)
@pytest.mark.parametrize("M,N,K,pitch", [(300, 777, 64, 784), (257, 131, 500, 136), (1000, 8, 1024, 8), (513, 33, 2048, 64)])
def test_bf16_rows_by_bulk_copies(kernel, M, N, K, pitch):
    """Rows in whole 16-byte pieces whose last columns are not: nothing is written past them."""
    A, W, av, wv = make(np.random.default_rng(M), M, N, K)
    out = torch.full((M + 300, pitch), float("nan"), device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_fp4_gemm(A, W, out[:M, :N], act=cm.ACT_RELU)
    assert within(out[:M, :N], *reference(av, wv, None, cm.ACT_RELU))
    assert bool(out[M:].isnan().all()) and bool(out[:, N:].isnan().all())


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("M,N,pitch", [(100, 32, 40), (300, 100, 101), (77, 33, 36), (130, 1, 3), (65, 287, 290), (260, 64, 65), (1, 95, 97)])
@pytest.mark.parametrize("start", [0, 1, 2])
def test_bf16_rows_that_start_anywhere(kernel, M, N, pitch, start):
    """Rows at whole words, between them and by turns; nothing beside them is written."""
    A, W, av, wv = make(np.random.default_rng(M), M, N, 200)
    flat = torch.full((start + (M + 1) * pitch,), float("nan"), device="cuda", dtype=torch.bfloat16)
    out = flat[start:].view(M + 1, pitch)
    cm.clearmoe_fp4_gemm(A, W, out[:M, :N], act=cm.ACT_RELU)
    assert within(out[:M, :N], *reference(av, wv, None, cm.ACT_RELU))
    assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all()) and bool(flat[:start].isnan().all())
    if kernel != (16, 0):
        flat.fill_(float("nan"))
        at = torch.randperm(M, device="cuda").to(torch.int32)
        cm.clearmoe_fp4_grouped_gemm(A, [W] * 3, torch.tensor([0, M // 3, M // 2, M], dtype=torch.int32, device="cuda"), out[:M, :N], perm=at,
                                     act=cm.ACT_RELU)
        assert within(out[:M, :N][at.long()], *reference(av, wv, None, cm.ACT_RELU))
        assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all()) and bool(flat[:start].isnan().all())


@pytest.mark.parametrize("perm", [True, False])
@pytest.mark.parametrize("counts", [[0, 300, 1, 0, 129, 700], [1130], [3, 2, 0, 1], [128, 128, 256], [127, 1, 129, 255, 0, 77, 500, 41],
                                    [1] * 16])
@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
def test_every_kernel_grouped(kernel, counts, perm):
    rng = np.random.default_rng(77)
    N, K = 320, 640
    M, off = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    A, _, av, _ = make(rng, M, N, K)
    pairs = [make(rng, 1, N, K)[1::2] for _ in counts]
    at = rng.permutation(M) if perm else np.arange(M)
    for pad, dtype in ((0, torch.float32), (3, torch.bfloat16), (3, torch.float32)):
        out = torch.full((M + 1, N + pad), float("nan"), device="cuda", dtype=dtype)
        cm.clearmoe_fp4_grouped_gemm(A, [p[0] for p in pairs], torch.tensor(off, dtype=torch.int32, device="cuda"), out[:M, :N],
                                     perm=torch.tensor(at, dtype=torch.int32, device="cuda") if perm else None)
        for e in range(len(counts)):
            sl = slice(int(off[e]), int(off[e + 1]))
            y, err = reference(av[sl], pairs[e][1], None, cm.ACT_NONE)
            assert within(out[torch.tensor(at[sl], device="cuda", dtype=torch.long), :N], y, err)
        assert bool(out[M].isnan().all()) and bool(out[:, N:].isnan().all())


def test_grouped_rows_outside_the_offsets_are_left():
    """Offsets that end before A does (a padded batch): the rows behind the last group stay as they were."""
    rng = np.random.default_rng(3)
    A, W, av, wv = make(rng, 300, 96, 128)
    out = torch.full((300, 96), 7.0, device="cuda")
    cm.clearmoe_fp4_grouped_gemm(A, [W, W], torch.tensor([5, 100, 201], dtype=torch.int32, device="cuda"), out)
    y, err = reference(av, wv, None, cm.ACT_NONE)
    assert within(out[5:201], y[5:201], err[5:201])
    assert bool((out[:5] == 7).all()) and bool((out[201:] == 7).all())


@pytest.mark.parametrize("M,N,K", [(1, 128, 128), (130, 768, 192), (77, 200, 300), (4000, 1536, 384), (9, 1, 5), (3, 97, 64)])
def test_gemm_to_blocks(M, N, K):
    rng = np.random.default_rng(M + N + K)
    A, W, av, wv = make(rng, M, N, K)
    bias = dev(rng.standard_normal(N) * 0.1, torch.bfloat16)
    out = cm.fp4_matrix(M, N)
    out.q.fill_(0x33)
    cm.clearmoe_fp4_gemm(A, W, out, bias=bias, act=cm.ACT_GELU)
    check_blocks(out, *reference(av, wv, bias, cm.ACT_GELU))
    assert out.rows == M


@pytest.mark.parametrize("kernel", KERNELS + [(0, 0)], indirect=True)
@pytest.mark.parametrize("M", [4, 257])
def test_blocks_keep_their_scales(kernel, M):
    """Every block of A and W in a scale of its own, over several stages, tiles and words: one byte read from the wrong
    place is off by a power of two."""
    N, K = 320, 1536 + 96
    rng = np.random.default_rng(5)
    a = rng.standard_normal((M, K)) * np.repeat(2.0 ** rng.integers(-20, 20, (M, K // 32)), 32, 1)
    w = rng.standard_normal((N, K)) * np.repeat(2.0 ** rng.integers(-20, 20, (N, K // 32)), 32, 1)
    A, W, out = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K), torch.empty(M, N, device="cuda")
    cm.clearmoe_fp4_quantize(dev(w), W)
    wv = values(W)
    for kb in [None, *range(K // 32)]:  # all, then each block alone
        one = a if kb is None else np.where(np.arange(K) // 32 == kb, a, 0.0)
        cm.clearmoe_fp4_quantize(dev(one), A)
        cm.clearmoe_fp4_gemm(A, W, out)
        assert within(out, *reference(values(A), wv, None, cm.ACT_NONE))


@pytest.mark.parametrize("kernel", KERNELS + [(0, 0)], indirect=True)
@pytest.mark.parametrize("M", [3, 200])
def test_nan_stays_in_its_row_and_column(kernel, M):
    rng = np.random.default_rng(11)
    N, K = 200, 300
    x, w = rows_of(rng, M, K, 1.0), rows_of(rng, N, K, 0.5)
    x[1, 299], w[131, 5], w[7, 100] = np.inf, np.nan, -np.inf
    A, W, out = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K), torch.zeros(M, N, device="cuda")
    cm.clearmoe_fp4_quantize(dev(x), A)
    cm.clearmoe_fp4_quantize(dev(w), W)
    for act in (cm.ACT_NONE, cm.ACT_RELU, cm.ACT_GELU):
        cm.clearmoe_fp4_gemm(A, W, out, act=act)
        want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        want[1], want[:, 131], want[:, 7] = True, True, True
        assert torch.equal(out.isnan(), want)
        q = cm.fp4_matrix(M, N)
        cm.clearmoe_fp4_gemm(A, W, q, act=act)
        blocks = torch.nn.functional.pad(want, (0, -N % 32)).view(M, -1, 32).any(2).repeat_interleave(32, 1)[:, :N]
        assert torch.equal(values(q).isnan(), blocks)


@pytest.mark.parametrize("kernel", KERNELS + [(0, 0)], indirect=True)
@pytest.mark.parametrize("M", [2, 130])
def test_scales_at_the_ends_of_their_range(kernel, M):
    """Values near fp32's ends, and past them as rounded, whose products are not: the scales are applied together. An input
    past fp32 is an infinity: NaN."""
    def values(m):  # in float64: 4 2^126 is past fp32
        c = R.unpack(m.q.cpu().numpy(), m.cols)[0]
        s = np.repeat(R.scale_bytes(m.scale.cpu().numpy(), m.rows, m.cols), 32, 1)[:, :m.cols].astype(np.float64)
        return torch.from_numpy(np.where(s == 255, np.nan, R.e2m1_value(c) * 2.0 ** (s - 127))).cuda()

    N, K = 70, 128
    rng = np.random.default_rng(13)
    a = rng.standard_normal((M, K))
    w = rng.standard_normal((N, K))
    for p, q in ((120, -118), (-120, 118), (100, -3), (-126, 126)):
        A, W, out = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K), torch.empty(M, N, device="cuda")
        cm.clearmoe_fp4_quantize(dev(a * 2.0 ** p), A)
        cm.clearmoe_fp4_quantize(dev(w * 2.0 ** q), W)
        cm.clearmoe_fp4_gemm(A, W, out)
        y, err = reference(values(A), values(W), None, cm.ACT_NONE)
        fine = ~y.isnan()
        assert torch.equal(~out.isnan(), fine) and float(fine.float().mean()) > 0.8
        assert within(out[fine], y[fine], err[fine])


def test_two_products_in_a_row():
    """A whole FFN whose hidden state is in 4-bit blocks, on a stream of its own and then replayed from a graph."""
    rng = np.random.default_rng(17)
    T, d, H = 300, 192, 768
    W1, W2 = (rows_of(rng, *s, 0.0) * 0.05 for s in ((H, d), (d, H)))
    w1, w2, xq, zq = cm.fp4_matrix(H, d), cm.fp4_matrix(d, H), cm.fp4_matrix(T, d), cm.fp4_matrix(T, H)
    x, b1, b2 = torch.empty(T, d, device="cuda"), dev(rng.standard_normal(H) * 0.1), dev(rng.standard_normal(d) * 0.1)
    out = torch.empty(T, d, device="cuda")
    cm.clearmoe_fp4_quantize(dev(W1), w1)
    cm.clearmoe_fp4_quantize(dev(W2), w2)

    def ffn():
        cm.clearmoe_fp4_quantize(x, xq)
        cm.clearmoe_fp4_gemm(xq, w1, zq, bias=b1, act=cm.ACT_GELU)
        cm.clearmoe_fp4_gemm(zq, w2, out, bias=b2)

    def check():
        torch.cuda.synchronize()
        check_blocks(zq, *reference(values(xq), values(w1), b1, cm.ACT_GELU))
        assert within(out, *reference(values(zq), values(w2), b2, cm.ACT_NONE))

    side = torch.cuda.Stream()
    x.copy_(dev(rows_of(rng, T, d, 1.0)))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ffn()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffn()
    for _ in range(2):
        x.copy_(dev(rows_of(rng, T, d, 1.0)))
        out.zero_()
        graph.replay()
        check()


def test_two_streams_and_two_graphs():
    """Calls share nothing: products of two streams at once, and two graphs replayed side by side."""
    rng = np.random.default_rng(23)
    sets = []
    for M, N, K in ((500, 640, 1024), (20, 640, 1024), (500, 640, 1024), (20, 640, 1024)):
        A, W, av, wv = make(rng, M, N, K)
        sets.append((A, W, torch.zeros(M, N, device="cuda"), reference(av, wv, None, cm.ACT_NONE)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(20):
        for s, (A, W, out, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                cm.clearmoe_fp4_gemm(A, W, out)
    torch.cuda.synchronize()
    for _, _, out, ref in sets:
        assert within(out, *ref)
        out.zero_()
    graphs = []
    for A, W, out, _ in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            cm.clearmoe_fp4_gemm(A, W, out)
    for _ in range(20):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, _, out, ref in sets:
        assert within(out, *ref)


@pytest.mark.parametrize("kernel", KERNELS, indirect=True)
@pytest.mark.parametrize("blocks", [False, True])
def test_waits_that_run_out(kernel, blocks):
    """Under limits of 1 to 200 microseconds the kernels give up between their copies, let what is in flight land, and
    return; the call reports CLEARMOE_ETIMEOUT or completes, and the next call with the usual limit gives the same bits."""
    M = 100 if kernel[0] == 16 else 3000
    A, W, av, wv = make(np.random.default_rng(29), M, 1024, 16384)
    out = cm.fp4_matrix(M, 1024) if blocks else torch.empty(M, 1024, device="cuda", dtype=torch.bfloat16)
    bits = out.q if blocks else out
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cm.clearmoe_fp4_gemm(A, W, out, status=status)
    want, gave_up = bits.clone(), []
    try:
        for limit in (1_000, 4_000, 16_000, 50_000, 200_000):
            for _ in range(4):
                cm.clearmoe_debug_fp4_wait(limit)
                cm.clearmoe_fp4_gemm(A, W, out, status=status)
                cm.clearmoe_fp4_gemm(A, W, out, status=status)
                st = status.item()
                assert st in (0, cm.ETIMEOUT)
                gave_up.append(st == cm.ETIMEOUT)
                status.zero_()
                cm.clearmoe_debug_fp4_wait()
                bits.zero_()
                cm.clearmoe_fp4_gemm(A, W, out, status=status)
                assert torch.equal(bits, want) and status.item() == 0
    finally:
        cm.clearmoe_debug_fp4_wait()
    assert kernel[0] == 16 or any(gave_up)


@pytest.mark.parametrize("kernel", [(256, 1)], indirect=True)
@pytest.mark.parametrize("counts,N", [([200, 0, 0, 0], 512), ([3000, 2120], 1280)])
def test_waits_that_run_out_in_halves_of_tiles(kernel, counts, N):
    """The same of tiles in halves, the first and the last that a pair has."""
    M, E = sum(counts), len(counts)
    A, W, *_ = make(np.random.default_rng(30), M, N, 8192)
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    out, status = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32, device="cuda")
    cm.clearmoe_fp4_grouped_gemm(A, [W] * E, off, out, status=status)
    want = out.clone()
    try:
        for limit in (200, 1_000, 4_000, 12_000, 16_000, 24_000):
            for _ in range(4):
                cm.clearmoe_debug_fp4_wait(limit)
                cm.clearmoe_fp4_grouped_gemm(A, [W] * E, off, out, status=status)
                cm.clearmoe_fp4_grouped_gemm(A, [W] * E, off, out, status=status)
                assert status.item() in (0, cm.ETIMEOUT)
                status.zero_()
                cm.clearmoe_debug_fp4_wait()
                out.zero_()
                cm.clearmoe_fp4_grouped_gemm(A, [W] * E, off, out, status=status)
                assert torch.equal(out, want) and status.item() == 0
    finally:
        cm.clearmoe_debug_fp4_wait()


@pytest.mark.parametrize("M,N,K", [(3, 2048, 16384), (300, 512, 1024)])
def test_weights_and_rows_just_written(M, N, K):
    """Weights and rows quantised by the kernels right before the product, new ones each time: what is asked for into L2
    before they are written is not what the product reads."""
    rng = np.random.default_rng(31)
    xs, ws = [dev(rows_of(rng, M, K, 1.0)) for _ in range(2)], [dev(rows_of(rng, N, K, 0.5)) for _ in range(2)]
    A, W, want = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K), []
    for x, w in zip(xs, ws):
        cm.clearmoe_fp4_quantize(x, A)
        cm.clearmoe_fp4_quantize(w, W)
        torch.cuda.synchronize()
        want.append(torch.empty(M, N, device="cuda"))
        cm.clearmoe_fp4_gemm(A, W, want[-1])
        torch.cuda.synchronize()
        assert within(want[-1], *reference(values(A), values(W), None, cm.ACT_NONE))
    outs = [torch.empty(M, N, device="cuda") for _ in range(40)]
    for i, out in enumerate(outs):
        cm.clearmoe_fp4_quantize(xs[i & 1], A)
        cm.clearmoe_fp4_quantize(ws[i & 1], W)
        cm.clearmoe_fp4_gemm(A, W, out)
    assert all(torch.equal(out, want[i & 1]) for i, out in enumerate(outs))


@pytest.mark.parametrize("kernel", KERNELS[:-1], indirect=True)
def test_offsets_of_a_routing_that_gave_up(kernel):
    """Offsets that descend or lie outside the rows, and rows outside the output, are held to the buffers: each row stored
    is its expert's or stays."""
    rng = np.random.default_rng(37)
    M, N, K = 700, 96, 128
    A, W, av, wv = make(rng, M, N, K)
    y, err = reference(av, wv, None, cm.ACT_NONE)
    for off in ([0, -5, 2 ** 31 - 1, 3, 9], [500, 20, 300, 650, -1], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        out = torch.full((M + 1, N), 7.0, device="cuda")
        cm.clearmoe_fp4_grouped_gemm(A, [W] * 4, torch.tensor(off, dtype=torch.int32, device="cuda"), out[:M])
        lo = min(max(off[0], 0), M)
        hi = min(max(max(off), 0), M)
        assert within(out[lo:hi], y[lo:hi], err[lo:hi])
        assert bool((out[:lo] == 7).all()) and bool((out[hi:] == 7).all())
    perm = torch.arange(M, dtype=torch.int32, device="cuda")
    perm[::3] = -1
    perm[1::3] = M
    out = torch.full((M + 1, N), 7.0, device="cuda")
    cm.clearmoe_fp4_grouped_gemm(A, [W], torch.tensor([0, M], dtype=torch.int32, device="cuda"), out[:M], perm=perm)
    assert within(out[2:M:3], y[2::3], err[2::3])
    assert bool((out[0::3] == 7).all()) and bool((out[1::3] == 7).all())


def test_long_sums():
    """K of 300,007 columns: exact values (integers of few bits) in sums that fp32 holds exactly."""
    rng = np.random.default_rng(41)
    for M, N in ((1, 40), (40, 130)):
        K = 300_007
        a, w = rng.integers(-1, 2, (M, K)).astype(np.float32), rng.integers(-1, 2, (N, K)).astype(np.float32)
        A, W, out = cm.fp4_matrix(M, K), cm.fp4_matrix(N, K), torch.empty(M, N, device="cuda")
        cm.clearmoe_fp4_quantize(dev(a), A)
        cm.clearmoe_fp4_quantize(dev(w), W)
        cm.clearmoe_fp4_gemm(A, W, out)
        assert np.array_equal(f64(out), a.astype(np.float64) @ w.T.astype(np.float64))


def test_empty_matrices_are_refused():
    with pytest.raises(cm.ClearMoEError):
        cm.clearmoe_fp4_quantize(torch.empty(0, 64, device="cuda"), cm.fp4_matrix(0, 64))
    with pytest.raises(cm.ClearMoEError):
        cm.clearmoe_rms_norm(torch.empty(0, 64, device="cuda"), torch.empty(0, 64, device="cuda"))


def test_matrices_of_another_gpu_are_refused():
    x, A, W, q = torch.randn(5, 64, device="cuda"), cm.fp4_matrix(5, 64), cm.fp4_matrix(9, 64), cm.fp4_matrix(5, 9)
    out, e = torch.empty(5, 9, device="cuda"), cm.fp8_rows(5, 64)
    for m in (A, W, q, e):
        assert m.get_device() == 0
        m.c.device = 1  # as if it lay there
        for call in (lambda: cm.clearmoe_fp4_quantize(x, A), lambda: cm.clearmoe_fp4_gemm(A, W, q), lambda: cm.clearmoe_fp4_gemm(A, W, out),
                     lambda: cm.clearmoe_rms_norm(x, A), lambda: cm.clearmoe_rms_norm(x, e), lambda: cm.clearmoe_fp4_dequantize(A, x)):
            if any(c.cell_contents is m for c in call.__closure__):
                with pytest.raises(ValueError, match="GPU 1"):
                    call()
        m.c.device = 0
