"""4-bit blocks and the norm without a GPU: the tests' own reference, what the library and the binding refuse before any
call, and the rules that their kernels' sources keep."""
import ctypes
import pathlib
import re

import numpy as np
import pytest

import fp4_ref as R
from paper_2606_28516_gb300 import build, clearmoe as cm

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_reference_rounds_to_nearest_even():
    v = np.array([0, .25, .250001, .75, 1.25, 1.75, 2.5, 2.500001, 3.5, 5, 5.00001, 6, -5, -.2])
    assert R.e2m1_value(R.e2m1_code(v)).tolist() == [0, 0, .5, 1, 1, 2, 2, 3, 4, 4, 6, 6, -4, 0]
    assert R.scale_byte(6.0) == 127 and R.scale_byte(6.0000001) == 128 and R.scale_byte(0.0) == 0 and R.scale_byte(np.inf) == 255
    s = np.arange(2 * 3 * 512).reshape(2, 3, 512)
    assert R.scale_bytes(s, 256, 384)[133, 9] == 1 * 1536 + 2 * 512 + 16 * 5 + 1  # row 5 of tile 1, block 1 of tile 2
    assert R.scale_bytes(s, 256, 384)[97, 0] == 16 * 1 + 4 * 3


A32 = 0x1000  # an aligned address that nothing follows: every call below is refused before


def fp4(rows=4, cols=64, q=A32, scale=A32):
    return cm.clearmoe_fp4(q, scale, rows, cols)


def test_library_refuses():
    L = cm.lib()
    P = ctypes.byref
    good = fp4()
    for bad in (fp4(rows=0), fp4(cols=0), fp4(rows=(1 << 30) + 1), fp4(cols=(1 << 24) + 1), fp4(q=None), fp4(scale=None),
                fp4(q=A32 + 16), fp4(scale=A32 + 4)):
        assert L.clearmoe_fp4_quantize(A32, 4, cm.F32, 64, None, P(bad), None) == cm.EINVAL
        assert L.clearmoe_fp4_dequantize(P(bad), A32, cm.F32, 64, None) == cm.EINVAL
        assert L.clearmoe_fp4_gemm(P(bad), P(good), None, A32, cm.F32, 4, None) == cm.EINVAL
        assert L.clearmoe_fp4_gemm(P(good), P(bad), None, A32, cm.F32, 1 << 28, None) == cm.EINVAL
        assert L.clearmoe_fp4_gemm_fp4(P(good), P(good), None, P(bad), None) == cm.EINVAL
    q = lambda x=A32, n=4, dt=cm.F32, ld=64, g=None: L.clearmoe_fp4_quantize(x, n, dt, ld, g, P(good), None)  # noqa: E731
    assert q(x=None) == q(n=3) == q(n=0) == q(dt=7) == q(ld=63) == q(x=A32 + 2) == q(g=A32 + 1) == q(ld=(1 << 30) + 1) == cm.EINVAL
    assert q(x=A32 + 1, dt=cm.BF16) == cm.EINVAL
    g = lambda A=good, W=good, e=None, o=A32, dt=cm.F32, ld=4: L.clearmoe_fp4_gemm(P(A), P(W), e, o, dt, ld, None)  # noqa: E731
    assert g(o=None) == g(dt=2) == g(ld=3) == g(o=A32 + 2) == g(W=fp4(cols=65)) == g(W=fp4(rows=(1 << 24) + 1), ld=1 << 26) == cm.EINVAL
    epi = lambda *a: P(cm.clearmoe_fp8_epilogue(*a))  # noqa: E731
    assert g(e=epi(None, cm.F32, 5, None)) == g(e=epi(A32, 9, cm.ACT_NONE, None)) == g(e=epi(A32 + 2, cm.F32, cm.ACT_NONE, None)) == cm.EINVAL
    assert g(e=epi(None, cm.F32, cm.ACT_NONE, A32 + 2)) == cm.EINVAL
    assert L.clearmoe_fp4_gemm_fp4(P(good), P(good), None, P(fp4(cols=5)), None) == cm.EINVAL
    arr = (cm.clearmoe_fp4 * 2)(good, fp4(rows=5))
    gg = lambda W=arr, E=1, off=A32, perm=None, ld=4: L.clearmoe_fp4_grouped_gemm(P(good), W, E, off, perm, None, A32, cm.F32, ld, None)  # noqa: E731
    assert gg(E=0) == gg(E=17) == gg(W=None) == gg(off=None) == gg(off=A32 + 2) == gg(perm=A32 + 2) == gg(E=2) == gg(ld=3) == cm.EINVAL
    assert L.clearmoe_debug_fp4_kernel(100, 0) == L.clearmoe_debug_fp4_kernel(192, 1) == L.clearmoe_debug_fp4_kernel(256, 0) == cm.EINVAL
    assert L.clearmoe_debug_fp4_kernel(0, 0) == cm.OK
    assert L.clearmoe_debug_fp4_wait(-1) == L.clearmoe_debug_fp4_wait(1_000_000_001) == cm.EINVAL
    assert L.clearmoe_debug_fp4_wait(0) == cm.OK


def norm(**kw):
    a = dict(x=A32, residual=A32, sum=A32, weight=A32, ldx=64, ldr=64, lds=64, rows=4, cols=64, dtype=cm.F32, weight_dtype=cm.F32,
             eps=1e-6) | kw
    return cm.clearmoe_norm(**a)


@pytest.mark.parametrize("kw", [dict(x=None), dict(rows=0), dict(rows=(1 << 30) + 1), dict(cols=0), dict(dtype=2), dict(weight_dtype=5),
                                dict(ldx=63), dict(ldr=63), dict(lds=63), dict(x=A32 + 2, sum=None), dict(residual=A32 + 2),
                                dict(sum=A32 + 1, dtype=cm.BF16), dict(weight=A32 + 2), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(eps=float("inf")), dict(ldx=65), dict(ldr=65), dict(ldx=(1 << 30) + 1)])
def test_norm_refuses(kw):
    L, n = cm.lib(), norm(**kw)
    P = ctypes.byref
    assert L.clearmoe_rms_norm(P(n), A32 + 4096, cm.F32, 64, None) == cm.EINVAL
    assert L.clearmoe_rms_norm_fp8(P(n), P(cm.clearmoe_fp8(A32, A32, 4, 64)), None) == cm.EINVAL
    assert L.clearmoe_rms_norm_fp4(P(n), P(fp4()), None) == cm.EINVAL


def test_norm_refuses_outputs():
    L, P = cm.lib(), ctypes.byref
    f = lambda o=A32 + 4096, dt=cm.F32, ld=64, **kw: L.clearmoe_rms_norm(P(norm(**kw)), o, dt, ld, None)  # noqa: E731
    assert f(o=None) == f(dt=4) == f(ld=63) == f(o=A32 + 4098) == f(o=A32) == cm.EINVAL  # the last: over the sum
    assert f(o=A32, sum=None, dt=cm.BF16) == f(o=A32, sum=None, ld=65) == cm.EINVAL
    assert f(cols=cm.NORM_MAX + 1, ldx=1 << 20, ldr=1 << 20, lds=1 << 20, ld=1 << 20) == cm.EUNSUPPORTED
    for m in (cm.clearmoe_fp8(A32, A32, 5, 64), cm.clearmoe_fp8(A32, A32, 4, 65), cm.clearmoe_fp8(A32 + 1, A32, 4, 64)):
        assert L.clearmoe_rms_norm_fp8(P(norm()), P(m), None) == cm.EINVAL
    for m in (fp4(rows=5), fp4(cols=65), fp4(q=A32 + 1)):
        assert L.clearmoe_rms_norm_fp4(P(norm()), P(m), None) == cm.EINVAL
    assert L.clearmoe_rms_norm(None, A32, cm.F32, 64, None) == cm.EINVAL


class Dense:  # a CUDA tensor as far as the binding looks
    is_cuda = True

    def __init__(self, *shape, dtype="torch.float32", step=1):
        self.shape, self.dtype, self.step = shape, dtype, step

    def stride(self):
        return self.shape[1] * self.step, self.step

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return True

    def element_size(self):
        return 1

    def data_ptr(self):
        return 0


class Stream:
    cuda_stream = 0


def matrix4(rows, cols):
    return cm.Fp4Matrix(Dense(rows, cm.fp4_pitch(cols)), Dense(-(-rows // 128), -(-cols // 128), 512), rows, cols)


def matrix8(rows, cols, weight=False):
    return cm.Fp8Matrix(Dense(rows, cm.fp8_pitch(cols)), Dense(-(-rows // 128) if weight else rows, cm.fp8_scale_pitch(cols)), rows, cols,
                        weight)


S = dict(stream=Stream())
I32 = "torch.int32"
GOOD = [  # these reach the library, which refuses their null pointers
    lambda: cm.clearmoe_fp4_quantize(Dense(300, 64), matrix4(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(7, 64), matrix4(300, 64), gather=Dense(300, dtype=I32), **S),
    lambda: cm.clearmoe_fp4_dequantize(matrix4(4, 64), Dense(4, 64), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), Dense(4, 9), bias=Dense(9), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), matrix4(4, 9), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64)] * 2, Dense(3, dtype=I32), Dense(4, 9), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), residual=Dense(4, 64), weight=Dense(64, dtype="torch.bfloat16"), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), matrix8(4, 64), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), matrix4(4, 64), **S),
]


@pytest.mark.parametrize("call", GOOD)
def test_calls_that_reach_the_library(call):
    with pytest.raises(cm.ClearMoEError) as e:
        call()
    assert e.value.code == cm.EINVAL


BAD = [
    lambda: cm.clearmoe_fp4_quantize(Dense(300, 64), matrix8(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(299, 64), matrix4(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(300, 65), matrix4(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(300, 64, step=2), matrix4(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(300, 64, dtype="torch.float16"), matrix4(300, 64), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(7, 64), matrix4(300, 64), gather=Dense(299, dtype=I32), **S),
    lambda: cm.clearmoe_fp4_quantize(Dense(7, 64), matrix4(300, 64), gather=Dense(300, dtype="torch.int64"), **S),
    lambda: cm.clearmoe_fp4_dequantize(matrix8(4, 64), Dense(4, 64), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix8(4, 64), matrix4(9, 64), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix8(9, 64, True), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), Dense(4, 8), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), Dense(4, 9), bias=Dense(8), **S),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), Dense(4, 9), status=Dense(1), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64), matrix8(9, 64)], Dense(3, dtype=I32), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [], Dense(1, dtype=I32), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64)], Dense(3, dtype=I32), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64)], None, Dense(4, 9), **S),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64)], Dense(2, dtype=I32), Dense(4, 9), perm=Dense(3, dtype=I32), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 63), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), residual=Dense(4, 64, dtype="torch.bfloat16"), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), residual=Dense(1, 64), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), sum_out=Dense(4, 64, dtype="torch.bfloat16"), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), weight=Dense(63), **S),
    lambda: cm.clearmoe_rms_norm(Dense(64), Dense(64), **S),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), matrix8(4, 64, True), **S),
    # calls on 8-bit blocks refuse these matrices
    lambda: cm.clearmoe_fp8_quantize_rows(Dense(4, 64), matrix4(4, 64), **S),
    lambda: cm.clearmoe_fp8_quantize_weight(Dense(4, 64), matrix4(4, 64), **S),
    lambda: cm.clearmoe_fp8_dequantize(matrix4(4, 64), Dense(4, 64), **S),
    lambda: cm.clearmoe_fp8_gemm(matrix4(4, 64), matrix8(9, 64, True), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp8_gemm(matrix8(4, 64), matrix4(9, 64), Dense(4, 9), **S),
    lambda: cm.clearmoe_fp8_grouped_gemm(matrix8(4, 64), [matrix4(9, 64)], Dense(2, dtype=I32), Dense(4, 9), **S),
    # buffers of another size
    lambda: cm.Fp4Matrix(Dense(4, 31), Dense(1, 1, 512), 4, 64),
    lambda: cm.Fp4Matrix(Dense(4, 32), Dense(1, 1, 511), 4, 64),
    lambda: cm.Fp4Matrix(Dense(129, 32), Dense(1, 1, 512), 129, 64),
]


@pytest.mark.parametrize("call", BAD)
def test_calls_that_the_binding_refuses(call):
    with pytest.raises(ValueError):
        call()


class Elsewhere(Dense):
    def get_device(self):
        return 1


class Stream0(Stream):
    device_index = 0


def matrix4_elsewhere(rows, cols):
    return cm.Fp4Matrix(Elsewhere(rows, cm.fp4_pitch(cols)), Elsewhere(-(-rows // 128), -(-cols // 128), 512), rows, cols)


def matrix8_elsewhere(rows, cols):
    return cm.Fp8Matrix(Elsewhere(rows, cm.fp8_pitch(cols)), Elsewhere(rows, cm.fp8_scale_pitch(cols)), rows, cols)


@pytest.mark.parametrize("call", [
    lambda: cm.clearmoe_fp4_quantize(Elsewhere(4, 64), matrix4(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_fp4_dequantize(matrix4(4, 64), Elsewhere(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), Dense(4, 9), bias=Elsewhere(9), stream=Stream0()),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64)], Elsewhere(2, dtype=I32), Dense(4, 9), stream=Stream0()),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), Dense(4, 64), residual=Elsewhere(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_fp4_quantize(Dense(4, 64), matrix4_elsewhere(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_fp4_quantize(Dense(9, 64), matrix4_elsewhere(4, 64), gather=Dense(4, dtype=I32), stream=Stream0()),
    lambda: cm.clearmoe_fp4_dequantize(matrix4_elsewhere(4, 64), Dense(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_fp4_gemm(matrix4_elsewhere(4, 64), matrix4(9, 64), Dense(4, 9), stream=Stream0()),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4_elsewhere(9, 64), matrix4(4, 9), stream=Stream0()),
    lambda: cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), matrix4_elsewhere(4, 9), stream=Stream0()),
    lambda: cm.clearmoe_fp4_grouped_gemm(matrix4(4, 64), [matrix4(9, 64), matrix4_elsewhere(9, 64)], Dense(3, dtype=I32), Dense(4, 9),
                                         stream=Stream0()),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), matrix4_elsewhere(4, 64), stream=Stream0()),
    lambda: cm.clearmoe_rms_norm(Dense(4, 64), matrix8_elsewhere(4, 64), stream=Stream0()),
    lambda: cm.Fp4Matrix(Elsewhere(4, 32), Dense(1, 1, 512), 4, 64),
])
def test_tensors_of_another_gpu_are_refused(call):
    with pytest.raises(ValueError, match="GPU 1"):
        call()


def source(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


@pytest.mark.parametrize("name", ["fp4.cu", "fp4_gemm.cu", "fp4_gemm2.cu", "fp4_few.cu", "norm.cu"])
def test_reads_and_releases_after_the_wait(name):
    """Every kernel waits for its predecessor before it releases its successor (a run cannot show that one does not)."""
    s = source(name)
    for body in s.split("__global__ void")[1:]:
        body = body[:body.index("cudaError_t launch")] if "cudaError_t launch" in body else body
        wait = body.index("pdl_wait();")
        assert "pdl_launch_dependents();" not in body[:wait]


@pytest.mark.parametrize("name", ["fp4.cu", "fp4_gemm.cuh", "fp4_gemm.cu", "fp4_gemm2.cu", "fp4_few.cu", "norm.cu", "lane16.cuh"])
def test_no_loads_for_data_that_never_changes(name):
    """A kernel that starts beside its predecessor lives while that one still writes: what ld.global.nc must not read."""
    assert "__ldg(" not in source(name) and ".nc" not in source(name) and "__restrict__" not in source(name)


def kernel(name):
    s = source(name)
    return s[s.index("__global__ void"):s.index("cudaError_t launch")]


@pytest.mark.parametrize("name,drains,last", [
    ("fp4_gemm.cu", ["mbar_wait_warp(full_bar(s), (par >> s) & 1", "mbar_wait_warp(drain_bar, 0"], "tmem_dealloc(tmem"),
    ("fp4_few.cu", ["mbar_wait_warp(full_bar(s), (par >> s) & 1", "mbar_wait_warp(done_bar, 0"], "tmem_dealloc(tmem"),
    ("fp4_gemm2.cu", ["mbar_wait_warp(full_bar(s), (k / STAGES) & 1", "mbar_wait_warp(drain_bar, 0"], "tcgen05.dealloc"),
])
def test_copies_and_mmas_end_before_tensor_memory_is_freed(name, drains, last):
    """Each role waits for what it started; then all meet; then the memory is freed, in no role's branch."""
    s = kernel(name)
    free = s.index(last)
    meet = s.rindex("__syncthreads();", 0, free)
    for d in drains:
        assert s.count(d) == 1 and s.index(d) < meet, d
    assert "return;" not in re.sub(r"auto prefetch = .*?\n        };", "", s[:meet], flags=re.S)  # no thread leaves early
    if name == "fp4_gemm2.cu":
        assert meet < s.index("cluster_sync();", meet) < free


@pytest.mark.parametrize("name", ["fp4_gemm.cu", "fp4_gemm2.cu", "fp4_few.cu"])
def test_tensor_memory_accesses_follow_a_fence(name):
    s = kernel(name)
    waits = [m.start() for m in re.finditer(r"\bmbar_wait_warp\(", s)]
    uses = [m for m in re.finditer(r"\b(CM_TMEM_LD_X\d+|umma2?_mxf4|umma_few|tmem_cp_scales<\d>)\(", s)]
    assert uses and not re.search(r"\bmbar_wait\(", s)
    for m in uses:
        last = max(w for w in waits if w < m.start())
        assert "tc_fence_after();" in s[last:m.start()], m.group()
