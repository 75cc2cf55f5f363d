"""Matrices in 8-bit blocks come in two kinds, whose scales have one row per row or per 128 rows. The library sees addresses
only, so the binding refuses the wrong kind before any call: taken for the other, the rows of one would be read or written
past the other's scales. Without a GPU: matrices without storage, which the library would refuse another way."""
import ctypes

import pytest

from paper_2606_28516_gb300 import build, clearmoe as cm


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def matrix(rows, cols, weight):
    m = object.__new__(cm.Fp8Matrix)
    m.q = m.scale = None
    m.rows, m.cols, m.weight = rows, cols, weight
    m.c = cm.clearmoe_fp8(None, None, rows, cols)
    m.ref, m.addr = ctypes.pointer(m.c), ctypes.addressof(m.c)
    return m


class Dense:  # a CUDA tensor as far as the binding looks
    is_cuda = True

    def __init__(self, *shape, dtype="torch.float32"):
        self.shape, self.dtype = shape, dtype

    def stride(self):
        return self.shape[1], 1

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0


class Stream:
    cuda_stream = 0


def rows(*s):
    return matrix(*s, False)


def weight(*s):
    return matrix(*s, True)


GOOD = [
    lambda: cm.clearmoe_fp8_quantize_rows(Dense(300, 64), rows(300, 64), stream=Stream()),
    lambda: cm.clearmoe_fp8_quantize_weight(Dense(300, 64), weight(300, 64), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(rows(300, 64), weight(200, 64), Dense(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(rows(300, 64), weight(200, 64), rows(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_grouped_gemm(rows(300, 64), [weight(200, 64)] * 2, Dense(3, 1, dtype="torch.int32"),
                                         Dense(300, 200), stream=Stream()),
]
WRONG = [
    lambda: cm.clearmoe_fp8_quantize_rows(Dense(300, 64), weight(300, 64), stream=Stream()),
    lambda: cm.clearmoe_fp8_quantize_rows(Dense(300, 64), weight(300, 64), gather=Dense(300, 1), stream=Stream()),
    lambda: cm.clearmoe_fp8_quantize_weight(Dense(300, 64), rows(300, 64), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(weight(300, 64), weight(200, 64), Dense(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(rows(300, 64), rows(200, 64), Dense(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(rows(300, 64), weight(200, 64), weight(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_gemm(weight(300, 64), weight(200, 64), rows(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_grouped_gemm(weight(300, 64), [weight(200, 64)] * 2, Dense(3, 1), Dense(300, 200), stream=Stream()),
    lambda: cm.clearmoe_fp8_grouped_gemm(rows(300, 64), [weight(200, 64), rows(200, 64)], Dense(3, 1), Dense(300, 200),
                                         stream=Stream()),
]


@pytest.mark.parametrize("call", GOOD)
def test_the_right_kind_reaches_the_library(call):
    with pytest.raises(cm.ClearMoEError):  # which refuses matrices without storage
        call()


@pytest.mark.parametrize("call", WRONG)
def test_the_wrong_kind_is_refused(call):
    with pytest.raises(ValueError, match="8-bit blocks of"):
        call()


def indices(n, dtype="torch.int32"):
    return Dense(n, 1, dtype=dtype)


@pytest.mark.parametrize("dtype,gather,offsets,perm,status", [
    ("torch.int32", 301, 4, 299, 0), ("torch.int64", 300, 3, 300, 1), ("torch.int16", 300, 3, 300, 1), ("torch.float32", 300, 3, 300, 1)])
def test_indices_of_another_type_or_number_are_refused(dtype, gather, offsets, perm, status):
    """Kernels read them as int32: of a narrower type past their end, of a wider one other rows."""
    A, W, out = rows(300, 64), weight(200, 64), Dense(300, 200)
    fine = dict(offsets=indices(3), perm=indices(300))
    for name, n in (("offsets", offsets), ("perm", perm)):
        kw = {**fine, name: indices(n, dtype)}
        with pytest.raises(ValueError, match=name + " must be int32"):
            cm.clearmoe_fp8_grouped_gemm(A, [W] * 2, out=out, stream=Stream(), **kw)
    with pytest.raises(ValueError, match="gather must be int32"):
        cm.clearmoe_fp8_quantize_rows(Dense(1000, 64), A, gather=indices(gather, dtype), stream=Stream())
    for o in (out, rows(300, 200)):
        with pytest.raises(ValueError, match="status must be int32"):
            cm.clearmoe_fp8_gemm(A, W, o, status=indices(status, dtype), stream=Stream())
    with pytest.raises(ValueError, match="status must be int32"):
        cm.clearmoe_fp8_grouped_gemm(A, [W] * 2, out=out, stream=Stream(), status=indices(status, dtype), **fine)
    with pytest.raises(cm.ClearMoEError):  # these reach the library
        cm.clearmoe_fp8_grouped_gemm(A, [W] * 2, out=out, stream=Stream(), status=indices(1), **fine)
    with pytest.raises(ValueError):
        cm.clearmoe_fp8_grouped_gemm(A, [], out=out, stream=Stream(), **fine)
