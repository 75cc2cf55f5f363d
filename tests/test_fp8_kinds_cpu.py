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
    is_cuda, dtype = True, "torch.float32"

    def __init__(self, *shape):
        self.shape = shape

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
    lambda: cm.clearmoe_fp8_grouped_gemm(rows(300, 64), [weight(200, 64)] * 2, Dense(3, 1), Dense(300, 200), stream=Stream()),
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
