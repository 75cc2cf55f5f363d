"""The compiled part of the binding: it builds, takes integers and None, and refuses other arguments before any call."""
import pytest

from paper_2606_28516_gb300 import build, clearmoe as cm


@pytest.fixture(scope="module")
def calls():
    build.build()
    return cm._bind_calls()


def test_arguments(calls):
    assert calls.quantize_rows(None, cm.F32, 4, None, None, None) == cm.EINVAL  # reaches the library, which refuses it
    assert calls.gemm(None, None, None, cm.F32, cm.ACT_NONE, None, None, cm.F32, 4, None) == cm.EINVAL
    assert calls.gemm_fp8(None, None, None, cm.F32, cm.ACT_NONE, None, None, None) == cm.EINVAL
    assert calls.ffn_few(None, None, 1, None, None, None) == cm.EINVAL
    assert calls.ffn_fp8(None, None, 1, None, None, None) == cm.EINVAL
    for f, n in ((calls.quantize_rows, 6), (calls.gemm, 10), (calls.gemm_fp8, 8), (calls.ffn_few, 6), (calls.ffn_fp8, 6)):
        with pytest.raises(TypeError):
            f(*[0] * (n - 1))
        with pytest.raises(TypeError):
            f(*[0] * (n + 1))
        with pytest.raises(TypeError):
            f(*[0] * (n - 1), "0")
        with pytest.raises(TypeError):
            f(*[0] * (n - 1), 0.5)


def test_errors_name_their_call(calls):
    m = cm.clearmoe_fp8(None, None, 4, 4)

    class Rows:
        import ctypes
        rows, cols, addr = 4, 4, ctypes.addressof(m)

    class Posing:  # a CUDA matrix as far as the binding looks
        shape, is_cuda, dtype = (4, 4), True, "torch.float32"

        def stride(self):
            return 4, 1

        def data_ptr(self):
            return 0

    class Stream:
        cuda_stream = 0

    with pytest.raises(cm.ClearMoEError, match="clearmoe_fp8_quantize_rows"):
        cm.clearmoe_fp8_quantize_rows(Posing(), Rows(), stream=Stream())
    with pytest.raises(cm.ClearMoEError, match="clearmoe_fp8_gemm"):
        cm.clearmoe_fp8_gemm(Rows(), Rows(), Posing(), stream=Stream())
