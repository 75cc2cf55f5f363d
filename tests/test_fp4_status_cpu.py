"""The compiled binding of the 4-bit product looks at its status word as at every other tensor: on the GPU of the stream, dense,
int32. Without a GPU: tensors that describe themselves by exchange capsules made here, and null pointers, which the library
refuses (ClearMoEError) when the binding lets a call through."""
import ctypes

import pytest
import torch

from paper_2606_28516_gb300 import build, clearmoe as cm


class DL(ctypes.Structure):  # DLPack's tensor
    _fields_ = [("data", ctypes.c_void_p), ("device_type", ctypes.c_int32), ("device_id", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("code", ctypes.c_uint8), ("bits", ctypes.c_uint8), ("lanes", ctypes.c_uint16), ("shape", ctypes.c_void_p),
                ("strides", ctypes.c_void_p), ("byte_offset", ctypes.c_uint64)]


new_capsule = ctypes.pythonapi.PyCapsule_New
new_capsule.restype, new_capsule.argtypes = ctypes.py_object, [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p]
TYPES = {torch.float32: (2, 32), torch.bfloat16: (4, 16), torch.int32: (0, 32), torch.int64: (0, 64)}


class Posing:
    """A CUDA tensor as far as the binding looks, on GPU `device`."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0, strides=None):
        self.shape, self.dtype, self.device = shape, dtype, device
        dense, step = [], 1
        for n in reversed(shape):
            dense.insert(0, step)
            step *= n
        self.strides = tuple(strides or dense)
        self.dense = all(n == 1 or a == b for n, a, b in zip(shape, self.strides, dense))
        self.s, self.t = (ctypes.c_int64 * len(shape))(*shape), (ctypes.c_int64 * len(shape))(*self.strides)
        self.dl = DL(None, 2, device, len(shape), *TYPES[dtype], 1, ctypes.addressof(self.s), ctypes.addressof(self.t), 0)

    def capsule(self):
        return new_capsule(ctypes.addressof(self.dl), b"dltensor", None)

    def get_device(self):
        return self.device

    def stride(self):
        return self.strides

    def numel(self):
        return torch.Size(self.shape).numel()

    def is_contiguous(self):
        return self.dense

    def data_ptr(self):
        return 0


class Bytes(Posing):
    def element_size(self):
        return 1


class Stream:
    cuda_stream, device_index = 0, 0


@pytest.fixture(scope="module", autouse=True)
def binding():
    build.build()
    m = cm._bind_calls()
    m.bind_dlpack(lambda t: t.capsule())
    yield m
    m.bind_dlpack(torch._C._to_dlpack)


def matrix4(rows, cols):
    return cm.Fp4Matrix(Bytes(rows, cm.fp4_pitch(cols)), Bytes(-(-rows // 128), -(-cols // 128), 512), rows, cols)


def product(blocks=False, **kw):
    out = matrix4(4, 9) if blocks else Posing(4, 9)
    cm.clearmoe_fp4_gemm(matrix4(4, 64), matrix4(9, 64), out, stream=Stream(), **kw)


@pytest.mark.parametrize("blocks", [False, True])
def test_status_on_another_gpu_is_refused(blocks):
    with pytest.raises(ValueError, match="GPU 1"):
        product(blocks, status=Posing(1, dtype=torch.int32, device=1))


@pytest.mark.parametrize("status", [Posing(1), Posing(1, dtype=torch.int64), Posing(4, dtype=torch.int32, strides=(2,)),
                                    Posing(2, 2, dtype=torch.int32, strides=(1, 2)), Posing(0, dtype=torch.int32)])
def test_other_status_words_are_refused(status):
    with pytest.raises(ValueError):
        product(status=status)


@pytest.mark.parametrize("status", [None, Posing(1, dtype=torch.int32), Posing(dtype=torch.int32), Posing(3, 2, dtype=torch.int32),
                                    Posing(1, 4, dtype=torch.int32, strides=(9, 1))])
def test_status_words_that_reach_the_library(binding, status):
    a, w = matrix4(4, 64), matrix4(9, 64)
    code = binding.fp4_gemm_t(a.addr, w.addr, cm.ACT_NONE, None, status, Posing(4, 9), Stream())
    assert code == cm.EINVAL  # None: the call would go by way of the integers, slower
