"""ffn_weights and the forwards that take them refuse tensors whose shape or dtype is not the layer's: the library gets
addresses, and reads or writes past the end of a tensor of another size. Without a GPU: stand-ins for CUDA tensors."""
import ctypes

import pytest

from paper_2606_28516_gb300 import build, clearmoe as cm

BF16, F32, F16 = "torch.bfloat16", "torch.float32", "torch.float16"
d, H, E = 64, 256, 3


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


class Dense:
    is_cuda = True

    def __init__(self, *shape, dtype=BF16):
        self.shape, self.dtype = shape, dtype

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def stride(self):
        return self.shape[1], 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Stream:
    cuda_stream = 0


def block(rows, cols):
    m = object.__new__(cm.Fp8Matrix)
    m.q = m.scale = None
    m.rows, m.cols, m.weight = rows, cols, True
    m.c = cm.clearmoe_fp8(1 << 20, 1 << 20, rows, cols)
    m.ref, m.addr = ctypes.pointer(m.c), ctypes.addressof(m.c)
    return m


def weights(fp8=False, dtype=BF16, **kw):
    mat = block if fp8 else (lambda r, c: Dense(r, c, dtype=dtype))
    a = dict(W1=mat(H, d), b1=Dense(H, dtype=dtype), W_comb=[mat(d, H) for _ in range(E)], Wg=Dense(E, d, dtype=dtype),
             bg=Dense(E, dtype=dtype), b2=Dense(d, dtype=dtype), W2=mat(d, H), cls_stride=5)
    a.update(kw)
    return cm.ffn_weights(**a)


@pytest.mark.parametrize("fp8,dtype,code", [(False, BF16, cm.BF16), (False, F32, cm.F32), (True, BF16, cm.FP8)])
def test_of_one_dtype(fp8, dtype, code):
    w = weights(fp8, dtype)
    assert w.c.dtype == code and w.d == d and w.dtype == (cm.F32 if dtype == F32 else cm.BF16)


@pytest.mark.parametrize("fp8,dtype", [(False, BF16), (False, F32), (True, BF16)])
def test_of_several_dtypes_or_shapes(fp8, dtype):
    mat = block if fp8 else (lambda r, c: Dense(r, c, dtype=dtype))
    for other in {BF16, F32, F16} - {dtype}:
        for kw in (dict(b1=Dense(H, dtype=other)), dict(bg=Dense(E, dtype=other)), dict(b2=Dense(d, dtype=other)),
                   dict(Wg=Dense(E, d, dtype=other))):
            with pytest.raises(ValueError):
                weights(fp8, dtype, **kw)
        if not fp8:
            for kw in (dict(W1=Dense(H, d, dtype=other)), dict(W2=Dense(d, H, dtype=other)),
                       dict(W_comb=[Dense(d, H, dtype=dtype)] * 2 + [Dense(d, H, dtype=other)])):
                with pytest.raises(ValueError):
                    weights(fp8, dtype, **kw)
    for kw in (dict(W1=mat(H, d + 64)), dict(W1=mat(H + 64, d)), dict(W_comb=[mat(d, H)] * 2 + [mat(d, H - 64)]),
               dict(W_comb=[mat(d, H)] * 2), dict(W2=mat(d + 1, H)), dict(b1=Dense(H - 1, dtype=dtype)), dict(bg=Dense(E + 1, dtype=dtype)),
               dict(b2=Dense(H, dtype=dtype))):
        with pytest.raises(ValueError):
            weights(fp8, dtype, **kw)


def test_8_bit_weights_are_of_bf16_layers():
    with pytest.raises(ValueError, match="bf16 layers"):
        weights(True, F32)


@pytest.mark.parametrize("call", [cm.clearmoe_ffn_forward_few, cm.clearmoe_ffn_forward_fp8])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_of_another_shape_or_dtype(call, dtype):
    w = weights(dtype=dtype)
    x, out, other = Dense(4, d, dtype=dtype), Dense(4, d, dtype=dtype), F32 if dtype == BF16 else BF16
    for a, b in ((Dense(4, d, dtype=other), out), (x, Dense(4, d, dtype=other)), (x, Dense(3, d, dtype=dtype)), (x, Dense(4, d - 1, dtype=dtype)),
                 (Dense(4, 2 * d, dtype=dtype), out), (Dense(4 * d, dtype=dtype), out), (x, Dense(2, 2, d, dtype=dtype)),
                 (Dense(4, d, dtype=F16), out)):
        with pytest.raises(ValueError, match="must be"):
            call(None, a, w, b, stream=Stream())
    with pytest.raises(cm.ClearMoEError):  # no handle: refused by the library
        call(None, x, w, out, stream=Stream())
