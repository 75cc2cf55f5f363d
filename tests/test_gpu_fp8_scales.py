"""Products of blocks whose scales multiply to a power of two outside fp32: exact as long as the result is inside."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu

KERNELS = [(16, 0), (256, 1), (192, 1), (128, 1), (192, 0), (128, 0), (64, 0), (32, 0)]
# scale bytes of A's row and W's block, an e4m3 value of each
CASES = [(247, 247, 0.0, 1.0), (250, 134, 2.0 ** -9, 2.0 ** -9), (192, 192, 2.0 ** -9, 2.0 ** -9), (52, 52, 256.0, 256.0),
         (0, 109, 256.0, 256.0), (57, 57, 1.0, 1.0), (254, 1, 1.0, 1.0), (0, 254, 2.0, 4.0), (0, 0, 256.0, 256.0), (127, 128, 3.0, 5.0)]


def blocks(rows, weight, byte, value, k):
    m = cm.fp8_weight(rows, 256) if weight else cm.fp8_rows(rows, 256)
    m.q.view(torch.uint8).zero_()
    m.scale.zero_()
    m.q.view(torch.float8_e4m3fn)[0, k] = value
    m.scale[:, :2] = byte
    return m


@pytest.fixture(params=KERNELS)
def kernel(request):
    cm.clearmoe_debug_fp8_kernel(*request.param)
    yield
    cm.clearmoe_debug_fp8_kernel()


@pytest.mark.parametrize("sa,sw,a,w", CASES)
@pytest.mark.parametrize("M", [1, 12])
def test_exact(kernel, M, sa, sw, a, w):
    for k in (0, 130):
        A, W, out = blocks(M, False, sa, a, k), blocks(40, True, sw, w, k), torch.full((M, 40), float("nan"), device="cuda")
        cm.clearmoe_fp8_gemm(A, W, out)
        want = torch.tensor(a * w * 2.0 ** (sa + sw - 254), dtype=torch.float64).float().item()  # 0 below fp32's range
        assert out[0, 0].item() == want
        out[0, 0] = 0
        assert not out.any()  # zeros stay zeros (NaN would count)


@pytest.mark.parametrize("sa,sw", [(255, 120), (0, 255), (255, 255)])
def test_nan_scales(kernel, sa, sw):
    A, W, out = blocks(3, False, sa, 0.0, 0), blocks(40, True, sw, 0.0, 0), torch.zeros(3, 40, device="cuda")
    cm.clearmoe_fp8_gemm(A, W, out)
    assert bool(out.isnan().all())


def test_by_the_quantiser():
    """A row of 1e38 against weights of which every other row is zero, the rest 1e4: 0 there."""
    A, W = cm.fp8_rows(5, 300), cm.fp8_weight(64, 300)
    x, w = torch.full((5, 300), 1e38, device="cuda"), torch.full((64, 300), 1e4, device="cuda")
    w[::2] = 0
    cm.clearmoe_fp8_quantize_rows(x, A)
    cm.clearmoe_fp8_quantize_weight(w, W)
    out = torch.full((5, 64), float("nan"), device="cuda")
    cm.clearmoe_fp8_gemm(A, W, out)
    assert not out[:, ::2].any() and bool((out[:, 1::2] == float("inf")).all())


def test_a_fixed_kernel_is_its_threads_alone():
    """The kernel for few rows sums in another order than the tiled ones, which a width past its own choice gets: its bits
    appear in the thread that fixed it, and in no other."""
    import threading
    g = torch.Generator(device="cuda").manual_seed(4)
    A, W = cm.fp8_rows(5, 4096), cm.fp8_weight(12000, 4096)
    cm.clearmoe_fp8_quantize_rows(torch.randn(5, 4096, generator=g, device="cuda"), A)
    cm.clearmoe_fp8_quantize_weight(torch.randn(12000, 4096, generator=g, device="cuda"), W)

    def product():
        out = torch.empty(5, 12000, device="cuda")
        cm.clearmoe_fp8_gemm(A, W, out)
        torch.cuda.synchronize()
        return out

    by_size, fixed, ready, done = product(), [], threading.Event(), threading.Event()

    def other():
        cm.clearmoe_debug_fp8_kernel(16, 0)
        fixed.append(product())
        ready.set()
        done.wait(60)
        cm.clearmoe_debug_fp8_kernel()

    t = threading.Thread(target=other)
    t.start()
    try:
        assert ready.wait(60)
        here = product()
    finally:
        done.set()
        t.join()
    assert not torch.equal(fixed[0], by_size)
    assert torch.equal(here, by_size)
