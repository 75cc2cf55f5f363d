"""Products of 8-bit blocks right behind the kernels that write their weights, rows and bias, new ones each time: the same bits
as after a synchronisation. A norm writes the rows and another product the bias, kernels that let their successor start early.
The kernel for few rows, tiles of one SM and of pairs; outputs in fp32 and in 8-bit blocks."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("kernel,M,N,K", [((16, 0), 3, 2048, 8192), ((16, 0), 12, 512, 4096), ((64, 0), 300, 512, 1024), ((128, 0), 300, 512, 1024),
                                          ((128, 1), 700, 1024, 1024), ((256, 1), 3000, 1024, 512)])
def test_operands_and_bias_just_written(kernel, M, N, K, blocks):
    g = torch.Generator("cuda").manual_seed(M + N + K)
    xs = [torch.randn(M, K, device="cuda", generator=g) for _ in range(2)]
    ws = [torch.randn(N, K, device="cuda", generator=g) for _ in range(2)]
    A, W, b = cm.fp8_rows(M, K), cm.fp8_weight(N, K), torch.empty(N, device="cuda")
    Wb, cs = cm.fp8_weight(N, 256), [cm.fp8_rows(1, 256) for _ in range(2)]
    cm.clearmoe_fp8_quantize_weight(torch.randn(N, 256, device="cuda", generator=g), Wb)
    for c in cs:
        cm.clearmoe_fp8_quantize_rows(torch.randn(1, 256, device="cuda", generator=g), c)

    def new():
        return cm.fp8_rows(M, N) if blocks else torch.empty(M, N, device="cuda")

    def bits(o):
        return (o.q.view(torch.uint8), o.scale[:, :N // 128]) if blocks else (o,)

    def product(i, out, sync):
        """Every operand in turn is the one that the kernel right before has written."""
        steps = [lambda: cm.clearmoe_rms_norm(xs[i & 1], A), lambda: cm.clearmoe_fp8_quantize_weight(ws[i & 1], W),
                 lambda: cm.clearmoe_fp8_gemm(cs[i & 1], Wb, b.view(1, N))]
        for k in range(3):
            steps[(i // 2 + k) % 3]()
            if sync:
                torch.cuda.synchronize()
        cm.clearmoe_fp8_gemm(A, W, out, bias=b)
        if sync:
            torch.cuda.synchronize()

    cm.clearmoe_debug_fp8_kernel(*kernel)
    try:
        want = [new(), new()]
        for i in (0, 1):
            product(i, want[i], True)
        outs = [new() for _ in range(36)]
        for i, out in enumerate(outs):
            product(i, out, False)
    finally:
        cm.clearmoe_debug_fp8_kernel()
    for i, out in enumerate(outs):
        for mine, theirs in zip(bits(out), bits(want[i & 1])):
            assert torch.equal(mine, theirs), i
