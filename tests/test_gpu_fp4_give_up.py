"""Products of 4-bit blocks whose waits do run out: the kernel for few rows, and tiles in halves. Each gives up some of the time at
least under limits of a few microseconds at these sizes, says so, and lets what is in flight land by the right count of bytes: with
a wrong one the wait for it would take its own limit, 10 ms, where the whole call takes a tenth of a millisecond. The next call with
the usual limit gives the same bits."""
import numpy as np
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu

DRAIN_MS = 10.0


def mat(rows, cols):
    m = cm.fp4_matrix(rows, cols)
    cm.clearmoe_fp4_quantize(torch.randn(rows, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(rows)), m)
    return m


def runs_out(call, bits, limits, times, before=lambda: None):
    """The number of calls that gave up; each is timed, and followed by one that does not."""
    status, n = torch.zeros(1, dtype=torch.int32, device="cuda"), 0
    call(status)
    want = bits.clone()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    try:
        for limit in limits:
            for _ in range(times):
                before()
                cm.clearmoe_debug_fp4_wait(limit)
                a.record()
                call(status)
                b.record()
                cm.clearmoe_debug_fp4_wait()
                torch.cuda.synchronize()
                assert status.item() in (0, cm.ETIMEOUT)
                n += status.item() != 0
                assert a.elapsed_time(b) < 0.8 * DRAIN_MS
                status.zero_()
                bits.zero_()
                call(status)
                assert status.item() == 0 and torch.equal(bits, want)
    finally:
        cm.clearmoe_debug_fp4_wait()
    return n


@pytest.mark.parametrize("blocks", [False, True])
def test_few_rows(blocks):
    M, N, K = 64, 4096, 65536
    A, W = mat(M, K), mat(N, K)
    out = cm.fp4_matrix(M, N) if blocks else torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    cold = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")  # past L2: loads take the longer
    cm.clearmoe_debug_fp4_kernel(16, 0)
    try:
        assert runs_out(lambda s: cm.clearmoe_fp4_gemm(A, W, out, status=s), out.q if blocks else out, (1, 1000, 3000), 14,
                        lambda: cold.fill_(1))
    finally:
        cm.clearmoe_debug_fp4_kernel()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", [([200, 0, 0, 0], 512, 65536), ([3000, 2120], 1280, 8192)])
def test_groups_in_halves_of_tiles(counts, N, K, dtype):
    """All tiles in halves; and the last of each pair's."""
    M, E = sum(counts), len(counts)
    A, W = mat(M, K), mat(N, K)
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    out = torch.empty(M, N, device="cuda", dtype=dtype)
    cm.clearmoe_debug_fp4_kernel(256, 1)
    try:
        assert runs_out(lambda s: cm.clearmoe_fp4_grouped_gemm(A, [W] * E, off, out, status=s), out, (1, 200, 1000, 4000), 4)
    finally:
        cm.clearmoe_debug_fp4_kernel()


@pytest.mark.parametrize("kind", ["bf16", "fp32", "blocks"])
def test_halves_of_tiles(kind):
    M, N, K = 2560, 2048, 8192
    A, W = mat(M, K), mat(N, K)
    out = cm.fp4_matrix(M, N) if kind == "blocks" else torch.empty(M, N, device="cuda", dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    cm.clearmoe_debug_fp4_kernel(256, 1)
    try:
        assert runs_out(lambda s: cm.clearmoe_fp4_gemm(A, W, out, status=s), out.q if kind == "blocks" else out, (1, 200, 1000, 4000), 4)
    finally:
        cm.clearmoe_debug_fp4_kernel()
