"""The order in which the 8-bit kernels end, checked on the sources, and that their scale warps' loop does."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"


def source(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


def kernel(name):
    s = source(name)
    return s[s.index("__global__ void"):s.index("cudaError_t launch")]


def without_lambdas(s):
    out, at = "", 0
    for m in re.finditer(r"\[&\]\([^()]*\) \{", s):
        if m.start() < at:
            continue
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(s[i], 0)
            i += 1
        out, at = out + s[at:m.start()], i
    return out + s[at:]


@pytest.mark.parametrize("name,drains,last", [
    ("fp8_gemm.cu", ["mbar_wait_warp(full_bar(s), (par >> s) & 1", "mbar_wait_warp(drain_bar, 0"], "tmem_dealloc(tmem"),
    ("fp8_gemm2.cu", ["mbar_wait_warp(full_bar(s), (k / STAGES) & 1", "mbar_wait_warp(drain_bar, 0", "bulk_wait_all();"], "tcgen05.dealloc"),
])
def test_copies_and_mmas_end_before_tensor_memory_is_freed(name, drains, last):
    """Each role waits for what it started; then all meet; then the memory is freed, in no role's branch."""
    s = kernel(name)
    free = s.index(last)
    meet = s.rindex("__syncthreads();", 0, free)
    for d in drains:
        assert s.count(d) == 1 and s.index(d) < meet, d
    assert "return;" not in without_lambdas(s[:meet])  # no thread leaves early
    if name == "fp8_gemm2.cu":
        assert meet < s.index("cluster_sync();", meet) < free


@pytest.mark.parametrize("name", ["fp8_gemm.cu", "fp8_gemm2.cu"])
def test_a_scale_warp_ends_with_its_tiles_or_its_wait(name):
    h = source("fp8_gemm.cuh")
    loops = [m.start() for m in re.finditer(r"for \([^;]*;;\)|while \((true|1)\)", h)]
    assert len(loops) == 1  # f8_scale_warp's
    body = h[loops[0]:h.index("__device__", loops[0])]
    assert "if (!full[i] || !put(w[i], " in body and "return;" in body
    assert "if (!t.live()) return false;" in h[h.index("void f8_scale_warp"):loops[0]]  # full[i] ends with the tiles
    s = kernel(name)
    put = s[s.index("f8_scale_warp<BN>("):]
    put = put[:put.index("return true;")]
    assert re.search(r"if \(!mbar_wait_warp\(sempty_bar\(slot\), ph \^ 1, abort_flag, a\.status, lim\)\) return false;", put)
