"""Rules of the 8-bit kernels that a hardware run cannot show to be broken, checked on the sources: every access to
tensor memory follows the last barrier wait before it with a tcgen05 fence in between, warps take a wait's outcome
together, no wait in them is without a limit, and what a routing that gave up may leave behind (boundaries, rows,
slots) is held to the buffers before it is used as an index."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"


def _source(name, start="__global__ void"):
    s = re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), (CSRC / name).read_text())
    return s[s.index(start):]


@pytest.mark.parametrize("name", ["fp8_gemm.cu", "fp8_gemm2.cu"])
def test_tensor_memory_accesses_follow_a_fence(name):
    s = _source(name)
    waits = [m.start() for m in re.finditer(r"\bmbar_wait_warp\((?!pair_bar)", s)]  # pair_bar: magnitudes in shared memory
    uses = list(re.finditer(r"\b(CM_TMEM_LD_X32|umma2?_mxf8|tmem_cp_scales<\d>)\(", s))
    assert len(uses) >= 3
    for m in uses:
        last = max(w for w in waits if w < m.start())
        assert "tc_fence_after();" in s[last:m.start()], (name, s[:m.start()].count("\n"), m.group())


@pytest.mark.parametrize("name", ["fp8_gemm.cu", "fp8_gemm2.cu", "fp8.cu", "fp8_few.cu", "few.cu"])
def test_waits_have_limits(name):
    s = _source(name, "namespace cm")
    assert not re.search(r"\bmbar_wait\(|\bmbar_try_wait\(|while \(true\)|while \(1\)|for \(;;\)", s)
    for m in re.finditer(r"mbar_wait_warp\(([^;]*?)\)\s*[){;]", s):
        assert "lim" in m.group(1) or "10000000ull" in m.group(1), m.group()


@pytest.mark.parametrize("name", ["fp8_gemm.cu", "fp8_gemm2.cu"])
def test_copies_land_before_a_cta_retires(name):
    s = _source(name)
    end = s[s.index("tcgen05.dealloc") if "tcgen05.dealloc" in s else s.index("tmem_dealloc"):]
    assert end
    assert ("drain_step" in s) if name == "fp8_gemm2.cu" else "issued & (1u << s)" in s
    if name == "fp8_gemm2.cu":  # stores by bulk copy read the CTA's shared memory
        assert "bulk_wait_all();" in s[:s.index("tcgen05.dealloc")]


def test_indices_of_a_routing_that_gave_up_are_held_to_the_buffers():
    h = _source("fp8_gemm.cuh", "namespace cm")
    assert "off[e] = min(max(v, acc), (int)a.M);" in h
    assert "(uint32_t)r < (uint32_t)a.M ? r : -1" in h
    q = _source("fp8.cu", "namespace cm")
    assert "if ((uint64_t)slot >= (uint64_t)r.T) slot = -1;" in q
    for name in ("fp8_gemm.cu", "fp8_gemm2.cu"):
        assert "a.rows" not in _source(name)[:_source(name).index("cudaError_t launch")]
