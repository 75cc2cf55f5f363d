"""Programmatic dependent launch, checked on the sources (a run cannot show it: it would have to lose a race). A kernel
may read weights before its predecessor has completed, so weights are safe once some call lies between their writer and
the call that reads them. That holds when each call has a kernel that releases its successor only after its own wait:
then everything before that call has completed when the next one starts."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"
RELEASE, WAIT = "pdl_launch_dependents();", "pdl_wait();"


def source(name):
    s = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    return re.sub(r"__(launch_bounds|cluster_dims)__\([^()]*\)", "", s)


def functions(name):
    """(name, body) of the device functions of a file that release a successor."""
    s = source(name)
    for m in re.finditer(r"\b(\w+)\(([^;{}]*)\)\s*\{", s):
        depth, i = 0, m.end() - 1
        while True:
            depth += {"{": 1, "}": -1}.get(s[i], 0)
            if depth == 0:
                break
            i += 1
        body = s[m.end():i]
        if RELEASE in body and m.group(1) not in ("if", "for", "while"):
            yield m.group(1), body


# Kernels inside a call, after one that releases late: few_expert_kernel's is few_fc1_kernel.
INSIDE = {"few_expert_kernel"}


@pytest.mark.parametrize("name,count", [("few.cu", 3), ("fp8.cu", 3), ("fp8_few.cu", 1), ("fp8_gemm.cu", 1), ("fp8_gemm2.cu", 1),
                                        ("simt.cu", 2), ("route.cu", 3)])
def test_released_after_the_wait(name, count):
    found = list(functions(name))
    assert len(found) == count, [n for n, _ in found]
    for fn, body in found:
        if fn not in INSIDE:
            at = [m.start() for m in re.finditer(re.escape(RELEASE), body)]
            assert all(re.search(r"(^|\n)\s*pdl_wait\(\);", body[:i]) for i in at), (name, fn)


def test_the_dense_forward_starts_with_a_late_release():
    """Its kernels release early unless told otherwise; the fp32 CUDA-core ones are simt.cu's."""
    s = source("api.cu")
    s = s[s.index("static int dense_impl"):s.index("int clearmoe_dense_ffn_forward_ex")]
    first = [p for p in s.split("std::memset(&g, 0, sizeof(g));")[1:] if "launch_tc_gemm" in p]
    assert len(first) == 2
    for p in first:
        assert "g.pdl_trigger_late = 1;" in p[:p.index("launch_tc_gemm")]
