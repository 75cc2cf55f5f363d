"""What the products of 8-bit blocks read may have been written by the kernel right before, beside which theirs have started:
ld.global.nc must not read it (PTX: read-only for as long as the kernel lives), and no run shows reliably that it does."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"


def source(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


@pytest.mark.parametrize("name", ["fp8.cu", "fp8.cuh", "fp8_gemm.cuh", "fp8_gemm.cu", "fp8_gemm2.cu", "fp8_few.cu", "pair.cuh"])
def test_no_loads_for_data_that_never_changes(name):
    s = source(name)
    assert "__ldg(" not in s and ".nc" not in s and "__restrict__" not in s


def test_the_product_of_few_rows_shares_its_tiles_but_not_their_loads():
    """few.cuh reads a layer's weights, which are older, by __ldg in one place only, and there not a product's."""
    s = source("few.cuh")
    assert s.count("__ldg(") == 1 and ".nc" not in s and "__restrict__" not in s
    assert re.search(r"V == FEWV_W8A8 \? __ldcg\([^:]*: __ldg\(", s)
    used = set(re.findall(r"Few(?:T|Tile)<(FEWV_\w+)", source("fp8_few.cu")))
    assert used == {"FEWV_W8A8"}
