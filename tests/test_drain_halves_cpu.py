"""How a 2-SM product whose walk ends in half a tile lets its copies land when it gives up (csrc/drain.h, compiled here with the
host compiler): producers that stopped at any two stages before, at and after the half's first. Each stage's barrier, as the
hardware counts it, completes with what the drain supplies, and not before the last byte in flight has landed."""
import ctypes
import pathlib
import shutil
import subprocess

import pytest

from test_drain_cpu import Barrier

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_28516_gb300" / "csrc"
SRC = """
#include "drain.h"
extern "C" int step(unsigned k, unsigned n0, unsigned n1) {
    const cm::DrainStep d = cm::drain_step(k, n0, n1);
    return (d.arrive ? 1 : 0) | (d.complete ? 2 : 0);
}
extern "C" unsigned bytes(unsigned k, int halved, unsigned k_half, unsigned whole, unsigned half) {
    return cm::drain_bytes(k, halved != 0, k_half, whole, half);
}
"""
WHOLE, HALF = 35840, 27648  # of a tile of 256 columns, of one of 128


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    t = tmp_path_factory.mktemp("drain_halves")
    (t / "drain.cpp").write_text(SRC)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-I", str(CSRC), "-o", str(t / "drain.so"), str(t / "drain.cpp")],
                   check=True)
    return ctypes.CDLL(str(t / "drain.so"))


def loaded(k, halved, whole_tiles, nkb):
    """What a producer loads in its k-th stage: by tiles, as it walks."""
    return HALF if halved and k // nkb == whole_tiles else WHOLE


@pytest.mark.parametrize("halved", [False, True])
@pytest.mark.parametrize("nkb", [1, 3, 4])
@pytest.mark.parametrize("whole_tiles", [0, 1, 2])
def test_stages_on_both_sides_of_the_half(lib, halved, nkb, whole_tiles):
    total = (whole_tiles + 1) * nkb  # the last tile: half or not
    for n0 in range(total + 1):
        for n1 in range(total + 1):
            for k in range(max(n0, n1)):
                even, odd, size = k < n0, k < n1, loaded(k, halved, whole_tiles, nkb)
                bits, supplied = lib.step(k, n0, n1), lib.bytes(k, int(halved), whole_tiles * nkb, WHOLE, HALF)
                for late in range(even + odd + 1):  # boxes that land after the drain's part
                    b = Barrier()
                    if even:
                        b.arrive_expect(2 * size)
                    for _ in range(even + odd - late):
                        b.land(size)
                    if bits & 1:
                        b.arrive_expect(supplied)
                    if bits & 2:
                        b.land(supplied)
                    for left in range(late, 0, -1):
                        assert not b.done, (k, n0, n1, left)
                        b.land(size)
                    assert b.done, (k, n0, n1, late)
