"""bench.py holds a capture's DRAM traffic valid while the kernel's sources are unchanged: those have to be every file of the
package that the kernel is compiled from, or a change of one goes unseen and a move of code to another voids the figure."""
import importlib.util
import pathlib
import re

import pytest

ROOT = pathlib.Path(__file__).resolve().parents[1]
CSRC = ROOT / "paper_2606_28516_gb300" / "csrc"


@pytest.fixture(scope="module")
def bench():
    spec = importlib.util.spec_from_file_location("bench_under_test", ROOT / "bench.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def included(name, seen):
    if name not in seen and ".." not in name:  # the public header declares the calls only
        seen.add(name)
        for other in re.findall(r'#include "([^"]+)"', (CSRC / name).read_text()):
            included(other, seen)
    return seen


def test_every_included_file_counts(bench):
    for stage, files in bench.KERNEL_SOURCES.items():
        assert included(files[0], set()) == set(files), stage
    assert set(bench.TRAFFIC) == set(bench.KERNEL_SOURCES)
