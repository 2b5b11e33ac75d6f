"""How a block of the prompt attention ends, and what its row tile does with it: the decisions
are plain functions, compiled here for the host (no wait is made to run out on a GPU)."""
import itertools
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21835_gb300", "csrc")
GOOD, NOT_FINITE, STOPPED = 0, 1, 2


@pytest.fixture(scope="module")
def table(tmp_path_factory):
    cxx = shutil.which("g++") or pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("parts")
    (d / "t.cpp").write_text("""
#include <cstdio>
#include "window_parts.h"
using namespace loip;
int main() {
    for (int s = 0; s < 2; ++s)
        for (int b = 0; b < 2; ++b) std::printf("end %d %d %u\\n", s, b, part_end(s, b));
    for (unsigned x = 0; x < 3; ++x)
        for (unsigned y = 0; y < 3; ++y) std::printf("worse %u %u %u\\n", x, y, worse(x, y));
}
""")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(d / "t.cpp"), "-o", str(d / "t")], check=True)
    out = subprocess.run([str(d / "t")], check=True, capture_output=True, text=True).stdout.split("\n")
    return {tuple(l.split()[:3]): int(l.split()[3]) for l in out if l}


def test_a_block_that_stopped_is_neither_good_nor_walked(table):
    assert table["end", "0", "0"] == GOOD and table["end", "0", "1"] == NOT_FINITE
    assert table["end", "1", "0"] == STOPPED and table["end", "1", "1"] == STOPPED


def test_a_row_tile_ends_as_the_worst_of_its_parts(table):
    for n in (1, 2, 3):
        for parts in itertools.product((GOOD, NOT_FINITE, STOPPED), repeat=n):
            end = GOOD
            for x in parts:
                end = table["worse", str(end), str(x)]
            assert end == max(parts)


def test_no_row_is_stored_without_asking():
    """Every store of finished rows is behind the question, and the joining kernel returns for a stopped tile."""
    src = open(os.path.join(CSRC, "window_prefill.cu")).read()
    calls = [l.strip() for l in src.splitlines() if "leave(" in l and "auto leave" not in l]
    assert calls and all(l.startswith("if (!stopped()) leave(") for l in calls), calls
    join = src[src.index("window_join_kernel("):]
    assert join.index("if (end == kPartStopped) return;") < join.index("walk_row")
    assert "part_end(stopped()" in src and "p.ended[unit * p.splits + split] = end;" in src
