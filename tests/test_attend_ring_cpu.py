"""Waits of the linear attention's tensor-core kernel without a GPU: its rules on
which arrivals are asked for, compiled for the host, against the waits of its warps."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_08802_gb300", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "attend_ring.h"
using namespace pnn::attend;
int main() {
  std::printf("%d\n", RING);
  for (int per = 2; per <= 3; ++per)       // loads of a chunk: y, z for a segment's sum, x, y, z otherwise
    for (int chunks = 0; chunks <= 9; ++chunks) {
      std::printf("place %d %d :", per, chunks);
      for (int n = 0; n < per * chunks; ++n)
        if (place_again(n, per * chunks)) std::printf(" %d", n);
      std::printf("\nbuffer %d %d :", per, chunks);
      for (int g = 0; g < 4 * chunks; ++g)
        if (buffer_again(g, chunks)) std::printf(" %d", g);
      std::printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("ring")
    (d / "rules.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(d / "rules.cpp"), "-o", str(d / "rules")], check=True)
    ring, *lines = subprocess.run([str(d / "rules")], check=True, capture_output=True, text=True).stdout.splitlines()
    table = {}
    for line in lines:
        key, values = line.split(":")
        kind, per, chunks = key.split()
        table[kind, int(per), int(chunks)] = [int(v) for v in values.split()]
    return int(ring), table


@pytest.mark.parametrize("per", [2, 3])
@pytest.mark.parametrize("chunks", range(10))
def test_every_arrival_is_waited_for(rules, per, chunks):
    """An arrival that no warp of the CTA waits for may come after its end, into memory that is another CTA's by then; one that
    a warp waits for and nobody asks for ends in a wait that gives up."""
    ring, table = rules
    loads = per * chunks
    assert table["place", per, chunks] == [n - ring for n in range(ring, loads)]  # the loading warp, before load n
    assert table["buffer", per, chunks] == [g - 2 for g in range(2, 4 * chunks)]  # the warps that form K', before quarter g
