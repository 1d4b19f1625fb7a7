"""Addresses of the norms' asynchronous copies without a GPU: the kernels' rule,
compiled for the host, over rows of every width that begin inside a vector."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2103_08802_gb300", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "norm_place.h"
// pieces of `ve` values of `size` bytes, of the places of a team that holds the row with what lies before it
long long check(int ve, int size, int width, long long stride, long long rows, long long *pieces) {
  const uintptr_t tensor = 4096;
  long long bad = 0;
  int team = 8;
  while (team * 8 < width + 7) team *= 2;
  for (long long row = 0; row < rows; ++row) {
    const int off = (int)(row * stride % ve);
    const uintptr_t p = tensor + row * stride * size;
    for (int place = 0; place < team * 8; place += ve) {
      const uintptr_t at = pnn::norm::piece_address(p, p + (place - off) * size, place - off >= width, ve * size);
      ++*pieces;
      if (at < tensor || at % (ve * size) || at >= p + width * size) ++bad;
    }
  }
  return bad;
}
int main() {
  long long pieces = 0, bad = 0;
  const int widths[] = {1001, 1002, 1801, 2047, 4093, 4101, 8180, 8187}, forms[][2] = {{8, 2}, {4, 2}, {4, 4}};
  for (auto& f : forms) {
    for (int width = 1; width <= 300; ++width)
      for (int gap = 0; gap <= 9; ++gap) bad += check(f[0], f[1], width, width + gap, 17, &pieces);
    for (int width : widths) bad += check(f[0], f[1], width, width, 17, &pieces);
  }
  std::printf("%lld %lld\n", bad, pieces);
}
"""


def test_copies_begin_on_borders(tmp_path):
    """A copy of 8 or 16 bytes wants an address that is a multiple of them, also where it copies nothing and fills in zeros."""
    (tmp_path / "place.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(tmp_path / "place.cpp"), "-o", str(tmp_path / "place")], check=True)
    bad, pieces = map(int, subprocess.run([str(tmp_path / "place")], check=True, capture_output=True, text=True).stdout.split())
    assert pieces > 100000 and bad == 0
