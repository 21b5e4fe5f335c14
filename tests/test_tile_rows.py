"""Offsets of the chunks that a thread loads of a tile of rows (csrc/tile_rows.h, host code here), against the token and head of every row, for all distances
between chunks, numbers of them and group sizes that the attention kernels have, in layouts where no two strides are multiples of one another."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_22137_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "tile_rows.h"
int main() {
  int wrong = 0, looked = 0;
  const long long strides[][2] = {{100003, 7}, {7, 100003}, {0, 128}, {128, 0}, {3000000011ll, 5}, {5, 3000000011ll}};   // token, head
  for (int apart : {8, 16, 32})          // 256 threads, rows of 512, 256 and 128 bytes
    for (int chunks : {1, 2, 4})
      for (int G = 1; G <= 32; G *= 2)
        for (auto& s : strides) {
          const prism::RowSteps steps = prism::row_steps(apart, G, s[0], s[1]);
          bool same = true;
          for (int r = 0; r < apart; ++r)
            for (int u = 0; u < chunks; ++u) {
              const int row = r + u * apart;
              const long long at = row / G * s[0] + row % G * s[1];
              same = same && prism::row_offset(row, G, s[0], s[1]) == at && prism::row_offset(r, G, s[0], s[1]) + steps.to(u) == at;
              ++looked;
            }
          if (!same) { ++wrong; std::printf("apart %d, %d chunks, group of %d, strides %lld %lld\n", apart, chunks, G, s[0], s[1]); }
        }
  std::printf("%d wrong of %d\n", wrong, looked);
  return wrong != 0;
}
"""


def test_chunks_lie_where_their_rows_do(tmp_path):
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(src), "-o", str(exe)])
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
    assert done.stdout.strip() == "0 wrong of %d" % (56 * 7 * 6 * 6)
