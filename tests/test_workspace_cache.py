"""The workspaces that the library keeps (csrc/workspace_cache.h, host code without GPU calls), with an allocator that refuses blocks above a limit."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_22137_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "workspace_cache.h"
int main() {
  prism::WorkspaceCache cache;
  static char memory[64];
  int asked = 0;
  size_t limit = 100;
  auto alloc = [&](size_t n) -> void* { ++asked; return n <= limit ? memory + asked : nullptr; };
  int one, two;
  // a call that would like 150 and can do with 80
  auto call = [&](const void* owner, size_t wish, size_t least) -> size_t {
    if (cache.get(0, owner, wish, true, alloc)) return wish;
    return cache.get(0, owner, least, false, alloc) ? least : 0;
  };
  auto show = [&](size_t got) { std::printf("%zu %d\n", got, asked); };
  show(call(&one, 150, 80));      // 80: asked for 150 and 80
  show(call(&one, 150, 80));      // again: nothing is asked for
  show(call(&one, 200, 80));      // more than what was refused: nor here
  show(call(&one, 95, 80));       // less: there is such a block
  show(call(&two, 150, 120));     // neither: 0, both asked for
  show(call(&two, 150, 120));     // what the call needs at least is always asked for
  limit = 300;
  show(call(&two, 150, 120));     // 120: memory has come free, the wish stays refused
  show(call(&one, 90, 90));       // there
  cache.blocks.clear();           // released
  show(call(&one, 150, 80));      // 150
  std::printf("%zu\n", cache.blocks.size());
}
"""


def test_a_refused_size_is_not_asked_for_again(tmp_path):
    src, exe = tmp_path / "cache.cpp", tmp_path / "cache"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(src), "-o", str(exe)])
    got = [tuple(int(v) for v in line.split()) for line in subprocess.check_output([str(exe)], text=True).splitlines()]
    assert got == [(80, 2), (80, 2), (80, 2), (95, 3), (0, 5), (0, 6), (120, 7), (90, 7), (150, 8), (1,)]


GROWING = r"""
#include <cstdio>
#include "workspace_cache.h"
int main() {
  prism::WorkspaceCache cache;
  static char memory[64];
  size_t asked = 0, held = 0, limit = ~(size_t)0;
  auto alloc = [&](size_t n) -> void* {
    if (n > limit) return nullptr;
    held += n;
    return memory + asked++;
  };
  int one, two;
  // sequences that become longer from call to call
  for (size_t n = 1000; n <= 1000000; n += 1000)
    if (!cache.get(0, &one, n, false, alloc, true)) return 1;
  std::printf("%zu %zu\n", asked, held / 1000);
  // the first block is of the size asked for, and so is one where there is no room to spare
  asked = held = 0;
  limit = 1500;
  for (size_t n : {1000, 1100, 1050, 1600}) std::printf("%d ", cache.get(0, &two, n, false, alloc, true) != nullptr);
  std::printf("%zu %zu\n", asked, held);
  return 0;
}
"""


def test_blocks_that_are_outgrown_again_and_again(tmp_path):
    """All blocks together stay within a few times the last, and are few."""
    src, exe = tmp_path / "growing.cpp", tmp_path / "growing"
    src.write_text(GROWING.replace("#include <cstdio>", "#include <cstdio>\n#include <initializer_list>"))
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(src), "-o", str(exe)])
    first, second = subprocess.check_output([str(exe)], text=True).splitlines()
    blocks, held = (int(x) for x in first.split())
    assert blocks == 11 and held == 2 ** 11 - 1          # 1, 2, 4 ... 1024 thousand
    assert second.split() == ["1", "1", "1", "0", "2", "2100"]
