"""The ranges that conf_kv_constrain's workgroups own, worked through on the CPU with the header that the kernel and its launch use:
every logit in one range, no slot of a token or bias outside a range's room, no range that no row needs."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "constrain_ranges.h"
using namespace confkv;

static void check(int V, int B, unsigned at, int range, bool whole) {
  const int n = con_grid_ranges(at, B, V, range, whole);
  auto fail = [&](const char *what, int b, int j) {
    printf("%s: V %d rows %d result at %u range %d whole %d row %d workgroup %d of %d\n", what, V, B, at, range, whole, b, j, n);
    exit(1);
  };
  bool last_used = false;
  for (int b = 0; b < B; ++b) {
    const int off = whole ? 0 : con_off((uintptr_t)at + (uintptr_t)b * V * 4);
    int next = 0;
    for (int j = 0; j < n; ++j) {
      const int lo = con_first(j, off, range);
      if (con_empty(lo, V)) continue;
      const int size = con_size(lo, V, range);
      // the kernel compares (unsigned)(id - lo) with (unsigned)size and addresses that slot of `range`
      if (size < 1 || size > range) fail("slots outside the room", b, j);
      const int from = lo < 0 ? 0 : lo, to = lo + size;
      if (from != next || to <= from || to > V) fail("logits left out or shared", b, j);
      next = to;
      last_used = last_used || j == n - 1;
    }
    if (next != V) fail("logits left out at the end", b, n);
  }
  if (!last_used) fail("a range that no row needs", 0, n - 1);
}

int main() {
  long cases = 0;
  for (int quads : {1, 2, 4, 5}) {
    const int range = 1024 * 4 * quads;
    auto all = [&](int V) {
      for (int B : {1, 2, 3, 4, 7})
        for (unsigned at = 0; at < 16; at += 4) check(V, B, at, range, false), ++cases;
      if (V % 4 == 0) check(V, 3, 0, range, true), ++cases;
    };
    for (int V = 1; V <= 40; ++V) all(V);
    for (int k = 1; k <= 40; ++k)
      for (int d = -5; d <= 5; ++d) all(k * range + d);
    for (int V : {32000, 50257, 128256, 131072, 152064, (1 << 27) - 1, 1 << 27}) all(V);
  }
  printf("%ld cases\n", cases);
}
"""


def test_every_logit_has_one_slot(tmp_path):
    source, exe = tmp_path / "ranges.cpp", str(tmp_path / "ranges")
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_24786_amd", "csrc"), str(source),
                    "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stdout
