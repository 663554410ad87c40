"""Where the rows of a paged cache may lie, worked through on the CPU with the header that the calls' checks use: rows of one plane that
overlap, and rows of two planes that do, against a list of every value's place."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "pages_layout.h"
using namespace confkv;

static std::vector<long long> rows_of(const PagesDim (&d)[3]) {
  std::vector<long long> rows;
  for (long long i = 0; i < d[0].size; ++i)
    for (long long j = 0; j < d[1].size; ++j)
      for (long long k = 0; k < d[2].size; ++k) rows.push_back(i * d[0].stride + j * d[1].stride + k * d[2].stride);
  return rows;
}

int main() {
  const int D = 16;
  long layouts = 0, good = 0, met = 0;
  unsigned seed = 1;
  auto draw = [&](int n) { return (int)((seed = seed * 1664525u + 1013904223u) >> 8) % n; };
  for (int c = 0; c < 6000; ++c) {
    PagesDim d[3];
    long long at = D + 8 * draw(3);
    int order[3] = {0, 1, 2};
    std::swap(order[0], order[draw(3)]);
    std::swap(order[1], order[1 + draw(2)]);
    for (int i : order) {
      d[i] = {1 + draw(4), at};
      at = d[i].stride * (d[i].size - 1) + at + 8 * draw(4);
      if (draw(20) == 0) d[i].stride -= 8;                                // some that overlap
      if (d[i].size == 1 && draw(2)) d[i].stride = 8 * draw(100);         // a stride that nothing uses
    }
    const std::vector<long long> rows = rows_of(d);
    bool apart = true;
    long long last = 0;
    for (size_t i = 0; i < rows.size(); ++i) {
      last = std::max(last, rows[i]);
      for (size_t j = 0; j < i; ++j) apart = apart && (rows[i] - rows[j] >= D || rows[j] - rows[i] >= D);
    }
    const long long extent = pages_extent(d, D);
    ++layouts;
    if (extent == 0) continue;                                            // (some of these do not overlap: nested layouts are taken only)
    if (!apart || extent != last + D) { printf("layout %d: extent %lld, last row %lld, apart %d\n", c, extent, last, apart); return 1; }
    ++good;
    for (long long by = -extent - 24; by <= extent + 24; by += 8) {
      bool share = false;
      for (long long x : rows)
        for (long long y : rows) share = share || (x - y - by < D && y + by - x < D);
      if (planes_meet(d, D, by) != share) { printf("layout %d: planes %lld apart share values: %d\n", c, by, share); return 1; }
      met += share;
    }
  }
  // sizes as in earnest: keys and values in turns by pages, tokens and heads; one piece of sixteen bytes too near
  for (int unit = 0; unit < 3; ++unit) {
    long long H = 8, page = 64, n = 1 << 20, head = unit == 0 ? 256 : 128, token = unit == 1 ? 2 * H * head : H * head, stride = unit == 2 ? 2 * page * token : page * token;
    PagesDim d[3] = {{n, stride}, {page, token}, {H, head}};
    if (pages_extent(d, 128) == 0) return 2;
    const long long turn = unit == 0 ? 128 : unit == 1 ? H * head : page * token;
    if (planes_meet(d, 128, turn) || planes_meet(d, 128, -turn)) { printf("turns of unit %d\n", unit); return 3; }
    for (long long by : {0ll, 8ll, turn - 8, turn + 8, -turn + 8, n / 2 * stride + turn + 8, (n - 1) * stride})
      if (!planes_meet(d, 128, by)) { printf("unit %d: %lld apart\n", unit, by); return 4; }
  }
  PagesDim far[3] = {{4, 1ll << 40}, {8, 128}, {1, 0}}, wide[3] = {{4, (1ll << 40) + 8}, {8, 128}, {1, 0}}, odd[3] = {{4, 1028}, {8, 128}, {1, 0}};
  if (pages_extent(far, 128) == 0 || pages_extent(wide, 128) != 0 || pages_extent(odd, 128) != 0) return 5;
  printf("%ld layouts, %ld taken, %ld distances at which planes meet\n", layouts, good, met);
  return good > 1000 && met > 1000 ? 0 : 6;
}
"""


def test_rows_that_overlap(tmp_path):
    source, exe = tmp_path / "layout.cpp", str(tmp_path / "layout")
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_24786_amd", "csrc"), str(source),
                    "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, (run.returncode, run.stdout)
