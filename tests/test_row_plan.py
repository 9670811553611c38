"""How rows are dealt out to lanes (csrc/row_plan.h), enumerated by a plain C++ program (CPU only)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_02317_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include <vector>
#include "row_plan.h"
using namespace moe;
static int fail(const char* what, long a, long b) { printf("%s %ld %ld\n", what, a, b); return 1; }
int main() {
  // division: around every multiple that a rounding could miss, and the ends
  unsigned state = 1;
  auto check = [&](uint32_t n, uint32_t d) { return divide(n, divisor(d)) == n / d; };
  for (uint32_t d = 1; d < 70000; ++d) {
    const uint32_t top = 0x7FFFFFFFu;
    for (uint32_t n : {0u, 1u, d - 1, d, d + 1, 2 * d - 1, 2 * d, top, top - 1, top / d * d, top / d * d - 1})
      if (n <= top && !check(n, d)) return fail("divide", n, d);
    for (int i = 0; i < 20; ++i) {
      state = state * 1664525u + 1013904223u;
      const uint32_t q = state >> 1, at = q / d * d;
      if (!check(q, d) || !check(at, d) || (at && !check(at - 1, d))) return fail("divide", q, d);
    }
  }
  for (uint32_t d : {0x3FFFFFFFu, 0x40000000u, 0x40000001u, 0x7FFFFFFEu, 0x7FFFFFFFu})
    for (uint32_t n : {0u, d - 1, d, 0x7FFFFFFFu})
      if (!check(n, d)) return fail("divide", n, d);
  // rows of the norm: every piece has one place, shapes are those that kernels exist for, the sums of a workgroup fit its memory
  for (int bytes : {2, 4})
    for (int most : {4, 2})
      for (int D = 8; D <= 16384; D += 8) {
        const int n = 16 / bytes, all = D / n;
        const RowSplit s = split_row(all, most);
        if (s.lanes > 64 || (s.lanes & (s.lanes - 1)) || (s.waves > 1 && s.lanes != 64)) return fail("lanes", D, bytes);
        if (s.pieces != 1 && s.pieces != 2 && s.pieces != 4) return fail("pieces", D, bytes);
        if (s.pieces > most && !(bytes == 4 && most == 2 && s.waves == 16)) return fail("more pieces than meant", D, bytes);
        std::vector<int> seen(all, 0);
        for (int p = 0; p < s.pieces; ++p)
          for (int l = 0; l < s.lanes * s.waves; ++l) {
            const int i = p * s.lanes * s.waves + l;
            if (i < all) ++seen[i];
          }
        for (int i = 0; i < all; ++i) if (seen[i] != 1) return fail("piece", D, i);
        const int threads = threads_of(s, most == 4 ? 256 : 512), units = threads / 64 / s.waves;
        if (threads > (most == 4 && bytes == 2 ? 512 : 1024) || threads % 64 || groups_of(s, threads) < 1) return fail("threads", D, threads);
        if (most == 2 && units > 1 && (units % 2 || units / 2 * D * 4 > 32768)) return fail("memory", D, units);
        for (int rows : {1, 2, 3, 100, 4097, 1 << 20, 0x7FFFFFFF}) {
          const int step = groups_of(s, threads) * rows_at_once(s.pieces, most), b = blocks_of(rows, s, threads, most, 256);
          if (b < 1 || b > 256 || b > rows || (b < 256 && (long)b * step < rows)) return fail("blocks", D, rows);
        }
      }
  // rows of the losses
  for (int E = 1; E <= 1024; ++E) {
    const ColumnSplit s = split_columns(E, 2);
    if (s.row % 4 || s.row < E || s.row >= E + 4 || s.lanes > 64 || (s.lanes & (s.lanes - 1))) return fail("row", E, s.row);
    if (s.lanes * s.pieces * 4 < s.row || (s.pieces != 1 && s.pieces != 2 && s.pieces != 4)) return fail("columns", E, s.pieces);
  }
  puts("ok");
  return 0;
}
"""


def test_every_row_is_dealt_out_once(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "p.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "p")
    subprocess.run([cxx, "-O2", "-std=c++17", "-I", CSRC, str(tmp_path / "p.cpp"), "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
