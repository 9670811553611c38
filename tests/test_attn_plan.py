"""Which workgroup of the attention over a paged cache sees which tokens: the arithmetic that launch and kernel share, compiled as a plain
C++ program and enumerated (CPU only)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(tmp_path, body):
    gxx = shutil.which("g++") or shutil.which("clang++")
    if gxx is None:
        pytest.skip("no host compiler")
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    with open(src, "w") as f:
        f.write("#include <cstdio>\n#include <random>\n#include <vector>\n#include \"attn_plan.h\"\nusing namespace moe;\n" + body)
    subprocess.run([gxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2508_02317_amd", "csrc"), src, "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout
    return res.stdout


def test_every_tile_has_one_owner_and_pieces_follow_each_other(tmp_path):
    _run(tmp_path, """int main() {
      for (int total = 0; total < 3000; total += total < 1100 ? 1 : 37)
        for (int blocks : {1, 2, 7, 64, 255, kAttnMaxBlocks}) {
          const AttnCut c = attn_cut(total, blocks);
          if (attn_begin(c, 0) != 0 || attn_begin(c, blocks) != total) { printf("ends: %d on %d\\n", total, blocks); return 1; }
          for (int b = 0; b < blocks; ++b) {
            const int n = attn_begin(c, b + 1) - attn_begin(c, b);
            if (n < c.size || n > c.size + 1) { printf("piece: %d on %d\\n", total, blocks); return 1; }
            for (int t = attn_begin(c, b); t < attn_begin(c, b + 1); ++t)
              if (attn_owner(c, t) != b) { printf("owner of %d: %d on %d\\n", t, total, blocks); return 1; }
          }
        }
      return 0;
    }""")


def test_every_token_of_a_context_lies_in_one_tile(tmp_path):
    _run(tmp_path, """int main() {
      for (int sub : {16, 32})
        for (int held : {0, 16, 128, 400})
          for (int window : {0, 1, 15, 16, 17, 100, 128, 399, 1000})
            for (int len = -2; len < 420; ++len) {
              const AttnSpan s = attn_span(len, held, window, sub, 4 * sub);
              const int n = len < 0 ? 0 : len > held ? held : len, lo = window && n > window ? n - window : 0;
              if (s.lo != lo || s.len != n || s.base % sub || s.base > lo || s.base <= lo - sub) { printf("len %d window %d\\n", len, window); return 1; }
              const int end = s.base + s.tiles * 4 * sub;
              if (end < n || (s.tiles && end - 4 * sub >= n) || (n == 0) != (s.tiles == 0)) { printf("tiles: len %d window %d\\n", len, window); return 1; }
            }
      return 0;
    }""")


def test_a_cut_context_is_put_together_from_the_slots_that_were_written(tmp_path):
    # the kernel's walk of a workgroup's piece and the join's list of slots, over random lengths
    _run(tmp_path, """int main() {
      std::mt19937 r(3);
      for (int c = 0; c < 3000; ++c) {
        const int B = 1 + r() % 9, units = 1 + r() % 5, W = 1 + r() % 40;
        std::vector<int> tiles(B);
        int total = 0;
        for (int& t : tiles) { t = r() % 3 ? r() % 30 : 0; total += t; }
        total *= units;
        const AttnCut cut = attn_cut(total, W);
        std::vector<std::vector<int>> slot(2 * W);                    // unit and number of tiles of what a slot holds
        std::vector<int> first(B * units, -2), last(B * units, -2), whole(B * units, 0);
        for (int me = 0; me < W; ++me) {
          int at = attn_begin(cut, me), b = 0, before = 0;
          const int end = attn_begin(cut, me + 1);
          while (at < end) {
            while (at >= (before + tiles[b]) * units) before += tiles[b++];
            const int u = (at - before * units) / tiles[b], ub = before * units + u * tiles[b], ue = ub + tiles[b];
            const int to = end < ue ? end : ue, id = b * units + u, s = 2 * me + (at == attn_begin(cut, me) ? 0 : 1);
            const bool complete = at == ub && to == ue;
            if (complete) ++whole[id];
            else { if (!slot[s].empty()) { printf("slot written twice\\n"); return 1; } slot[s] = {id, to - at}; }
            if (at == ub) { first[id] = complete ? -1 : s; last[id] = attn_owner(cut, ue - 1); }
            at = to;
          }
        }
        for (int b = 0; b < B; ++b) for (int u = 0; u < units; ++u) {
          const int id = b * units + u;
          if (!tiles[b]) { if (first[id] != -2) return 1; continue; }
          if (first[id] == -1) { if (whole[id] != 1) return 1; continue; }
          int seen = 0;
          const int w0 = first[id] >> 1;
          for (int i = 0; i <= last[id] - w0; ++i) {
            const auto& s = slot[i == 0 ? first[id] : 2 * (w0 + i)];
            if (s.empty() || s[0] != id) { printf("case %d: a piece is another's\\n", c); return 1; }
            seen += s[1];
          }
          if (seen != tiles[b] || whole[id]) { printf("case %d: %d of %d tiles\\n", c, seen, tiles[b]); return 1; }
        }
      }
      return 0;
    }""")
