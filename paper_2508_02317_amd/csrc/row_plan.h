// How rows are dealt out to lanes, waves and workgroups: integer arithmetic of norm.hip and balance.hip, without anything of a GPU in it, so that a plain C++
// program can enumerate it (tests/test_row_plan.py).
#pragma once
#include <stdint.h>

namespace moe {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 by a multiplication: mul = floor(2^32 (2^shift - d) / d) + 1 with 2^(shift - 1) < d <= 2^shift
struct Divisor { uint32_t mul, shift; };
constexpr Divisor divisor(uint32_t d) {
  uint32_t shift = 0;
  while ((uint64_t{1} << shift) < d) ++shift;
  return {static_cast<uint32_t>((((uint64_t{1} << shift) - d) << 32) / d + 1), shift};
}
constexpr uint32_t divide(uint32_t n, Divisor d) { return (static_cast<uint32_t>((static_cast<uint64_t>(n) * d.mul) >> 32) + n) >> d.shift; }

// A row of `all` pieces of 16 bytes: `lanes` lanes (a power of two) of each of `waves` waves (more than one only with 64 lanes), up to `pieces` pieces each;
// piece (p * waves * lanes + lane) is the p-th of a lane.  No more than `most` pieces a lane while 16 waves suffice.
struct RowSplit { int lanes, waves, pieces; };
constexpr RowSplit split_row(int all, int most) {
  RowSplit s{1, 1, 1};
  while (s.lanes < 64 && s.lanes < all) s.lanes *= 2;
  while (s.waves * 64 * most < all && s.waves < 16) s.waves *= 2;
  while (s.lanes * s.waves * s.pieces < all) s.pieces *= 2;
  return s;
}
constexpr int rows_at_once(int pieces, int most) { return pieces < most ? most / pieces : 1; }
constexpr int threads_of(const RowSplit& s, int least) { return s.waves * 64 > least ? s.waves * 64 : least; }
constexpr int groups_of(const RowSplit& s, int threads) { return s.waves > 1 ? threads / 64 / s.waves : threads / s.lanes; }
// workgroups of `threads` threads that take rows_at_once(s.pieces, most) rows a group and turn
constexpr int blocks_of(int rows, const RowSplit& s, int threads, int most, int most_blocks) {
  const int step = groups_of(s, threads) * rows_at_once(s.pieces, most), n = rows / step + (rows % step != 0);
  return n < most_blocks ? n : most_blocks;
}

// A row of E columns in one wave: up to `most` pieces of four columns a lane where 64 lanes suffice for that, as many as it takes otherwise.
struct ColumnSplit { int row, lanes, pieces; };        // row: E rounded up to whole pieces
constexpr ColumnSplit split_columns(int E, int most) {
  const int all = (E + 3) / 4;
  ColumnSplit s{4 * all, 1, 1};
  while (s.lanes < 64 && s.lanes * most < all) s.lanes *= 2;
  while (s.lanes * s.pieces < all) s.pieces *= 2;
  return s;
}

}  // namespace moe
