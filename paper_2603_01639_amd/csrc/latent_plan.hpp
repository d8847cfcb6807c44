// How latent attention's work is cut: shared by its kernels, its launcher and the
// tests of the cut.
//
// A unit is up to 128 of a sequence's stacked query rows (row r = node * heads + head:
// all heads share the keys) over all its keys.  The units are laid end to end,
// sequence by sequence, and cut into equal shares, one a workgroup; the pieces of
// units that were cut are merged by a second kernel.
#pragma once

#include <stdint.h>

namespace ltd {
namespace latent {

constexpr int kKeyTile = 32;
constexpr int kRows = 128;    // stacked rows of a unit ...
constexpr int kFewRows = 16;  // ... and the most of a call that takes the kernel for few rows
// How a kernel's calls are cut: rows of a unit, what a unit costs beside its tiles (in
// tiles: the workgroup that begins one behind another's last piece loads queries, and
// stores a piece, twice), and the shortest share.  A share may lie within a unit's own
// cost and has nothing to do then.  (With a cost of 6 and shares of 10, 4 and 8 for few
// rows, the workgroups with two units' pieces end last: one token of 16 sequences of 16 heads
// over 1024 to 8192 keys 35.8 us a call, 33.0 so, over 500 to 1500 27.8 and 22.4; 8 nodes of 128
// heads over 2048 keys 36.8 and 31.9, 60 nodes of 16 heads over 2041 40.0 and 35.8, over 16384 64.1
// and 61.9.  Shares of 3, or costs of 16 and 20, changed nothing beyond 2%.)
struct Cut {
  int rows, cost, min_share;
};
constexpr Cut kMany{kRows, 12, 4};
constexpr Cut kFew{kFewRows, 8, 4};
// Calls of up to 16 stacked rows a sequence (one token of a few heads) have a kernel of
// their own.
constexpr Cut cut_of(int64_t Nmax, int64_t heads) {
  return Nmax * heads <= kFewRows ? kFew : kMany;
}

constexpr int64_t units_of(int64_t n, int64_t heads, const Cut& c) { return (n * heads + c.rows - 1) / c.rows; }
constexpr int64_t tiles_of(int64_t P, int64_t n) { return (P + n + kKeyTile - 1) / kKeyTile; }
// Length of a sequence's units laid end to end (each its own cost, then its tiles).
constexpr int64_t length_of(int64_t P, int64_t n, int64_t heads, const Cut& c) {
  return units_of(n, heads, c) * (c.cost + tiles_of(P, n));
}
// floor(x / y) for 0 <= x < 2^52, by one division in float64 (a quotient just below an
// integer is below it by 1 / x or more of itself, which float64 keeps apart).
constexpr int64_t quotient(int64_t x, int64_t y) {
  return static_cast<int64_t>(static_cast<double>(x) / static_cast<double>(y));
}
// Length of a share, for `total` and W workgroups.
constexpr int64_t share_of(int64_t total, int W, const Cut& c) {
  const int64_t even = quotient(total + W - 1, W);
  return even < c.min_share ? c.min_share : even;
}
// The tile that a unit's place `at` belongs to (its own cost comes first).
constexpr int64_t tile_at(int64_t at, const Cut& c) { return at < c.cost ? 0 : at - c.cost; }
// row / kv_rows by a multiplication: floor(2 row * magic / 2^(32 + shift)).  With kv_rows <=
// 2^shift and magic = floor(2^(31 + shift) / kv_rows) + 1 it is exact for every row below
// 2^31.
struct RowDivisor {
  uint32_t magic;
  int shift;
};
constexpr RowDivisor row_divisor(int kv_rows) {
  int shift = 0;
  while (shift < 31 && (uint32_t{1} << shift) < static_cast<uint32_t>(kv_rows)) ++shift;
  return {static_cast<uint32_t>((uint64_t{1} << (31 + shift)) / static_cast<uint32_t>(kv_rows) + 1), shift};
}
// Workgroups a call can use at most.
constexpr int workgroups(int64_t B, int64_t Nmax, int64_t heads, int64_t max_prefix, int cus) {
  const Cut c = cut_of(Nmax, heads);
  if (B >= static_cast<int64_t>(cus) * c.min_share) return cus;  // (the product below could pass 2^63)
  // (one unit that is too short for two shares needs no merge)
  if (B * units_of(Nmax, heads, c) == 1 && tiles_of(max_prefix, Nmax) <= c.min_share) return 1;
  const int64_t total = B * length_of(max_prefix, Nmax, heads, c);
  const int64_t most = (total + c.min_share - 1) / c.min_share;
  return static_cast<int>(most < cus ? most : cus);
}

}  // namespace latent
}  // namespace ltd
