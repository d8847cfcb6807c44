// How latent attention's work is cut: shared by its kernels, its launcher and the
// tests of the cut.
//
// A unit is 128 of a sequence's stacked query rows (row r = node * heads + head:
// all heads share the keys) over all its keys.  The units are laid end to end,
// sequence by sequence, and cut into equal shares, one a workgroup; the pieces of
// units that were cut are merged by a second kernel.
#pragma once

#include <stdint.h>

namespace ltd {
namespace latent {

constexpr int kUnitRows = 128;
constexpr int kKeyTile = 32;
constexpr int kUnitCost = 6;              // what a unit costs beside its tiles, in tiles
constexpr int kMinShare = kUnitCost + 4;  // a share at least

constexpr int64_t units_of(int64_t n, int64_t heads) { return (n * heads + kUnitRows - 1) / kUnitRows; }
constexpr int64_t tiles_of(int64_t P, int64_t n) { return (P + n + kKeyTile - 1) / kKeyTile; }
// Length of a sequence's units laid end to end (each its own cost, then its tiles).
constexpr int64_t length_of(int64_t P, int64_t n, int64_t heads) {
  return units_of(n, heads) * (kUnitCost + tiles_of(P, n));
}
// floor(x / y) for 0 <= x < 2^52, by one division in float64 (a quotient just below an
// integer is below it by 1 / x or more of itself, which float64 keeps apart).
constexpr int64_t quotient(int64_t x, int64_t y) {
  return static_cast<int64_t>(static_cast<double>(x) / static_cast<double>(y));
}
// Length of a share, for `total` and W workgroups.
constexpr int64_t share_of(int64_t total, int W) {
  const int64_t even = quotient(total + W - 1, W);
  return even < kMinShare ? kMinShare : even;
}
// The tile that a unit's place `at` belongs to (its own cost comes first).
constexpr int64_t tile_at(int64_t at) { return at < kUnitCost ? 0 : at - kUnitCost; }
// Workgroups a call can use at most.
constexpr int workgroups(int64_t B, int64_t Nmax, int64_t heads, int64_t max_prefix, int cus) {
  const int64_t total = B * length_of(max_prefix, Nmax, heads);
  const int64_t most = (total + kMinShare - 1) / kMinShare;
  return static_cast<int>(most < cus ? most : cus);
}

}  // namespace latent
}  // namespace ltd
