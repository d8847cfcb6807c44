// How latent attention's work is cut: shared by its kernels, its launcher and the
// tests of the cut.
//
// A unit is 128 of a sequence's stacked query rows (row r = node * heads + head:
// all heads share the keys) over all its keys.  The units' key tiles are laid
// end to end, sequence by sequence, and cut into equal shares, one a workgroup;
// unit pieces that a cut leaves are merged by a second kernel.
#pragma once

#include <stdint.h>

namespace ltd {
namespace latent {

constexpr int kUnitRows = 128;
constexpr int kKeyTile = 32;
constexpr int kMinShare = 4;  // key tiles of a share at least

constexpr int64_t units_of(int64_t n, int64_t heads) { return (n * heads + kUnitRows - 1) / kUnitRows; }
constexpr int64_t tiles_of(int64_t P, int64_t n) { return (P + n + kKeyTile - 1) / kKeyTile; }
// Key tiles of a share, for `total` tiles and W workgroups.
constexpr int64_t share_of(int64_t total, int W) {
  const int64_t even = (total + W - 1) / W;
  return even < kMinShare ? kMinShare : even;
}
// Workgroups a call can use at most.
constexpr int workgroups(int64_t B, int64_t Nmax, int64_t heads, int64_t max_prefix, int cus) {
  const int64_t total = B * units_of(Nmax, heads) * tiles_of(max_prefix, Nmax);
  const int64_t most = (total + kMinShare - 1) / kMinShare;
  return static_cast<int>(most < cus ? most : cus);
}

}  // namespace latent
}  // namespace ltd
