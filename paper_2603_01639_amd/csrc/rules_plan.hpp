// How the sampling rules' launch groups a sequence's nodes, in plain integers: the
// launch's and, in a host build, its tests'.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace ltd {
namespace rules {

// Nodes of a workgroup at most, for the argmax and for written rows.
constexpr int nodes_max(bool argmax) { return argmax ? 8 : 4; }

// As many nodes a workgroup as leave no more of them (of `threads` threads, for
// `chunks` chunks of the vocabulary) than fit the card's `cus` compute units at
// once, up to 4 where rows are written (in us, for 2, 3, 4, 6 and 8: 16 trees of 16
// to 96 nodes, 128256 tokens 200 / 198 / 196 / 206 / 211 without and 203 / 194 / 190 /
// 197 / 201 with masks; 64 of 1 to 16 123 / 124 / 125 / 131 / 136) and up to 8 for the
// argmax.  Its workgroups, one to a compute unit by their LDS, come to an end at once
// then; in more rounds than two 7 nodes do better than 8, and 6 as well as 7 (in us,
// for 4, 6, 7 and 8: 16 trees of 60, 32000 tokens 41 / 48 / 50 / 37; of 128256 tokens,
// 16 of 16 to 128 nodes 148 / 136 / 137 / 141, 32 of 16 to 64 171 / 149 / 150 / 160, 64
// of 1 to 16 113 / 80 / 80 / 94).
constexpr int nodes(int64_t B, int Nmax, int chunks, bool argmax, int threads, int cus) {
  const int64_t rows = B * Nmax * chunks;
  const int64_t card = static_cast<int64_t>(cus) * (1024 / threads);
  const int most = nodes_max(argmax);
  const int64_t fullest = B * ((Nmax + most - 1) / most) * chunks;
  const int limit = argmax && fullest > 2 * card ? most - 1 : most;
  return static_cast<int>(std::min<int64_t>((rows + card - 1) / card, limit));
}

}  // namespace rules
}  // namespace ltd
