// How attention over an 8-bit cache cuts its short units (at most 32 stacked
// rows) into splits.  All of a call's splits have one length, in whole key
// tiles, such that the splits number at most `target` workgroups.  It follows
// from the call's own lengths; max_prefix bounds the launch and the workspace,
// not the length (a graph captured for a model's longest prefix cuts as a call
// with tight bounds does: 16 sequences of 64/8 heads over 1024 to 8192 keys, one
// node, bounds of 8192, 32768 and 131072: 39.6, 40.4 and 40.6 us).  Only where
// that length would pass kMaxKeys are there more splits than workgroups: up to
// the next multiple of `target`, and each workgroup takes several.
//
// Everything here is constexpr, so the same functions run in the kernel and in a
// plain host build (how they are tested without a GPU).
#pragma once

#include <stdint.h>

namespace ltd {
namespace few {

constexpr int kKeyTile = 64;
constexpr int kMinKeys = 128;      // shortest split: a 32-key block for each of four waves
constexpr int kMaxKeys = 7680;     // longest: its block ids (16 rows a page at least) fit the kernel's table
constexpr int kMostSplits = 1024;  // splits of a unit that the merge takes

// Workgroups that the splits of `units` units are cut for, with `per_cu` of them
// resident on each of `cus` compute units.  Up to a quarter as many units as fit
// the card at once: that many, so that all splits run side by side (16 sequences
// of 64/8 heads, 1024 to 8192 keys: 41.0 us, 43.3 in shorter ones).  With more
// units the remainders of so few splits would leave compute units idle, and the
// splits are cut into 4 a compute unit beyond the units, which the hardware deals
// out as they end (in us, for a grid of 2, 3, 4 and 6 times the units: 256 units of
// 500 to 6000 keys 67 / 64 / 57 / 57, 384 of 2000 52 / 50 / 52 / 56, 512 of 200 to
// 3000 62 / 57 / 58 / 65, 1024 of 100 to 1500 65 / 69 / 73 / 85).
constexpr int64_t target(int64_t units, int per_cu, int cus) {
  const int64_t resident = static_cast<int64_t>(per_cu) * cus;
  if (4 * units <= resident) return resident < kMostSplits ? resident : kMostSplits;
  return units + (4 * cus < kMostSplits ? 4 * cus : kMostSplits - 1);
}

// Splits that a call can come to, and workgroups of its launch.
constexpr int64_t most_splits(int64_t units, int64_t max_prefix, int64_t target) {
  const int64_t longest = max_prefix > kMaxKeys ? (max_prefix + kMaxKeys - 1) / kMaxKeys : 1;
  const int64_t shortest = max_prefix > kMinKeys ? (max_prefix + kMinKeys - 1) / kMinKeys : 1;
  const int64_t wide = units * longest > target ? units * longest + target : target;
  return wide < units * shortest ? wide : units * shortest;
}
constexpr int64_t workgroups(int64_t units, int64_t max_prefix, int64_t target) {
  const int64_t most = most_splits(units, max_prefix, target);
  return most < target ? most : target;
}

struct Length {
  int keys;
  int rounds;  // the splits number at most rounds * target
};

// Shortest length in more than one round: a unit has at most kMostSplits of them
// (bounds above 3.9 million rows can lengthen it).
constexpr int rounds_min_keys(int max_prefix) {
  constexpr int kRows = kMostSplits * kKeyTile;
  const int keys = (max_prefix / kRows + (max_prefix % kRows != 0 ? 1 : 0)) * kKeyTile;
  return keys > kMaxKeys / 2 ? keys : kMaxKeys / 2;
}

// One sequence.  A length of more than P Hkv / (W - Hkv) fits W workgroups, for the
// splits number at most P Hkv / length + Hkv.  (The shortest that fits puts more
// workgroups to use, but the merge has more to read: one of 32/8 heads, 16384 keys,
// one node: 17.6 us a call with 256 keys a split, 16.7 with 320; 8192 keys 14.0 and
// 14.0, 32768 keys 22.0 and 22.0.)
constexpr Length one_length(int P, int Hkv, int target, int max_prefix) {
  int rounds = 1, least = kMinKeys;
  int64_t tiles = static_cast<int64_t>(P) * Hkv / (target - Hkv) / kKeyTile + 1;
  if (tiles > kMaxKeys / kKeyTile) {
    const int64_t splits = static_cast<int64_t>((P + kMaxKeys - 1) / kMaxKeys) * Hkv;  // at kMaxKeys
    rounds = static_cast<int>((splits + target - 1) / target);
    tiles = static_cast<int64_t>(P) * Hkv / (static_cast<int64_t>(rounds) * target - Hkv) / kKeyTile + 1;
    if (rounds > 1) least = rounds_min_keys(max_prefix);
  }
  const int keys = tiles < kMaxKeys / kKeyTile ? static_cast<int>(tiles) * kKeyTile : kMaxKeys;
  return Length{keys > least ? keys : least, rounds};
}

// A batch of `units` units, T prefix keys in all its sequences; splits(length)
// counts the call's splits.  As above a length of more than T Hkv / (W - units)
// fits W workgroups; one below T Hkv / W does not.  Where the splits run side by
// side, or nearly, the longest is what the call takes, and a search finds the
// shortest length that fits (16 sequences of 1024 to 8192 keys, 64/8 heads: 1280 to
// 1536 keys instead of 1472 to 1792, 39.5 us a call instead of 42.0; in more rounds
// it has nothing to give: 64 sequences of 32/8 heads, 200 to 3000 keys, 60.2 us
// with it and 59.5 without, 128 of 100 to 1500 71.1 and 65.1).  (Float estimates:
// the upper one raised so that it is never short of the quotient, the lower one
// mattering in whole tiles only.)
template <class Splits>
constexpr Length batch_length(int64_t T, int Hkv, int units, int target, int max_prefix, Splits splits) {
  const float keys = static_cast<float>(T) * static_cast<float>(Hkv);
  float W = static_cast<float>(target);
  float most = keys / (W - static_cast<float>(units)) * 1.00001f;
  int rounds = 1, lo = kMinKeys, hi = kMaxKeys;
  if (most >= kMaxKeys) {
    const int at_most = splits(kMaxKeys);
    if (at_most > target) {
      rounds = (at_most + target - 1) / target;
      W *= static_cast<float>(rounds);
      most = keys / (W - static_cast<float>(units)) * 1.00001f;
      lo = rounds_min_keys(max_prefix);
    }
  }
  if (most < kMaxKeys) hi = (static_cast<int>(most) / kKeyTile + 1) * kKeyTile;
  if (hi < lo) hi = lo;
  if (4 * units > target) return Length{hi, rounds};
  const int below = static_cast<int>(keys / W) / kKeyTile * kKeyTile;
  if (lo < below) lo = below;
  while (lo < hi) {  // (whole tiles both; hi fits)
    const int mid = (lo + hi) / (2 * kKeyTile) * kKeyTile;
    if (splits(mid) <= rounds * target) hi = mid;
    else lo = mid + kKeyTile;
  }
  return Length{hi, rounds};
}

}  // namespace few
}  // namespace ltd
