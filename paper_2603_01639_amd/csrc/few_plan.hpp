// How attention over an 8-bit cache cuts its short units (at most 32 stacked
// rows) into splits.  All of a call's splits have one length, in whole key
// tiles, such that the splits number at most `target` workgroups.  It follows
// from the call's own lengths; max_prefix bounds the launch and the workspace,
// not the length (a graph captured for a model's longest prefix cuts as a call
// with tight bounds does: 16 sequences of 64/8 heads over 1024 to 8192 keys, one
// node, bounds of 8192, 32768 and 131072: 39.4, 38.8 and 38.8 us).  Only where
// that length would be too long are there more splits, and a launch whose bounds
// allow so has the workgroups for a wider cut, which take one split after
// another where even that does not do.
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

// Workgroups that the splits of `units` units are cut for, with `resident` of them
// on the card at once.  Up to a quarter as many units as that: as many as are
// resident, so that all splits run side by side (16 sequences of 64/8 heads, 1024
// to 8192 keys: 41.0 us, 43.3 in shorter ones).  With more units the remainders of
// so few splits would leave compute units idle, and the splits are cut into twice
// the resident ones beyond the units, which the hardware deals out as they end (in
// us, for a grid of 2, 3, 4 and 6 times the units: 256 units of 500 to 6000 keys 67 /
// 64 / 57 / 57, 384 of 2000 52 / 50 / 52 / 56, 512 of 200 to 3000 62 / 57 / 58 / 65,
// 1024 of 100 to 1500 65 / 69 / 73 / 85).
constexpr int64_t target(int64_t units, int resident) {
  if (4 * units <= resident) return resident < kMostSplits ? resident : kMostSplits;
  return units + (2 * resident < kMostSplits ? 2 * resident : kMostSplits - 1);
}

// Workgroups of the wider cut, and longest split that the target is kept for.
// Splits that are dealt out end within half the longest of each other then: 64
// sequences of 32/8 heads, 8000 to 24000 keys, 395 us a call, 430 with splits of
// up to kMaxKeys.
constexpr int64_t round_width(int64_t units, int resident) {
  const int64_t t = target(units, resident);
  return 4 * units <= resident ? t : 2 * t;
}

constexpr int longest(int64_t target, int64_t width) { return width > target ? kMaxKeys / 2 : kMaxKeys; }

// Whether bounds allow the wider cut, the splits that a call can come to, and the
// workgroups of its launch.
constexpr int64_t pieces(int64_t max_prefix, int64_t keys) { return max_prefix > keys ? (max_prefix + keys - 1) / keys : 1; }
constexpr bool may_widen(int64_t units, int64_t max_prefix, int resident) {
  const int64_t t = target(units, resident);
  return units * pieces(max_prefix, longest(t, round_width(units, resident))) > t;
}
constexpr int64_t most_splits(int64_t units, int64_t max_prefix, int resident) {
  const int64_t t = target(units, resident), shortest = units * pieces(max_prefix, kMinKeys);
  if (!may_widen(units, max_prefix, resident)) return t < shortest ? t : shortest;
  const int64_t rounds = units * pieces(max_prefix, kMaxKeys) + round_width(units, resident);
  const int64_t in_rounds = units * pieces(max_prefix, kMaxKeys / 2);
  const int64_t wide = rounds < in_rounds ? rounds : in_rounds;
  return wide > t ? wide : t;
}
constexpr int64_t workgroups(int64_t units, int64_t max_prefix, int resident) {
  const int64_t most = most_splits(units, max_prefix, resident);
  return may_widen(units, max_prefix, resident) && most > round_width(units, resident) ? round_width(units, resident) : most;
}

struct Length {
  int keys;
  int rounds;  // splits of a workgroup at most
};

// Shortest length of the wider cut: a unit has at most kMostSplits of them (bounds
// above 3.9 million rows can lengthen it).
constexpr int wide_min_keys(int max_prefix) {
  constexpr int kRows = kMostSplits * kKeyTile;
  const int keys = (max_prefix / kRows + (max_prefix % kRows != 0 ? 1 : 0)) * kKeyTile;
  return keys > kMaxKeys / 2 ? keys : kMaxKeys / 2;
}

// One sequence.  A length of more than P Hkv / (W - Hkv) fits W workgroups, for the
// splits number at most P Hkv / length + Hkv.  (The shortest that fits puts more
// workgroups to use, but the merge has more to read: one of 32/8 heads, 16384 keys,
// one node: 17.6 us a call with 256 keys a split, 16.7 with 320; 8192 keys 14.0 and
// 14.0, 32768 keys 22.0 and 22.0.)
constexpr Length one_length(int P, int Hkv, int target, int width, int max_prefix) {
  int rounds = 1, least = kMinKeys;
  int64_t tiles = static_cast<int64_t>(P) * Hkv / (target - Hkv) / kKeyTile + 1;
  if (tiles > kMaxKeys / kKeyTile) {
    const int64_t splits = static_cast<int64_t>((P + kMaxKeys - 1) / kMaxKeys) * Hkv;  // at kMaxKeys
    if (splits > target) {
      rounds = static_cast<int>((splits + width - 1) / width);
      tiles = static_cast<int64_t>(P) * Hkv / (static_cast<int64_t>(rounds) * width - Hkv) / kKeyTile + 1;
      least = wide_min_keys(max_prefix);
    }
  }
  const int keys = tiles < kMaxKeys / kKeyTile ? static_cast<int>(tiles) * kKeyTile : kMaxKeys;
  return Length{keys > least ? keys : least, rounds};
}

// A batch of `units` units, T prefix keys in all its sequences; splits(length)
// counts the call's splits.  As above a length of more than T Hkv / (W - units)
// fits W workgroups; one below T Hkv / W does not.  Where the splits run side by
// side, or nearly, the longest is what the call takes, and a search finds the
// shortest length that fits (16 sequences of 1024 to 8192 keys, 64/8 heads: 1280 to
// 1536 keys instead of 1472 to 1792, 39.5 us a call instead of 42.0; where many more
// are dealt out it has nothing to give: 64 sequences of 32/8 heads, 200 to 3000
// keys, 60.2 us with it and 59.5 without, 128 of 100 to 1500 71.1 and 65.1).  (Float
// estimates: the upper one raised so that it is never short of the quotient, the
// lower one mattering in whole tiles only.)
template <class Splits>
constexpr Length batch_length(int64_t T, int Hkv, int units, int target, int width, int max_prefix, Splits splits) {
  const float keys = static_cast<float>(T) * static_cast<float>(Hkv);
  int W = target, rounds = 1, lo = kMinKeys, hi = kMaxKeys;
  float most = keys / static_cast<float>(W - units) * 1.00001f;
  if (most >= longest(target, width)) {
    hi = longest(target, width);
    if (splits(hi) > target) {
      hi = kMaxKeys;
      rounds = (splits(kMaxKeys) + width - 1) / width;
      W = rounds * width;
      most = W > units ? keys / static_cast<float>(W - units) * 1.00001f : static_cast<float>(kMaxKeys);
      lo = wide_min_keys(max_prefix);
    }
  }
  if (most < hi) hi = (static_cast<int>(most) / kKeyTile + 1) * kKeyTile;
  if (hi < lo) hi = lo;
  if (4 * units > target) return Length{hi, rounds};
  const int below = static_cast<int>(keys / static_cast<float>(W)) / kKeyTile * kKeyTile;
  if (lo < below) lo = below;
  while (lo < hi) {  // (whole tiles both; hi fits)
    const int mid = (lo + hi) / (2 * kKeyTile) * kKeyTile;
    if (splits(mid) <= W) hi = mid;
    else lo = mid + kKeyTile;
  }
  return Length{hi, rounds};
}

}  // namespace few
}  // namespace ltd
