// Launch plans of the matrix-core attention (attn_mfma.hpp), and its launch over a 16-bit
// cache.  The kernels over an 8-bit cache are compiled apart (attn_mfma_q8.hip): beside
// them in one file hipcc schedules the 16-bit ones' tile loop differently, and 16
// sequences' verify step takes 351 us instead of 348.
#include "attn_mfma.hpp"
#include "few_plan.hpp"

namespace ltd {
namespace {

constexpr int kMinTilesPerWg = 2;   // a share shorter than this is mostly fixed cost

// Stacked-row tiles and key tiles of the longest unit the launch allows.
int64_t max_unit_tiles(const AttnShape& s) {
  return (s.max_prefix + kKT - 1) / kKT + (s.Nmax + kKT - 1) / kKT;
}

// Whether every workgroup's share of a grid of W fits the paged block table
// staged in LDS: a share is at most one unit's keys and, on the axis, at most
// (C / W) / 2 + 1 key tiles (the smallest tile weight is 2), plus the tree.
bool share_fits(const AttnShape& s, int W) {
  if (s.max_blocks <= 0) return true;  // contiguous cache: no table
  const int64_t unit_rows = static_cast<int64_t>(s.max_prefix) + s.Nmax;
  const int64_t axis_tiles =
      max_units(s) *
      plan::unit_extent(static_cast<int>((s.max_prefix + kKT - 1) / kKT), (s.Nmax + kKT - 1) / kKT) *
      plan::tile_weight(8);
  const int64_t share_rows =
      std::min(unit_rows, (axis_tiles / W / 2 + 2) * kKT + static_cast<int64_t>(s.Nmax));
  return share_rows / s.kv_rows + 2 <= kMaxSplitBlocks;
}

// Stream plan grid: W workgroups, a power of two of at least 8 (one eighth of
// the axis per XCD; the partition's arithmetic is then shifts),
// at most one resident round (one workgroup per compute unit), each with at
// least kMinTilesPerWg key tiles of the largest call the shape allows.  It
// does not depend on the cache layout, so neither does the workspace.
int choose_grid(const AttnShape& s, int num_cus) {
  const int64_t tiles = max_units(s) * max_unit_tiles(s);
  const int64_t want = std::min<int64_t>(std::min(num_cus, kMaxGrid), tiles / kMinTilesPerWg);
  int W = 8;
  while (2 * W <= want) W *= 2;
  return W;
}

constexpr size_t kDescBytes = 64;  // sizeof(MergeDesc)

}  // namespace

// Single sequences take the split plan (every unit has the same length, and
// the plan's cost model picks the split length and whether the tree keys get
// a split of their own); batches take the stream plan, which balances units
// of different lengths, unless a paged layout's blocks are so small that a
// workgroup's share could span more block ids than the LDS table holds (the
// split plan shortens its splits for those).
bool use_stream(const AttnShape& s) { return s.B > 1 && share_fits(s, choose_grid(s, 256)); }

// Longest split (in keys, a multiple of the key tile) whose paged block ids
// fit the LDS table: the last split's rows (its prefix keys plus up to Nmax
// tree keys) span at most (keys + Nmax) / kv_rows + 2 blocks.  A contiguous
// cache has no such bound.
int64_t split_key_cap(const AttnShape& s) {
  if (s.max_blocks <= 0) return int64_t{1} << 40;
  const int64_t cap = static_cast<int64_t>(kMaxSplitBlocks - 2) * s.kv_rows - s.Nmax;
  return cap / kKT * kKT;
}

// The smallest cap over every cache layout (paged with 1-row blocks); the
// supported range and the workspace size use it, so that neither depends on
// the layout of the call.
int64_t worst_split_key_cap(const AttnShape& s) {
  AttnShape w = s;
  w.kv_rows = 1;
  w.max_blocks = 1;
  return split_key_cap(w);
}

// Two key groups when every unit of the call fits two waves' rows.  A compute
// unit has four SIMDs: with one group, units of 33 to 64 rows leave two of them
// without work and shorter ones three, which the second group puts to use; from
// 65 rows on the waves of one group already cover three or four SIMDs, and the
// join costs more than it gives.  One group against two, a call: 32/8 heads,
// 16 nodes (64 rows), prefix 128: 9.0 / 8.6 us, 4096: 12.2 / 12.1, 16384: 21.4 /
// 20.3, 16 sequences of prefix 1024: 25.9 / 24.1; 24 nodes (96 rows): 9.0 / 10.1,
// 12.4 / 13.8, 21.8 / 22.1 and 26.5 / 28.2; 32 nodes 9.0 / 10.5, 12.8 / 14.2,
// 23.3 / 23.2 and 27.8 / 29.7.  Head size 64 and ungrouped queries have the line
// in much the same place.  (Mixed calls stay with one group: a choice per unit, with
// both loops in one kernel, overran the instruction cache and lost 2-4% on
// batches of 32- to 220-row units.)
bool two_key_groups(const AttnShape& s) { return s.Hq / s.Hkv * s.Nmax <= kTileRows / 4; }

// Whether every unit of a call over an 8-bit cache has at most 32 rows
// (attn_few_kernel).
bool few_rows(const AttnShape& s) { return s.scale_rows > 0 && s.Hq / s.Hkv * s.Nmax <= kFewRows; }

void plan_few(const AttnShape& s, int num_cus, AttnPlan* p) {
  const int64_t units = static_cast<int64_t>(s.B) * s.Hkv;
  const int resident = kFewPerCu * num_cus;
  p->mfma = true;
  p->few = true;
  p->stream = false;
  p->tile_rows = kFewRows;
  p->row_tiles = 1;
  p->max_splits = s.max_prefix > few::kMinKeys ? 2 : 1;  // (whether a unit can be cut at all)
  p->few_target = static_cast<int>(few::target(units, resident));
  p->few_width = static_cast<int>(few::round_width(units, resident));
  p->few_wide = few::may_widen(units, s.max_prefix, resident);
  p->few_slots = few::most_splits(units, s.max_prefix, resident);
  p->grid = static_cast<int>(few::workgroups(units, s.max_prefix, resident));
  p->workspace_bytes = static_cast<size_t>(p->few_slots) * kFewRows * part_row_bytes(s) +
                       static_cast<size_t>(units) * sizeof(FewDesc);
}

// Estimated time of a split plan, in key tiles of a 256-row unit (about 2 us).
// `tile` is the cost of one key tile for the plan's units (less with two key
// groups).
static double plan_cost(int64_t P, int n, int64_t sk, bool alone, int64_t units, int64_t target, double tile) {
  constexpr double kFixedTiles = 3.0, kMaskTiles = 0.5, kMergeTiles = 2.5;
  const int64_t tps = sk / kKT;
  const int64_t tree_tiles = (n + kKT - 1) / kKT;
  const int64_t pre = (P + sk - 1) / sk;
  const int S = n_splits_of(static_cast<int>(P), n, static_cast<int>(sk), alone);
  double longest;
  if (pre <= 1) {
    longest = tile * static_cast<double>((P + kKT - 1) / kKT + tree_tiles) + kMaskTiles;
  } else {
    const int64_t last = (P - (pre - 1) * sk + kKT - 1) / kKT;
    const double tree_split =
        tile * static_cast<double>(S > pre ? tree_tiles : last + tree_tiles) + kMaskTiles;
    longest = std::max(tile * static_cast<double>(tps), tree_split);
  }
  const int64_t rounds = (units * S + target - 1) / target;
  return static_cast<double>(rounds) * (longest + kFixedTiles) +
         (S > 1 ? kMergeTiles + S / 32.0 : 0.0);
}

constexpr double kHalfTile = 0.55;  // a key tile's cost with two key groups

void plan_split(const AttnShape& s, int num_cus, AttnPlan* p) {
  const int G = s.Hq / s.Hkv;
  const int rows = G * s.Nmax;
  // A (sequence, kv head, row tile) unit is split along the keys into about
  // as many workgroups as keep one resident round of one workgroup per
  // compute unit busy (a second, nearly empty round would double the kernel
  // time).  That gives the shortest split considered; a split holds at least
  // two key tiles, at most the paged table's cap, and the merge kernel's
  // table bounds the number of splits.  From there up to the cap, the split
  // length (and whether the tree takes a split of its own) with the lowest
  // estimated time: this balances the split that carries the tree against
  // the others.  (Half-size units for longer trees too, to leave fewer compute
  // units idle, were slower: 240 rows over a prefix of 2048 on 8 kv heads
  // 14.1 us in 144 workgroups instead of 13.5 in 136.)
  p->tile_rows = rows <= kTileRows / 2 ? kTileRows / 2 : kTileRows;  // (halves a short call's workspace)
  p->row_tiles = (rows + p->tile_rows - 1) / p->tile_rows;
  const double tile = two_key_groups(s) ? kHalfTile : 1.0;
  const int64_t units = static_cast<int64_t>(s.B) * s.Hkv * p->row_tiles;
  const int64_t target = num_cus;
  const int64_t want = std::max<int64_t>(1, target / units);
  const int64_t mp = s.max_prefix;
  const int64_t cap = std::min(split_key_cap(s), static_cast<int64_t>(kMaxSplitTiles) * kKT);
  int64_t sk0 = (mp + want - 1) / want;
  sk0 = std::max<int64_t>(sk0, (mp + kMaxMergeSplits - 1) / kMaxMergeSplits);
  sk0 = std::max<int64_t>((sk0 + kKT - 1) / kKT * kKT, 2 * kKT);
  sk0 = std::min(sk0, cap);
  int64_t best_sk = sk0;
  bool best_alone = false;
  double best = plan_cost(mp, s.Nmax, sk0, false, units, target, tile);
  for (int64_t sk = sk0; sk <= cap; sk += kKT) {
    for (int alone = 0; alone < 2; ++alone) {
      if (alone && n_splits_of(static_cast<int>(mp), s.Nmax, static_cast<int>(sk), 1) >
                       kMaxMergeSplits)
        continue;
      const double c = plan_cost(mp, s.Nmax, sk, alone != 0, units, target, tile);
      if (c < best) {
        best = c;
        best_sk = sk;
        best_alone = alone != 0;
      }
    }
  }
  p->split_keys = static_cast<int>(best_sk);
  p->tree_alone = best_alone;
  p->max_splits = n_splits_of(static_cast<int>(mp), s.Nmax, p->split_keys, best_alone);
  // Workspace for partials, sized from the shortest split considered (the
  // most splits any plan of this shape can have), so that a layout with a
  // smaller cap never needs more than the size reported for the worst one.
  // None when no sequence can have more than one split.
  const int64_t pre0 = (mp + sk0 - 1) / sk0;
  const int64_t bound = pre0 <= 1 ? 1 : std::min<int64_t>(pre0 + 1, kMaxMergeSplits);
  const int64_t slots = units * bound * p->tile_rows;
  p->workspace_bytes =
      bound > 1 ? static_cast<size_t>(slots) * part_row_bytes(s) : 0;
  p->mfma = true;
  p->stream = false;
  p->grid = s.B * s.Hkv * p->row_tiles * p->max_splits;
}

// The split plan needs splits of at least two key tiles whose block ids fit
// the LDS table even with one-row blocks, and at most kMaxMergeSplits of them.
bool mfma_supported(const AttnShape& s) {
  if (s.dtype != LTD_DTYPE_BF16 || (s.d != 128 && s.d != 64)) return false;
  if (few_rows(s)) return s.max_prefix <= static_cast<int64_t>(few::kMaxKeys) * few::kMostSplits;
  if (use_stream(s)) return true;
  const int64_t cap = worst_split_key_cap(s);
  return cap >= 2 * kKT && s.max_prefix <= cap * kMaxMergeSplits;
}

int attention_grid(const AttnPlan& p) { return p.mfma ? p.grid : 0; }

// Stream plan: two partial slots per workgroup and the merge table (a 64-byte
// header and one entry per unit the call can have).
void plan_stream(const AttnShape& s, int num_cus, AttnPlan* p) {
  p->mfma = true;
  p->stream = true;
  p->grid = choose_grid(s, num_cus);
  p->workspace_bytes =
      2 * static_cast<size_t>(p->grid) * kTileRows * part_row_bytes(s) + (1 + max_units(s)) * kDescBytes;
}

void plan_mfma(const AttnShape& s, int num_cus, AttnPlan* p) {
  if (few_rows(s))
    plan_few(s, num_cus, p);
  else if (use_stream(s))
    plan_stream(s, num_cus, p);
  else
    plan_split(s, num_cus, p);
}

hipError_t launch_attn_mfma_q8(const AttnShape& s, const AttnPlan& p, const void* q,
                               const void* k_cache, const void* v_cache, const int32_t* block_table,
                               const int32_t* prefix_len, const int32_t* parents,
                               const int32_t* n_nodes, void* out, float scale, void* workspace,
                               const KvScales& scales, const int32_t* status, hipStream_t stream);

hipError_t launch_attn_mfma(const AttnShape& s, const AttnPlan& p, const void* q,
                            const void* k_cache, const void* v_cache, const int32_t* block_table,
                            const int32_t* prefix_len, const int32_t* parents,
                            const int32_t* n_nodes, void* out, float scale, void* workspace,
                            const KvScales& scales, const int32_t* status, hipStream_t stream) {
  if (s.scale_rows > 0)
    return launch_attn_mfma_q8(s, p, q, k_cache, v_cache, block_table, prefix_len, parents, n_nodes, out, scale,
                               workspace, scales, status, stream);
  const MfmaArgs a = make_args(s, q, k_cache, v_cache, block_table, prefix_len, parents, n_nodes, out, scale, workspace,
                               status);
  return launch_tiles<false>(s, p, a, workspace, stream);
}

}  // namespace ltd
