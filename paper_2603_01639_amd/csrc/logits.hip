// A request's sampling rules on the target's logits at every tree node:
// penalties for tokens that occurred, biases and the grammar's mask, written
// out (ltd_tree_process_logits) or reduced to each node's argmax without being
// written (ltd_tree_accept_processed); and the table of occurrences the
// penalties read (ltd_token_counts).
//
// A workgroup takes a chunk of the vocabulary (16 tokens a thread) and a few
// nodes of one sequence, and sets up once what the nodes share: the tokens that a
// count or a bias touches, and, per node, the draft tokens of its root path that
// lie in the chunk.  Then it streams the nodes' rows in 16-byte groups, read
// only where the mask allows one of their tokens, with the next node's on the
// way.  Bound: HBM, 4 bytes read per logit and, when written, 4 more.
//
// Written rows: each thread applies the rules to its own tokens (single tokens
// stored by the threads of a list left lines half written: 16 trees of 16 to 96
// nodes, 128256 tokens, 620 us instead of 219; now 190 with the table's two
// launches, of which this kernel takes about 180, 833 MB at 4.6 TB/s; in place,
// where groups that no rule touches stay as they are, 175).  Rows are read and
// written past the caches: 181 us instead of 191 alone, 491 instead of 528 with
// acceptance by sampling reading them next; one user's 60 rows 60 us either way.
// Argmax: biased tokens go into a list in LDS that all threads share out.  Penalised
// ones stay with their owners, which bound what the rules may make of them and work
// them out where the bound reaches the largest logit so far, so that the rest is two
// maxima (a list of all touched tokens read each row's lines twice, for that and for
// itself: 16 trees of 16 to 128 nodes 167 us instead of 141; now 138.7 with the scan,
// about 135 of them here, 597 MB at 4.4 TB/s).
#include <algorithm>
#include <type_traits>

#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "rules_plan.hpp"

#pragma clang fp contract(off)  // every step of a rule is rounded, as documented

namespace ltd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
// (a row starts at any multiple of 4 bytes; the hardware takes 16-byte accesses there)
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_any __attribute__((aligned(4)));

constexpr int kVec = 4;              // 16-byte groups of a thread
constexpr int kAcceptChunk = 16384;  // the acceptance workspace's chunk
constexpr uint32_t kPrompt = 0x80000000u;

struct RuleArgs {
  const float* logits;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* n_nodes;
  const int32_t* counts;     // or nullptr
  const float* penalties;    // or nullptr
  const int32_t* bias_tokens;
  const float* bias_values;
  const int32_t* n_bias;
  const uint32_t* mask;      // or nullptr
  float* out;                // written rows, or nullptr
  uint64_t* partial;         // argmax keys [B][Nmax][chunks], or nullptr
  const int32_t* status;
  int B, Nmax, Voc, max_bias, chunks, nodes, groups;  // nodes a workgroup, node groups a sequence
};

struct Penalty {
  float rep, freq, pres;
};

// One token's logit under its count (bit 31: in the prompt) and bias.
__device__ __forceinline__ float apply_rule(float x, uint32_t count, const Penalty& p, bool biased, float bias) {
  const uint32_t c = count & ~kPrompt;
  if (count != 0) x = x > 0.f ? x / p.rep : x * p.rep;
  if (c != 0) {
    x = x - p.freq * static_cast<float>(c);
    x = x - p.pres;
  }
  return biased ? x + bias : x;
}

__device__ __forceinline__ uint64_t pack_key(float v, int idx) {
  if (v == 0.f) v = 0.f;  // -0.0 -> +0.0
  uint32_t u = __float_as_uint(v);
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<uint64_t>(u) << 32) | static_cast<uint32_t>(0xFFFFFFFFu - idx);
}

// A logit's bits where bit s of `set` is 1, those of -infinity elsewhere.
__device__ __forceinline__ uint32_t pick(uint32_t x, uint32_t set, int s) {
  const uint32_t all = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(set), s, 1));
  return (x & all) | (0xFF800000u & ~all);
}

// kArgmax: reduce to the chunk's argmax key; else write the row.  kInPlace: out
// is logits, and groups of 4 that no rule touches are neither read nor written.
template <int kThreads, bool kArgmax, bool kInPlace>
__global__ void __launch_bounds__(kThreads, 4) rules_kernel(RuleArgs a) {
  constexpr int kChunk = kThreads * 4 * kVec;
  constexpr int kNodesMax = rules::nodes_max(kArgmax);
  constexpr int kList = kArgmax ? kThreads : 1;  // biased tokens, an entry a thread
  static_assert(!kArgmax || kList >= LTD_MAX_BIAS, "room for every bias");
  static_assert(kChunk <= 65536, "offsets in a chunk fit 16 bits");
  __shared__ int32_t par_s[LTD_MAX_NODES], tok_s[LTD_MAX_NODES];
  __shared__ uint16_t path_s[kNodesMax][LTD_MAX_NODES];  // chunk offsets of the root path's draft tokens
  __shared__ int path_len_s[kNodesMax];
  __shared__ int32_t bias_tok_s[LTD_MAX_BIAS];
  __shared__ float bias_val_s[LTD_MAX_BIAS];
  __shared__ uint32_t biased_s[kChunk / 32];
  __shared__ uint16_t list_off_s[kList];
  __shared__ uint32_t list_cnt_s[kList];
  __shared__ float bias_s[kChunk];  // a biased token's bias
  __shared__ int list_n_s, twice_s;
  __shared__ unsigned long long best_s[kNodesMax];
  const int chunk = static_cast<int>(blockIdx.x) % a.chunks;
  const int group_id = static_cast<int>(blockIdx.x) / a.chunks;
  const int b = group_id / a.groups;
  const int i0 = group_id % a.groups * a.nodes;
  if (halted(a.status)) return;
  const int tid = threadIdx.x;
  const int n = min(a.n_nodes[b], a.Nmax);
  if (i0 >= n) return;
  const int i1 = min(i0 + a.nodes, n);
  const int lo = chunk * kChunk;
  const int hi = min(a.Voc, lo + kChunk);
  const int64_t seq = static_cast<int64_t>(b) * a.Nmax;
  const int words = (a.Voc + 31) / 32;
  const bool counted = a.penalties != nullptr;  // penalties act (and counts are read)
  const int32_t* counts = counted && a.counts != nullptr ? a.counts + static_cast<int64_t>(b) * a.Voc : nullptr;

  // Bits 4u + c of a 16-bit set stand for token c of the thread's group u.  The
  // tokens that exist; node i's mask words; and the tokens those allow.
  auto group = [&](int u) { return lo + (u * kThreads + tid) * 4; };
  uint32_t exist = 0;
#pragma unroll
  for (int u = 0; u < kVec; ++u) {
    const int v = group(u);
    exist |= (v + 4 <= hi ? 0xFu : v < hi ? (1u << (hi - v)) - 1u : 0u) << (4 * u);
  }
  auto load_mask = [&](int i, uint32_t(&w)[kVec]) {
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      w[u] = 0xFFFFFFFFu;
      if (a.mask != nullptr && group(u) < hi) w[u] = a.mask[(seq + i) * words + (group(u) >> 5)];
    }
  };
  auto allowed = [&](const uint32_t(&w)[kVec]) {
    uint32_t ok = 0;
#pragma unroll
    for (int u = 0; u < kVec; ++u) ok |= ((w[u] >> (group(u) & 31)) & 0xFu) << (4 * u);
    return ok & exist;
  };
  // A node on its way: its logits in the groups with a token in `want` (-infinity
  // elsewhere), what its mask allows and, for the argmax, the logit and mask word
  // of this thread's list entry.
  struct Node {
    f32x4 x[kVec];
    uint32_t ok;
    float y;
    uint32_t m;
  };
  auto load_row = [&](int i, uint32_t want, Node& nd) {
    const float* row = a.logits + (seq + i) * a.Voc;
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      const int v = group(u);
      nd.x[u] = (f32x4){-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (((want >> (4 * u)) & 0xFu) == 0) continue;
      if (v + 4 <= hi) {
        nd.x[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(row + v));
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (v + c < hi) nd.x[u][c] = row[v + c];
      }
    }
  };

  // ---- set up, with the first node's logits on the way
  Node na, nx;
  uint32_t mw[kVec];
  load_mask(i0, mw);
  na.ok = allowed(mw);
  if constexpr (!kInPlace) load_row(i0, na.ok, na);
  load_mask(min(i0 + 1, i1 - 1), mw);
  int32_t cnt[kVec][4] = {};
  if (counts != nullptr) {
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      const int v = lo + (u * kThreads + tid) * 4;
      if (v + 4 <= hi) {
        const i32x4 x = *reinterpret_cast<const i32x4_any*>(counts + v);
#pragma unroll
        for (int c = 0; c < 4; ++c) cnt[u][c] = x[c];
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (v + c < hi) cnt[u][c] = counts[v + c];
      }
    }
  }
  if (counted) {
    for (int j = tid; j < n; j += kThreads) {
      par_s[j] = a.parents[seq + j];
      tok_s[j] = a.tokens[seq + j];
    }
  }
  const int nb = a.max_bias > 0 ? min(max(a.n_bias[b], 0), a.max_bias) : 0;
  for (int j = tid; j < nb; j += kThreads) {
    bias_tok_s[j] = a.bias_tokens[static_cast<int64_t>(b) * a.max_bias + j];
    bias_val_s[j] = a.bias_values[static_cast<int64_t>(b) * a.max_bias + j];
  }
  for (int j = tid; j < kChunk / 32; j += kThreads) biased_s[j] = 0;
  if (tid == 0) list_n_s = twice_s = 0;
  if (tid < kNodesMax) {
    path_len_s[tid] = 0;
    best_s[tid] = 0;
  }
  Penalty pen{1.f, 0.f, 0.f};
  if (counted) pen = Penalty{a.penalties[3 * b], a.penalties[3 * b + 1], a.penalties[3 * b + 2]};
  __syncthreads();
  for (int j = tid; j < nb; j += kThreads) {
    const int t = bias_tok_s[j];
    if (t < lo || t >= hi) continue;
    const int o = t - lo;
    const uint32_t bit = 1u << (o & 31);
    if (atomicOr(&biased_s[o >> 5], bit) & bit) twice_s = 1;
    else bias_s[o] = bias_val_s[j];
  }
  // Root paths: one wave a node lists the draft tokens that lie in the chunk
  // (parents clamped below their child, so the walk ends whatever they hold).
  if (counted && tid % kWave == 0) {
    for (int k = tid / kWave; k < i1 - i0; k += kThreads / kWave) {
      int len = 0;
      for (int j = i0 + k; j > 0;) {
        const int t = tok_s[j];
        if (t >= lo && t < hi) path_s[k][len++] = static_cast<uint16_t>(t - lo);
        j = min(max(par_s[j], 0), j - 1);
      }
      path_len_s[k] = len;
    }
  }
  __syncthreads();
  // A token listed more than once gets the sum of its entries, in list order,
  // from the thread of its first.
  if (twice_s) {
    for (int j = tid; j < nb; j += kThreads) {
      const int t = bias_tok_s[j];
      if (t < lo || t >= hi) continue;
      float sum = bias_val_s[j];
      bool first = true;
      for (int k = 0; k < nb; ++k) {
        if (bias_tok_s[k] != t || k == j) continue;
        if (k < j) first = false;
        else sum = sum + bias_val_s[k];
      }
      if (first) bias_s[t - lo] = sum;
    }
  }
  // Of this thread's tokens (bit 4u + c): those a rule touches, and those of them
  // that only penalties do; the largest emitted count among the latter.
  uint32_t touched = 0, penal = 0;
  int cnt_max = 1;
#pragma unroll
  for (int u = 0; u < kVec; ++u) {
    const int o = (u * kThreads + tid) * 4;
    const uint32_t bits = (biased_s[o >> 5] >> (o & 31)) & 0xFu;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool biased = (bits >> c) & 1u;
      if (cnt[u][c] == 0 && !biased) continue;
      touched |= 1u << (4 * u + c);
      if constexpr (kArgmax) {
        if (biased) {
          const int at = atomicAdd(&list_n_s, 1);  // (at most LTD_MAX_BIAS)
          list_off_s[at] = static_cast<uint16_t>(o + c);
          list_cnt_s[at] = static_cast<uint32_t>(cnt[u][c]);
        } else {
          penal |= 1u << (4 * u + c);
          cnt_max = max(cnt_max, static_cast<int>(static_cast<uint32_t>(cnt[u][c]) & ~kPrompt));
        }
      }
    }
  }
  // The root path's draft tokens among this thread's (bits as touched).
  auto path_bits = [&](int i) {
    uint32_t on_path = 0;
    for (int k = 0; k < path_len_s[i - i0]; ++k) {
      const int o = path_s[i - i0][k];
      if ((o >> 2) % kThreads == tid) on_path |= 1u << ((o >> 2) / kThreads * 4 + (o & 3));
    }
    return on_path;
  };
  auto path_count = [&](int i, int o) {
    uint32_t count = 0;
    for (int k = 0; k < path_len_s[i - i0]; ++k) count += path_s[i - i0][k] == o ? 1u : 0u;
    return count;
  };

  __syncthreads();
  const bool listed = kArgmax && tid < list_n_s;  // (an entry's thread)
  const int item = listed ? list_off_s[tid] : 0;
  auto load_item = [&](int i, Node& nd) {
    nd.m = 0u;
    if (!listed) return;
    const int v = lo + item;
    nd.y = a.logits[(seq + i) * a.Voc + v];
    nd.m = a.mask != nullptr ? a.mask[(seq + i) * words + (v >> 5)] >> (v & 31) : 1u;
  };
  // The tokens whose logits node i needs, of those its mask allows: in place,
  // groups with all tokens allowed and none touched need nothing; for the argmax
  // biased tokens come by the list.
  auto wanted = [&](int i, uint32_t ok) {
    if constexpr (kArgmax) return ok & (~touched | penal);
    if constexpr (!kInPlace) return ok;
    const uint32_t act = touched | path_bits(i);
    uint32_t want = 0;
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      const uint32_t g4 = 0xFu << (4 * u);
      if ((ok & g4) != (exist & g4) || (act & g4) != 0) want |= ok & g4;
    }
    return want;
  };
  auto fetch = [&](int i, Node& nd) {
    load_row(i, wanted(i, nd.ok), nd);
    if constexpr (kArgmax) load_item(i, nd);
  };

  auto write = [&](int i, Node& nd) {
    const int len = path_len_s[i - i0];
    const uint32_t act = touched | (len > 0 ? path_bits(i) : 0u);
    float* orow = a.out + (seq + i) * a.Voc;
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      const int v = group(u);
      const uint32_t in = (exist >> (4 * u)) & 0xFu, ok = (nd.ok >> (4 * u)) & 0xFu, mine = (act >> (4 * u)) & 0xFu;
      if (in == 0 || (kInPlace && ok == in && mine == 0)) continue;
      if (mine != 0) {
        const uint32_t bits = (biased_s[(v - lo) >> 5] >> ((v - lo) & 31)) & 0xFu;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (!((mine >> c) & 1u)) continue;
          uint32_t count = static_cast<uint32_t>(cnt[u][c]);
          if (len > 0) count += path_count(i, v - lo + c);
          nd.x[u][c] = apply_rule(nd.x[u][c], count, pen, (bits >> c) & 1u, bias_s[v - lo + c]);
        }
      }
      if (ok != 0xFu) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (!((ok >> c) & 1u)) nd.x[u][c] = -INFINITY;
      }
      if (in == 0xFu) {
        __builtin_nontemporal_store(static_cast<f32x4_any>(nd.x[u]), reinterpret_cast<f32x4_any*>(orow + v));
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if ((in >> c) & 1u) orow[v + c] = nd.x[u][c];
      }
    }
  };

  auto reduce = [&](int i, Node& nd) {
    const int len = path_len_s[i - i0];
    const uint32_t on_path = len > 0 ? path_bits(i) : 0u;
    const uint32_t plain = nd.ok & ~(touched | on_path), mild = nd.ok & penal & ~on_path;
    uint64_t best = 0;  // this thread's largest key, -infinity aside
    auto take = [&](float r, int v) {
      if (r > -INFINITY) {
        const uint64_t key = pack_key(r, v);
        best = key > best ? key : best;
      }
    };
    // one of this thread's tokens (bit s), from memory
    auto take_token = [&](int s) {
      const int o = ((s >> 2) * kThreads + tid) * 4 + (s & 3);
      const int v = lo + o;
      const uint32_t count = (counts != nullptr ? static_cast<uint32_t>(counts[v]) : 0u) + path_count(i, o);
      const bool biased = (biased_s[o >> 5] >> (o & 31)) & 1u;
      take(apply_rule(a.logits[(seq + i) * a.Voc + v], count, pen, biased, bias_s[o]), v);
    };
    // the wave's largest key into the node's; its upper half
    auto publish = [&]() {
      uint32_t top;
      const uint32_t at =
          wave_argmax(static_cast<uint32_t>(best >> 32), ~static_cast<uint32_t>(best), tid % kWave, &top);
      if (tid % kWave == 0 && top != 0)
        atomicMax(&best_s[i - i0], (static_cast<unsigned long long>(top) << 32) | static_cast<uint32_t>(~at));
      return top;
    };
    float vm = -INFINITY, pm = -INFINITY;  // the largest logit of those no rule touches, and of those penalties do
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {  // (by bit masks: branches and conditions took 153 us where this takes 141)
        const uint32_t x = __float_as_uint(nd.x[u][c]);
        pm = fmaxf(pm, __uint_as_float(pick(x, mild, 4 * u + c)));
        nd.x[u][c] = __uint_as_float(pick(x, plain, 4 * u + c));
      }
      vm = fmaxf(vm, fmaxf(fmaxf(nd.x[u].x, nd.x[u].y), fmaxf(nd.x[u].z, nd.x[u].w)));
    }
    if (vm > -INFINITY) {  // the lowest index that holds the maximum
      int bi = 0;
#pragma unroll
      for (int u = kVec - 1; u >= 0; --u)
#pragma unroll
        for (int c = 3; c >= 0; --c) bi = nd.x[u][c] == vm ? group(u) + c : bi;
      best = pack_key(vm, bi);
    }
    // biased tokens, but for those of the path, which their owners take
    if ((nd.m & 1u) && !(len > 0 && path_count(i, item) != 0))
      take(apply_rule(nd.y, list_cnt_s[tid], pen, true, bias_s[item]), lo + item);
    for (uint32_t left = on_path & nd.ok; left != 0; left &= left - 1) take_token(__builtin_ctz(left));
    uint32_t bar = publish();
    // Penalised tokens matter where one may reach what the wave or the workgroup has
    // found (seldom: a token comes down, or up a little).  A rule's rounded steps
    // never fall as the logit grows or, under a negative frequency, the count, so
    // none exceeds the largest logit's result at the largest such count (at one,
    // otherwise; at none, in the prompt alone).
    if (counts != nullptr) {
      bar = max(bar, reinterpret_cast<volatile uint32_t*>(&best_s[i - i0])[1]);
      const float x = pm > 0.f ? pm / pen.rep : pm * pen.rep;
      const float up = fmaxf(x, (x - pen.freq * static_cast<float>(pen.freq < 0.f ? cnt_max : 1)) - pen.pres);
      const bool may = up > -INFINITY && static_cast<uint32_t>(pack_key(up, 0) >> 32) >= bar;
      if (__ballot(may) != 0) {
        best = 0;
        for (uint32_t left = may ? mild : 0u; left != 0; left &= left - 1) take_token(__builtin_ctz(left));
        publish();
      }
    }
  };

  // ---- the nodes, two sets of registers in turn: while one node is worked on,
  // the next one's logits and the mask of the one after it are on the way
  auto step = [&](int i, Node& cur, Node& next) {
    if (i + 1 < i1) {
      next.ok = allowed(mw);
      fetch(i + 1, next);
      if (i + 2 < i1) load_mask(i + 2, mw);
    }
    if constexpr (kArgmax) reduce(i, cur);
    else write(i, cur);
  };
  if constexpr (kInPlace) fetch(i0, na);
  if constexpr (kArgmax) load_item(i0, na);
  for (int i = i0; i < i1; i += 2) {
    step(i, na, nx);
    if (i + 1 < i1) step(i + 1, nx, na);
  }
  if constexpr (kArgmax) {
    __syncthreads();
    // (no key: every token of the chunk is at -infinity, and its first one stands for it)
    if (tid < i1 - i0)
      a.partial[(seq + i0 + tid) * a.chunks + chunk] = best_s[tid] != 0 ? best_s[tid] : pack_key(-INFINITY, lo);
  }
}

// ---- the table of occurrences

constexpr int kCountThreads = 256;
constexpr int kFreshChunk = 4096;  // tokens of a workgroup of the fresh table

// A table that starts anew: each workgroup counts the tokens of its chunk of the
// vocabulary in LDS, from all of the sequence's, and writes the chunk once (one
// launch instead of a clearing one and an adding one; 16 sequences of 4096
// tokens and 128256 entries, one node each: 19.5 us a pass instead of 16.1).
__global__ void __launch_bounds__(kCountThreads) counts_fresh_kernel(
    const int32_t* __restrict__ tokens, const int32_t* __restrict__ n_tokens, int T, int Voc, int prompt,
    int32_t* __restrict__ counts) {
  __shared__ uint32_t count_s[kFreshChunk];
  const int b = blockIdx.y;
  const int lo = blockIdx.x * kFreshChunk;
  const int size = min(kFreshChunk, Voc - lo);
  for (int j = threadIdx.x; j < kFreshChunk; j += kCountThreads) count_s[j] = 0;
  __syncthreads();
  const int n = T > 0 ? min(n_tokens[b], T) : 0;
  const int32_t* row = tokens + static_cast<int64_t>(b) * T;
  constexpr int kAhead = 8;  // loads in flight a thread
  for (int j0 = threadIdx.x; j0 < n; j0 += kAhead * kCountThreads) {
    int t[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * kCountThreads;
      t[u] = j < n ? row[j] : -1;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t[u] < lo || t[u] >= lo + size) continue;
      if (prompt) count_s[t[u] - lo] = kPrompt;  // (the same word from every thread)
      else atomicAdd(&count_s[t[u] - lo], 1u);
    }
  }
  __syncthreads();
  int32_t* out = counts + static_cast<int64_t>(b) * Voc + lo;
  for (int j = threadIdx.x; j < size; j += kCountThreads) out[j] = static_cast<int32_t>(count_s[j]);
}

// Integer atomics: the result does not depend on their order.
__global__ void __launch_bounds__(kCountThreads) counts_add_kernel(
    const int32_t* __restrict__ tokens, const int32_t* __restrict__ n_tokens, int T, int Voc, int prompt,
    int32_t* __restrict__ counts) {
  const int b = blockIdx.y;
  const int j = blockIdx.x * kCountThreads + threadIdx.x;
  if (j >= min(n_tokens[b], T)) return;
  const int t = tokens[static_cast<int64_t>(b) * T + j];
  if (t < 0 || t >= Voc) return;
  int32_t* c = counts + static_cast<int64_t>(b) * Voc + t;
  if (prompt) atomicOr(c, static_cast<int>(kPrompt));
  else atomicAdd(c, 1);
}

// Checks of the rules' data: trees, penalties and bias lengths; the code of the
// lowest failing sequence.
__global__ void __launch_bounds__(kCountThreads) validate_rules_kernel(
    const int32_t* parents, const int32_t* n_nodes, const float* penalties, const int32_t* n_bias, int B, int Nmax,
    int max_bias, int32_t* status) {
  __shared__ int best;
  if (threadIdx.x == 0) best = 0x7FFFFFFF;
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += kCountThreads) {
    int code = 0;
    const int n = n_nodes[b];
    const int32_t* par = parents + static_cast<int64_t>(b) * Nmax;
    if (n < 1 || n > Nmax) {
      code = LTD_STATUS_BAD_NNODES;
    } else {
      if (par[0] != -1) code = LTD_STATUS_BAD_PARENT;
      for (int i = 1; i < n && code == 0; ++i)
        if (par[i] < 0 || par[i] >= i) code = LTD_STATUS_BAD_PARENT;
    }
    if (code == 0 && penalties != nullptr) {
      const float* p = penalties + 3 * static_cast<int64_t>(b);
      if (!(p[0] > 0.f) || !isfinite(p[0]) || !isfinite(p[1]) || !isfinite(p[2])) code = LTD_STATUS_BAD_RULE;
    }
    if (code == 0 && max_bias > 0 && (n_bias[b] < 0 || n_bias[b] > max_bias)) code = LTD_STATUS_BAD_RULE;
    if (code != 0) {
      atomicMin(&best, (b << 8) | code);
      break;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) *status = best == 0x7FFFFFFF ? 0 : (best & 0xFF);
}

}  // namespace

hipError_t launch_validate_rules(const int32_t* parents, const int32_t* n_nodes, const float* penalties,
                                 const int32_t* n_bias, int B, int Nmax, int max_bias, int32_t* status,
                                 hipStream_t stream) {
  hipLaunchKernelGGL(validate_rules_kernel, dim3(1), dim3(kCountThreads), 0, stream, parents, n_nodes, penalties,
                     n_bias, B, Nmax, max_bias, status);
  return hipGetLastError();
}

hipError_t launch_token_counts(const int32_t* tokens, const int32_t* n_tokens, int B, int T, int Voc, bool prompt,
                               bool reset, int32_t* counts, hipStream_t stream) {
  if (reset) {
    hipLaunchKernelGGL(counts_fresh_kernel, dim3((Voc + kFreshChunk - 1) / kFreshChunk, B), dim3(kCountThreads), 0,
                       stream, tokens, n_tokens, T, Voc, prompt ? 1 : 0, counts);
    return hipGetLastError();
  }
  if (T > 0)
    hipLaunchKernelGGL(counts_add_kernel, dim3((T + kCountThreads - 1) / kCountThreads, B), dim3(kCountThreads), 0,
                       stream, tokens, n_tokens, T, Voc, prompt ? 1 : 0, counts);
  return hipGetLastError();
}

hipError_t launch_rules(const LogitRules& r, int B, int Nmax, int Voc, float* out, void* partial, int cus,
                        const int32_t* status, hipStream_t stream) {
  RuleArgs a{};
  a.logits = r.logits;
  a.tokens = r.tokens;
  a.parents = r.parents;
  a.n_nodes = r.n_nodes;
  a.counts = r.counts;
  a.penalties = r.penalties;
  a.bias_tokens = r.bias_tokens;
  a.bias_values = r.bias_values;
  a.n_bias = r.n_bias;
  a.mask = r.mask;
  a.out = out;
  a.partial = static_cast<uint64_t*>(partial);
  a.status = status;
  a.Nmax = Nmax;
  a.Voc = Voc;
  a.max_bias = r.max_bias;
  a.B = B;
  const auto launch = [&](auto threads, auto argmax, auto in_place) {
    constexpr int kChunk = threads() * 4 * kVec;
    a.chunks = (Voc + kChunk - 1) / kChunk;
    a.nodes = rules::nodes(B, Nmax, a.chunks, argmax(), threads(), cus);
    a.groups = (Nmax + a.nodes - 1) / a.nodes;
    hipLaunchKernelGGL((rules_kernel<threads(), argmax(), in_place()>),
                       dim3(static_cast<unsigned>(a.chunks) * a.groups * B),
                       dim3(threads()), 0, stream, a);
  };
  using Large = std::integral_constant<int, 1024>;
  using Small = std::integral_constant<int, 256>;
  static_assert(Large::value * 4 * kVec == kAcceptChunk, "the acceptance workspace holds one key per chunk");
  if (partial) launch(Large{}, std::true_type{}, std::false_type{});
  else if (out == r.logits) launch(Small{}, std::false_type{}, std::true_type{});
  else launch(Small{}, std::false_type{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace ltd
