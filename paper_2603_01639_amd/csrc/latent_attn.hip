// Tree attention over a latent cache (one vector a token that all heads share), in
// bf16 on the matrix cores.
//
// For stacked query row r (node r / heads, head r % heads) and key t with cache
// row x_t = [c_t (DL dims) | k_t (64 dims)]:
//   s[r][t] = scale <q[r], x_t>,  out[r] = softmax_t(s[r]) . c_t
// over the prefix and the node's root path: the keys' first DL dims are the
// values, so one tile in LDS feeds both products,
//   S^T[key][row] = X Q^T,  O^T[dim][row] += C^T P^T   (v_mfma_f32_32x32x16_bf16).
//
// A workgroup is four waves, one a SIMD, and takes 128 rows.  A wave scores its
// own 32 rows (their queries stay in 144 registers) and accumulates all 128
// rows over its own quarter of the DL dims (256 accumulators): each weight
// then passes through LDS once, and a tile's rows are read 1.9 times a wave
// row less than if a wave kept its 32 rows over all dims, which would need every
// byte that LDS can give during the products' time.
#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "latent_plan.hpp"
#include "mfma_tiles.hpp"
#include "tree_walk.hpp"

namespace ltd {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = latent::kUnitRows;
constexpr int kKeys = latent::kKeyTile;
constexpr int kRopeDims = 64;
constexpr int kStages = 3;                     // tiles in the LDS ring
constexpr int kAncWords = LTD_MAX_NODES / 32;  // 256 bits a node
constexpr int kPlane = kKeys * 128;             // bytes of a tile's plane in LDS
constexpr float kLazyMax = 8.f;                // a running max moves when a score passes it by 2^8 (log2 units)
constexpr int kAhead = 4;                      // key fragments in flight
constexpr float kNoMax = -__FLT_MAX__;

struct LatentArgs {
  LatentAttn in;
  float* ws_o;   // [2 W][128][DL]: a piece's O / l
  float* ws_ml;  // [2 W][128][2]: its rows' max (log2 units) and sum
  int W;         // workgroups
  float scale_log2, lazy_gap;
};

// Where a position of the laid-out tiles falls.
struct Place {
  int b;
  int64_t before;  // tiles before sequence b
};

// Tiles of sequence b (0 past the batch; counts out of range are clamped).
__device__ __forceinline__ int64_t seq_tiles(const LatentAttn& a, int b) {
  if (b >= a.B) return 0;
  const int n = min(max(a.n_nodes[b], 0), a.Nmax), P = max(a.prefix_len[b], 0);
  return latent::units_of(n, a.Hq) * latent::tiles_of(P, n);
}

__device__ __forceinline__ int64_t wave_scan(int64_t v, int lane) {  // inclusive
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int64_t o = __shfl_up(v, off, kWave);
    if (lane >= off) v += o;
  }
  return v;
}

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// All sequences' tiles, and the sequence that holds tile pos(total); every wave
// computes it by itself.
template <class Pos>
__device__ __forceinline__ Place find_place(const LatentAttn& a, int lane, int64_t* total_out, Pos pos) {
  int64_t total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) total += __shfl(wave_scan(seq_tiles(a, b0 + lane), lane), kWave - 1, kWave);
  total = uniform(total);
  *total_out = total;
  const int64_t at = pos(total);
  Place p{a.B, total};
  int64_t before = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const int64_t mine = seq_tiles(a, b0 + lane);
    const int64_t incl = wave_scan(mine, lane) + before;
    const uint64_t hit = __ballot(at < incl);
    if (hit != 0) {
      const int l = __ffsll(static_cast<long long>(hit)) - 1;
      p.b = b0 + l;
      p.before = __shfl(incl - mine, l, kWave);
      break;
    }
    before = __shfl(incl, kWave - 1, kWave);
  }
  p.b = __builtin_amdgcn_readfirstlane(p.b);
  p.before = uniform(p.before);
  return p;
}

template <int DL>
struct Smem {
  unsigned char kv[kStages][(DL + kRopeDims) / 64 * kPlane];
  unsigned char p[2][kKeys / 8][kRows][16];  // weights: 8 keys of a row
  float alpha[2][kRows];                     // what a row's sums so far are multiplied by
  int moved[2][kWaves];                      // whether a wave's rows have such factors
  float row_l[kRows], row_m[kRows];
  uint32_t anc[kAncWords][LTD_MAX_NODES];    // word w of every node's ancestor set
  int jump[LTD_MAX_NODES];
  uint32_t bad[2];                           // tree keys of a tile with a NaN or an infinity
};

// A tile in LDS: planes of 64 dims, each 128 bytes of every key.  A row's 16-byte
// chunks within a plane trade places by its key, so that the eight keys of an S^T
// operand's read, and the four of a transposed read, fall on different banks.
__device__ __forceinline__ int swz(int key) { return ((key & 3) << 1) | ((key >> 4) & 1); }

// The thread's index, computed anew: what a rare branch derives from it would be
// hoisted out of the tile loop into registers that the loop does not have.
__device__ __forceinline__ int rare_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// The products by hand: O's accumulators take all 256 accumulation registers, and S's
// go to vector registers (the compiler would keep both in the former, and move O out
// and in for every tile).  A product may follow one that it adds to at once; what
// else reads a sum waits for it, 18 wait states at most after a product of 8 passes
// (mfma_settle), which nobody else sees to.
__device__ __forceinline__ void mfma_acc(f32x16& o, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_first(f32x16& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_next(f32x16& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_settle(f32x16& s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }
__device__ __forceinline__ void mfma_settle_acc(f32x16& o) { asm volatile("s_nop 15\n\ts_nop 7" : "+a"(o)); }

// A direct load of 16 bytes a lane (lane i's land at lds + 16 i) from kOff bytes past
// p.  (The instruction's offset moves its place in LDS as well, so that is taken back.)
template <int kOff>
__device__ __forceinline__ void dma16_at(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off offset:%2" ::"s"(lds - kOff), "v"(p), "n"(kOff) : "memory");
}

// o *= f in the accumulation registers.
__device__ __forceinline__ void rescale(f32x16& o, float f) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float e = o[i], tmp;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(e), "=&v"(tmp)
                 : "v"(f));
    o[i] = e;
  }
}

template <int DL, bool kPaged>
__global__ void __launch_bounds__(kThreads, 1) latent_attn_kernel(LatentArgs a) {
  constexpr int DK = DL + kRopeDims;
  constexpr int kRowBytes = DK * 2;
  constexpr int kPlanes = DK / 64;                           // also a lane's direct loads of a tile
  constexpr int kTileBytes = kPlanes * kPlane;
  constexpr int kSteps = DK / 16;                            // k-steps of S^T
  constexpr int kCols = DL / kWaves;                         // a wave's dims of O
  constexpr int kDB = kCols / 32;                            // 32-dim blocks of them
  constexpr int kGroups = kRows / 32;
  static_assert(DL % 256 == 0, "a wave takes whole groups of dims");
  __shared__ Smem<DL> sm;
  const LatentAttn& in = a.in;
  if (halted(in.status)) return;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int l32 = lane & 31, h = lane >> 5;

  // ---- this workgroup's share.  Workgroups go to the 8 XCDs in turn, so the
  // shares are dealt in 8 runs: an XCD's workgroups are neighbours and read
  // the same sequences' keys through its L2.
  int64_t total, share, pos;
  const int rank = a.W % 8 == 0 ? static_cast<int>(blockIdx.x % 8) * (a.W / 8) + static_cast<int>(blockIdx.x / 8)
                                : static_cast<int>(blockIdx.x);
  const Place place = find_place(in, lane, &total, [&](int64_t t) {
    share = latent::share_of(t, a.W);
    return rank * share;
  });
  pos = rank * share;
  const int64_t end = min(pos + share, total);
  if (pos >= end) return;
  int b = place.b;
  int64_t before = place.before;
  int slot = 2 * rank;

  // ---- lane constants
  // direct loads: lane 8 k + c of wave w fetches chunk c of key 8 w + k in every group
  const int load_key = 8 * wave + (lane >> 3);
  const int load_off = ((lane & 7) ^ swz(load_key)) * 16;
  // S^T operand: row l32 reads key sigma(l32), chunk 2 kk + h
  const int s_key = sigma(l32);
  int k_rd[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k_rd[e] = s_key * 128 + (((2 * e + h) ^ swz(s_key)) << 4);
  // C^T operand: 16-lane group g reads keys 16 ks + 8 (g / 2) + .. (two reads of
  // 4), dims 32 db + 16 (g % 2) + ..
  const int tg = lane >> 4, ts = lane & 15;
  int v_rd[2][2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int key = 16 * ks + 8 * (tg >> 1) + (ts >> 2);
      const int c = 4 * e + 2 * (tg & 1) + ((ts & 3) >> 1);
      v_rd[e][ks] = wave * (kCols / 64) * kPlane + key * 128 + ((c ^ swz(key)) << 4) + (ts & 1) * 8;
    }
  const uint32_t kv_lds = lds_addr(sm.kv[0]);

  while (pos < end) {
    // ---- the unit's piece in this share
    const int n = min(max(in.n_nodes[b], 0), in.Nmax), P = max(in.prefix_len[b], 0);
    const int64_t units = latent::units_of(n, in.Hq), tiles = latent::tiles_of(P, n);
    if (pos >= before + units * tiles) {
      before += units * tiles;
      ++b;
      continue;
    }
    const int64_t unit = (pos - before) / tiles;
    const int t0 = static_cast<int>(pos - before - unit * tiles);
    const int t1 = static_cast<int>(min(tiles, t0 + (end - pos)));
    const bool whole = t0 == 0 && t1 == tiles;
    const int64_t R = static_cast<int64_t>(n) * in.Hq;
    const int64_t r0 = unit * kRows;
    const int valid = static_cast<int>(min(static_cast<int64_t>(kRows), R - r0));
    const int last = P + n - 1;
    const bool tree = static_cast<int64_t>(t1) * kKeys > P;
    __syncthreads();  // the last piece's LDS is free

    // the lane's chunk of its key's first group in tile t (rows past the last are
    // not read: the last one is, again, and never visible)
    auto source = [&](int t) -> const unsigned char* {
      const int row = min(t * kKeys + load_key, last);
      int64_t at;
      if constexpr (kPaged) {
        const int64_t blk = in.block_table[static_cast<int64_t>(b) * in.max_blocks + row / in.kv_rows];
        at = blk * in.kv_rows + row % in.kv_rows;
      } else {
        at = static_cast<int64_t>(b) * in.kv_rows + row;
      }
      return static_cast<const unsigned char*>(in.cache) + at * kRowBytes + load_off;
    };
    auto issue = [&](int t, const unsigned char* from) {
      const uint32_t dst = kv_lds + (t % kStages) * kTileBytes + wave * 1024;
      for_each_index<kPlanes>([&](auto g) { dma16_at<g() * 128>(dst + g() * kPlane, from); });
    };

    // ---- queries: lane holds row l32 of the wave's 32, dims 16 kk + 8 h ..
    bf16x8 qf[kSteps];
    int node;
    {
      const int64_t r = r0 + min(32 * wave + l32, valid - 1);
      node = static_cast<int>(r / in.Hq);
      const int head = static_cast<int>(r % in.Hq);
      const int64_t row = static_cast<int64_t>(b) * in.Nmax + node;
      const uint16_t* ql = static_cast<const uint16_t*>(in.q_latent) + row * in.ql_row + head * in.ql_head + 8 * h;
      const uint16_t* qr = static_cast<const uint16_t*>(in.q_rope) + row * in.qr_row + head * in.qr_head + 8 * h;
#pragma unroll
      for (int kk = 0; kk < DL / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(ql + 16 * kk);
#pragma unroll
      for (int kk = 0; kk < kRopeDims / 16; ++kk) qf[DL / 16 + kk] = *reinterpret_cast<const bf16x8*>(qr + 16 * kk);
    }

    // ---- ancestor sets (256 bits a node) by pointer doubling: anc(i) |= anc(jump(i)),
    // jump(i) = jump(jump(i)); thread i has node i
    if (tree) {
      const int i = rare_thread();
      uint32_t mine[kAncWords];
#pragma unroll
      for (int w = 0; w < kAncWords; ++w) mine[w] = (i < n && (i >> 5) == w) ? 1u << (i & 31) : 0u;
      int jump = -1;
      if (i > 0 && i < n) jump = min(max(in.parents[static_cast<int64_t>(b) * in.Nmax + i], -1), i - 1);
#pragma unroll 1
      for (int round = 0; round < 9; ++round) {
#pragma unroll
        for (int w = 0; w < kAncWords; ++w) sm.anc[w][i] = mine[w];
        sm.jump[i] = jump;
        if (__syncthreads_or(jump >= 0) == 0) break;
        uint32_t other[kAncWords];
        int next = -1;
        if (jump >= 0) {
#pragma unroll
          for (int w = 0; w < kAncWords; ++w) other[w] = sm.anc[w][jump];
          next = sm.jump[jump];
        }
        __syncthreads();
        if (jump >= 0) {
#pragma unroll
          for (int w = 0; w < kAncWords; ++w) mine[w] |= other[w];
          jump = next;
        }
      }
    }
    __syncthreads();

    float m_run = kNoMax, l_run = 0.f;
    f32x16 o[kDB][kGroups];
#pragma unroll
    for (int db = 0; db < kDB; ++db)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        o[db][g] = f32x16{};
        asm volatile("" : "+a"(o[db][g]));
      }
    const float c = a.scale_log2;
    auto settle_all = [&] {
#pragma unroll
      for (int db = 0; db < kDB; ++db)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) mfma_settle_acc(o[db][g]);
    };

    // bits base .. base + 15 of a node's visible tree keys (earlier ones are the prefix)
    auto visible = [&](int base) -> uint32_t {
      const auto word = [&](int w) -> uint32_t {
        return w < 0 ? 0xFFFFFFFFu : w >= kAncWords ? 0u : sm.anc[w][node];
      };
      const int w = base >> 5;
      const uint64_t two = (static_cast<uint64_t>(word(w + 1)) << 32) | word(w);
      return static_cast<uint32_t>(two >> (base & 31)) & 0xFFFFu;
    };

    // The weights of the tile whose scores are in s, in 16 pieces (each beside one of
    // the other products): the maximum, which moves only when a score passes it by
    // 2^kLazyMax, two weights a piece, and what follows from them.
    float alpha = 1.f, top, neg, ps;
    u32x4 pk[2];
    auto weigh = [&](auto piece, const f32x16& s, int par) {
      constexpr int i = piece();
      if constexpr (i < 4) {
        if constexpr (i == 0) top = s[0];
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, s[4 * i]), s[4 * i + 1]);
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, s[4 * i + 2]), s[4 * i + 3]);
      } else if constexpr (i == 4) {
        top = max_xor32(top);
        const float m_new = top > m_run + a.lazy_gap ? top : m_run;
        neg = fminf(-m_new * c, __FLT_MAX__);
        alpha = exp2_fast((m_run - m_new) * c);  // (1 where it has not moved)
        m_run = m_new;
        ps = 0.f;
      } else if constexpr (i < 13) {
        constexpr int j = i - 5;
        const float p0 = exp2_fast(__builtin_fmaf(s[2 * j], c, neg));
        const float p1 = exp2_fast(__builtin_fmaf(s[2 * j + 1], c, neg));
        // (the sum is that of the rounded weights, the very ones that multiply the values)
        const bf16x2 w = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
        ps = __builtin_amdgcn_fdot2_f32_bf16(w, __builtin_bit_cast(bf16x2, 0x3F803F80u), ps, false);
        pk[j >> 2][j & 3] = __builtin_bit_cast(uint32_t, w);
        if constexpr (j == 3) *reinterpret_cast<u32x4*>(sm.p[par][2 * h][32 * wave + l32]) = pk[0];
      } else if constexpr (i == 13) {
        *reinterpret_cast<u32x4*>(sm.p[par][2 * h + 1][32 * wave + l32]) = pk[1];
        l_run = l_run * alpha + ps;
      }
    };
    // Tells the other waves what the rows' sums so far are multiplied by.
    auto tell = [&](int par) {
      const uint64_t any = __ballot(alpha != 1.f);
      if (any != 0) sm.alpha[par][32 * wave + l32] = alpha;
      if (lane == 0) sm.moved[par][wave] = any != 0;
    };
    // Hides the keys that the lane's node does not see.  A tree key whose latent part
    // holds a NaN or an infinity (bad) gives NaN to the nodes that see it.
    auto mask = [&](f32x16& s, int t, uint32_t bad) {
      const uint32_t vis = visible(t * kKeys - P + 16 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (!((vis >> r) & 1u)) s[r] = -INFINITY;
        else if ((bad >> (16 * h + r)) & 1u) s[r] = NAN;
      }
    };
    auto masked = [&](int t) { return (t + 1) * static_cast<int64_t>(kKeys) > P; };
    // The keys of tile t (landed) whose latent part is not finite; the whole
    // workgroup looks.
    auto find_bad = [&](int t) -> uint32_t {
      const unsigned char* kv = sm.kv[t % kStages];
      if (threadIdx.x == 0) sm.bad[t & 1] = 0;
      __syncthreads();
#pragma unroll 1
      for (int e = rare_thread(); e < kKeys * DL / 8; e += kThreads) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(kv + e * 16);
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          any |= ((x[j] & 0x7F80u) == 0x7F80u) | ((x[j] & 0x7F800000u) == 0x7F800000u);
        if (any) atomicOr(&sm.bad[t & 1], 1u << (e / 8 % kKeys));
      }
      __syncthreads();
      return __builtin_amdgcn_readfirstlane(sm.bad[t & 1]);
    };
    // 0 times a NaN would be one in the rows that do not see it.
    auto clear_bad = [&](int t, uint32_t bad) {
      unsigned char* kv = sm.kv[t % kStages];
#pragma unroll 1
      for (int e = rare_thread(); e < kKeys * DL / 8; e += kThreads)
        if ((bad >> (e / 8 % kKeys)) & 1u) *reinterpret_cast<u32x4*>(kv + e * 16) = u32x4{0, 0, 0, 0};
      __syncthreads();
    };

    auto load_k = [&](const unsigned char* kv, int kk) {
      return *reinterpret_cast<const bf16x8*>(kv + k_rd[kk & 3] + (kk >> 2) * kPlane);
    };
    auto load_v = [&](const unsigned char* kv, int db, int ks) {
      const unsigned char* at = kv + v_rd[db & 1][ks] + (db >> 1) * kPlane;
      const s16x4 lo = lds_read_tr(at), hi = lds_read_tr(at + 4 * 128);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto load_p = [&](int par, int g, int ks) {
      return *reinterpret_cast<const bf16x8*>(sm.p[par][2 * ks + h][32 * g + l32]);
    };

    // One step: the scores and weights of tile t (kS) with the product of tile
    // t - 1's weights and values (kPV).  The score products and the first half
    // of the other ones alternate, which spreads the key reads (all that LDS can
    // give while scores alone run) over both; the weights are then worked out
    // beside the second half.
    constexpr int kPV1 = kDB * kGroups;  // products of 16 keys
    auto step = [&](auto with_s, auto with_pv, int t, uint32_t bad) {
      constexpr bool kS = with_s(), kPV = with_pv();
      const unsigned char* kv = sm.kv[t % kStages];
      const unsigned char* kv_old = sm.kv[(t + kStages - 1) % kStages];
      const int par = t & 1;
      f32x16 s;
      bf16x8 kf[kAhead], vf[kDB], pf[2];
      if constexpr (kS) {
#pragma unroll
        for (int kk = 0; kk < kAhead; ++kk) kf[kk] = load_k(kv, kk);
      }
      if constexpr (kPV) {
#pragma unroll
        for (int db = 0; db < kDB; ++db) vf[db] = load_v(kv_old, db, 0);
        pf[0] = load_p(par ^ 1, 0, 0);
      }
      // product i of 16 keys ks: rows g, dims db
      auto pv = [&](auto ix, auto half) {
        constexpr int i = ix(), g = i / kDB, db = i % kDB, ks = half();
        if constexpr (db == 0 && g + 1 < kGroups) pf[(g + 1) & 1] = load_p(par ^ 1, g + 1, ks);
        mfma_acc(o[db][g], vf[db], pf[g & 1]);
      };
      using first = std::integral_constant<int, 0>;
      using second = std::integral_constant<int, 1>;
      if constexpr (kS) {
        for_each_index<kSteps>([&](auto ix) {
          constexpr int kk = ix();
          if constexpr (kk == 0) mfma_first(s, kf[0], qf[0]);
          else mfma_next(s, kf[kk % kAhead], qf[kk]);
          if constexpr (kk + kAhead < kSteps) kf[kk % kAhead] = load_k(kv, kk + kAhead);
          if constexpr (kPV) {
            // (all but the last four: those stand between the scores and their readers)
            constexpr int from = kk * (kPV1 - 4) / kSteps, to = (kk + 1) * (kPV1 - 4) / kSteps;
            if constexpr (to > from) pv(std::integral_constant<int, from>{}, first{});
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (kPV)
          for_each_index<4>([&](auto ix) { pv(std::integral_constant<int, kPV1 - 4 + ix()>{}, first{}); });
        __builtin_amdgcn_sched_barrier(0);
      } else {
        for_each_index<kPV1>([&](auto ix) { pv(ix, first{}); });
      }
      if constexpr (kPV) {
#pragma unroll
        for (int db = 0; db < kDB; ++db) vf[db] = load_v(kv_old, db, 1);
        pf[0] = load_p(par ^ 1, 0, 1);
      }
      if constexpr (kS) {
        mfma_settle(s);
        __builtin_amdgcn_sched_barrier(0);
        if (masked(t)) mask(s, t, bad);
        __builtin_amdgcn_sched_barrier(0);
      }
      for_each_index<16>([&](auto ix) {
        constexpr int i = ix();
        if constexpr (kPV) {
          constexpr int from = i * kPV1 / 16, to = (i + 1) * kPV1 / 16;
          if constexpr (to > from) pv(std::integral_constant<int, from>{}, second{});
        }
        if constexpr (kS) weigh(ix, s, par);
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    using yes = std::true_type;
    using no = std::false_type;
    issue(t0, source(t0));
    if (t0 + 1 < t1) issue(t0 + 1, source(t0 + 1));
    if (t0 + 1 < t1) wait_vmcnt<kPlanes>();
    else wait_vmcnt<0>();
    barrier_only();
    uint32_t bad = masked(t0) ? find_bad(t0) : 0;
    step(yes{}, no{}, t0, bad);
    // (nothing has been summed up yet that the first maximum could change)
    // Tile t + 1 has landed, tile t's weights are in LDS, and everyone is done with
    // tile t - 1.
    auto turn = [&] {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      barrier_only();
    };
    auto catch_up = [&](int t) {
      const int par = t & 1;
      if (bad != 0) clear_bad(t, bad);
      if (t > t0 && (sm.moved[par][0] | sm.moved[par][1] | sm.moved[par][2] | sm.moved[par][3]) != 0) {
        settle_all();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const float al = sm.moved[par][g] ? sm.alpha[par][32 * g + l32] : 1.f;
#pragma unroll
          for (int db = 0; db < kDB; ++db) rescale(o[db][g], al);
        }
        settle_all();
      }
    };
#pragma unroll 1
    for (int t = t0; t + 1 < t1; ++t) {
      // (opaque to the compiler, which would keep every address that follows from
      // these in registers of its own over the loop)
      asm volatile("" : "+v"(k_rd[0]), "+v"(k_rd[1]), "+v"(k_rd[2]), "+v"(k_rd[3]));
      asm volatile("" : "+v"(v_rd[0][0]), "+v"(v_rd[0][1]), "+v"(v_rd[1][0]), "+v"(v_rd[1][1]));
      asm volatile("" : "+v"(l32), "+v"(h));
      turn();
      if (t + 2 < t1) issue(t + 2, source(t + 2));
      catch_up(t);
      bad = masked(t + 1) ? find_bad(t + 1) : 0;
      step(yes{}, yes{}, t + 1, bad);
      tell((t + 1) & 1);
    }
    turn();
    catch_up(t1 - 1);
    step(no{}, yes{}, t1, 0);
    settle_all();

    // ---- results
    {
      const float l = l_run + xor32(l_run);
      if (h == 0) {
        sm.row_l[32 * wave + l32] = l;
        sm.row_m[32 * wave + l32] = m_run * c;
      }
    }
    __syncthreads();
    if (!whole && threadIdx.x < kRows) {
      float* ml = a.ws_ml + (static_cast<int64_t>(slot) * kRows + threadIdx.x) * 2;
      if (threadIdx.x < valid) {
        ml[0] = sm.row_m[threadIdx.x];
        ml[1] = sm.row_l[threadIdx.x];
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int row = 32 * g + l32;
      if (row >= valid) continue;
      const float l = sm.row_l[row];
      // (a piece without a visible key has weight 0 in the merge, and O = 0)
      const float inv = !whole && l == 0.f ? 0.f : 1.f / l;
      const int col = wave * kCols + 4 * h;
      if (whole) {
        uint16_t* out = static_cast<uint16_t*>(in.out) + (static_cast<int64_t>(b) * in.Nmax * in.Hq + r0 + row) * DL + col;
#pragma unroll
        for (int db = 0; db < kDB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint2 w;
            w.x = pack_bf16x2(o[db][g][4 * q] * inv, o[db][g][4 * q + 1] * inv);
            w.y = pack_bf16x2(o[db][g][4 * q + 2] * inv, o[db][g][4 * q + 3] * inv);
            *reinterpret_cast<uint2*>(out + 32 * db + 8 * q) = w;
          }
      } else {
        float* out = a.ws_o + (static_cast<int64_t>(slot) * kRows + row) * DL + col;
#pragma unroll
        for (int db = 0; db < kDB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(out + 32 * db + 8 * q) =
                f32x4{o[db][g][4 * q] * inv, o[db][g][4 * q + 1] * inv, o[db][g][4 * q + 2] * inv, o[db][g][4 * q + 3] * inv};
      }
    }
    pos += t1 - t0;
    slot = 2 * rank + 1;
  }
}

// Joins the pieces of cut units: workgroup x looks after the unit that the cut
// after share x is the first to fall into, a wave a row.
template <int DL>
__global__ void __launch_bounds__(kThreads) latent_merge_kernel(LatentArgs a) {
  constexpr int kEach = DL / kWave;  // dims a lane
  const LatentAttn& in = a.in;
  if (halted(in.status)) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t total, share;
  const int x = blockIdx.x + 1;
  const Place place = find_place(in, lane, &total, [&](int64_t t) {
    share = latent::share_of(t, a.W);
    return x * share;
  });
  const int64_t cut = x * share;
  if (cut >= total) return;
  const int b = place.b;
  const int n = min(max(in.n_nodes[b], 0), in.Nmax), P = max(in.prefix_len[b], 0);
  const int64_t tiles = latent::tiles_of(P, n);
  const int64_t unit = (cut - place.before) / tiles;
  const int64_t first = place.before + unit * tiles;
  if (cut == first || cut - share > first) return;  // (not cut here, or an earlier cut's)
  const int64_t r0 = unit * kRows;
  const int valid = static_cast<int>(min(static_cast<int64_t>(kRows), static_cast<int64_t>(n) * in.Hq - r0));
  const int64_t past = first + tiles;
  const int slot0 = 2 * (x - 1) + (cut - share != first);
  for (int row = blockIdx.y * kWaves + wave; row < valid; row += gridDim.y * kWaves) {
    float M = kNoMax * __FLT_MAX__, L = 0.f;  // (-inf)
    float acc[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
    int slot = slot0;
    for (int64_t at = cut;; at += share) {
      const float2 ml = *reinterpret_cast<const float2*>(a.ws_ml + (static_cast<int64_t>(slot) * kRows + row) * 2);
      const float* p = a.ws_o + (static_cast<int64_t>(slot) * kRows + row) * DL + lane * kEach;
      if (ml.y != 0.f) {
        const float m_new = fmaxf(M, ml.x);
        const float old = exp2_fast(M - m_new), w = exp2_fast(ml.x - m_new) * ml.y;
        L = L * old + w;
#pragma unroll
        for (int e = 0; e < kEach; ++e) acc[e] = acc[e] * old + w * p[e];
        M = m_new;
      }
      if (at >= past) break;
      slot = 2 * static_cast<int>(at / share);
    }
    const float inv = 1.f / L;
    uint16_t* out = static_cast<uint16_t*>(in.out) + (static_cast<int64_t>(b) * in.Nmax * in.Hq + r0 + row) * DL + lane * kEach;
    uint32_t w[kEach / 2];
#pragma unroll
    for (int e = 0; e < kEach / 2; ++e) w[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
#pragma unroll
    for (int e = 0; e < kEach / 2; ++e) reinterpret_cast<uint32_t*>(out)[e] = w[e];
  }
}

// The float32 path, on the vector ALUs: a workgroup per (sequence, node, four
// heads), a wave a head.  Tiles of 32 visible rows (the prefix, then the node's
// root path: no others are read) go through LDS; half a wave's lanes take
// a key each for the scores' first dims, the other half their last, and each
// lane DL / 64 dims of the output.
template <int DL>
__global__ void __launch_bounds__(kThreads) latent_vector_kernel(LatentAttn a) {
  constexpr int DK = DL + kRopeDims;
  constexpr int kPad = DK + 4;
  constexpr int kQuads = DK / 4;
  __shared__ __attribute__((aligned(16))) float x_s[kKeys][kPad];
  __shared__ __attribute__((aligned(16))) float q_s[kWaves][DK];
  __shared__ float p_s[kWaves][kKeys];
  __shared__ int path_s[LTD_MAX_NODES];
  __shared__ int path_len_s;
  if (halted(a.status)) return;
  const int i = blockIdx.x, b = blockIdx.z;
  if (i >= a.n_nodes[b]) return;
  const int t = threadIdx.x, lane = t % kWave, w = t / kWave;
  const int head = blockIdx.y * kWaves + w;
  const bool live = head < a.Hq;
  const int P = max(a.prefix_len[b], 0);
  if (t == 0) path_len_s = root_path(a.parents + static_cast<int64_t>(b) * a.Nmax, i, path_s);
  const int64_t row = static_cast<int64_t>(b) * a.Nmax + i;
  for (int e = lane; e < DK; e += kWave) {
    float v = 0.f;
    if (live)
      v = e < DL ? static_cast<const float*>(a.q_latent)[row * a.ql_row + head * a.ql_head + e]
                 : static_cast<const float*>(a.q_rope)[row * a.qr_row + head * a.qr_head + e - DL];
    q_s[w][e] = v;
  }
  __syncthreads();
  const int n_keys = P + path_len_s;
  float m = -INFINITY, l = 0.f;
  float acc[DL / kWave];
#pragma unroll
  for (int e = 0; e < DL / kWave; ++e) acc[e] = 0.f;
  const float c = a.scale;
  for (int base = 0; base < n_keys; base += kKeys) {
    const int cnt = min(kKeys, n_keys - base);
    for (int e = t; e < cnt * kQuads; e += kThreads) {
      const int k = e / kQuads, col = e % kQuads * 4;
      const int kt = base + k;
      const int r = kt < P ? kt : P + path_s[kt - P];
      const float* src = static_cast<const float*>(a.cache) + cache_row(a.block_table, b, 0, r, 1, DK, a.kv_rows, a.max_blocks);
      *reinterpret_cast<float4*>(&x_s[k][col]) = *reinterpret_cast<const float4*>(src + col);
    }
    __syncthreads();
    const int key = lane & 31, half = lane >> 5;
    float s = 0.f;
    const float* xr = &x_s[min(key, cnt - 1)][half * (DK / 2)];
    const float* qr = &q_s[w][half * (DK / 2)];
#pragma unroll 4
    for (int e = 0; e < DK / 2; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(xr + e), q = *reinterpret_cast<const float4*>(qr + e);
      s = __builtin_fmaf(x.x, q.x, s);
      s = __builtin_fmaf(x.y, q.y, s);
      s = __builtin_fmaf(x.z, q.z, s);
      s = __builtin_fmaf(x.w, q.w, s);
    }
    s = (s + xor32(s)) * c;
    if (key >= cnt) s = -INFINITY;
    const float m_new = fmaxf(m, wave_max_dpp(s));
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float p = expf(s - m_use);
    const float alpha = expf(m - m_use);
    l = l * alpha + 0.5f * wave_sum_dpp(p);  // (a key is in two lanes)
    m = m_new;
    if (half == 0) p_s[w][key] = p;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
    for (int e = 0; e < DL / kWave; ++e) acc[e] *= alpha;
    for (int k = 0; k < cnt; ++k) {
      const float pk = p_s[w][k];
#pragma unroll
      for (int e = 0; e < DL / kWave; e += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&x_s[k][lane * 4 + e * kWave]);
        acc[e] = __builtin_fmaf(pk, x.x, acc[e]);
        acc[e + 1] = __builtin_fmaf(pk, x.y, acc[e + 1]);
        acc[e + 2] = __builtin_fmaf(pk, x.z, acc[e + 2]);
        acc[e + 3] = __builtin_fmaf(pk, x.w, acc[e + 3]);
      }
    }
    __syncthreads();  // the tile is replaced
  }
  if (!live) return;
  float* out = static_cast<float*>(a.out) + (row * a.Hq + head) * DL;
#pragma unroll
  for (int e = 0; e < DL / kWave; e += 4)
    *reinterpret_cast<float4*>(out + lane * 4 + e * kWave) = float4{acc[e] / l, acc[e + 1] / l, acc[e + 2] / l, acc[e + 3] / l};
}

int grid_of(const LatentAttn& s, int cus) {
  return latent::workgroups(s.B, s.Nmax, s.Hq, s.max_prefix, cus);
}

template <int DL>
hipError_t launch_bf16(const LatentArgs& a, hipStream_t stream) {
  if (a.in.block_table)
    hipLaunchKernelGGL((latent_attn_kernel<DL, true>), dim3(a.W), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((latent_attn_kernel<DL, false>), dim3(a.W), dim3(kThreads), 0, stream, a);
  const hipError_t rc = hipGetLastError();
  if (rc != hipSuccess || a.W < 2) return rc;
  hipLaunchKernelGGL((latent_merge_kernel<DL>), dim3(a.W - 1, 16), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t latent_attn_workspace_bytes(const LatentAttn& s, int d_latent, int dtype, int cus) {
  if (dtype == LTD_DTYPE_F32 || s.B == 0) return 0;
  const int W = grid_of(s, cus);
  return W < 2 ? 0 : static_cast<size_t>(2) * W * kRows * (d_latent + 2) * sizeof(float);
}

hipError_t launch_latent_attn(const LatentAttn& s, int d_latent, int dtype, void* workspace, int cus,
                              hipStream_t stream) {
  if (dtype == LTD_DTYPE_F32) {
    const dim3 grid(s.Nmax, (s.Hq + kWaves - 1) / kWaves, s.B);
    if (d_latent == 512) hipLaunchKernelGGL((latent_vector_kernel<512>), grid, dim3(kThreads), 0, stream, s);
    else hipLaunchKernelGGL((latent_vector_kernel<256>), grid, dim3(kThreads), 0, stream, s);
    return hipGetLastError();
  }
  LatentArgs a{};
  a.in = s;
  a.W = grid_of(s, cus);
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + static_cast<int64_t>(2) * a.W * kRows * d_latent;
  a.scale_log2 = s.scale * kLog2e;
  a.lazy_gap = kLazyMax / a.scale_log2;
  return d_latent == 512 ? launch_bf16<512>(a, stream) : launch_bf16<256>(a, stream);
}

}  // namespace ltd
