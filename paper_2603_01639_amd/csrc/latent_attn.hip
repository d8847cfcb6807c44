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
// rows over its own quarter of the DL dims (256 accumulators).  With 512 dims a wave then
// reads 53 KB of LDS a tile: its keys, a quarter of its values, 128 rows' weights.  With its
// 32 rows over all dims it would read 70 KB, and four waves at 128 bytes a cycle as long as
// the products take, 2176 cycles.
#include <algorithm>

#include "latent_attn.hpp"
#include "tree_walk.hpp"

namespace ltd {
namespace {

constexpr int kKeys = latent::kKeyTile;
constexpr int kStages = 3;           // tiles in the LDS ring
constexpr int kAhead = 6;            // key fragments in flight
constexpr int kPlane = kKeys * 128;  // bytes of a tile's plane in LDS
constexpr int kQPlane = 32 * 128;    // and of a wave's queries'
constexpr latent::Cut kCut = latent::kMany;

template <int DL>
struct Smem {
  alignas(16) unsigned char kv[kStages][(DL + kRopeDims) / 64 * kPlane];
  u32x4 p[2][kKeys / 8][kRows];              // weights: 8 keys of a row
  float alpha[2][kRows];                     // what a row's sums so far are multiplied by
  i32x4 moved[2];                            // whether a wave's rows have such factors
  float row_f[kRows];                        // 1 / sum
  uint32_t anc[kAncWords][LTD_MAX_NODES];    // word w of every node's ancestor set
  int jump[LTD_MAX_NODES];
  uint32_t bad[2];                           // tree keys of a tile with a NaN or an infinity
};

// The key in row i of an S^T operand.  Accumulator r of lane half h, row 8 (r / 4) +
// 4 h + r % 4 of the product, then holds key acc_key(r) + 8 h: the registers of
// (r / 4) % 2 = q are the eight keys of chunk 2 q + h, in order.
__device__ __forceinline__ int operand_key(int i) {
  return (i & 3) | ((i >> 4) & 1) << 2 | ((i >> 2) & 1) << 3 | ((i >> 3) & 1) << 4;
}
constexpr int acc_key(int r) { return (r & 3) | (r >> 3) << 2 | ((r >> 2) & 1) << 4; }

// A tile in LDS: planes of 64 dims, each 128 bytes of every key.  A row's 16-byte
// chunks within a plane trade places by its key, so that neither 16 lanes of an S^T
// operand's read (keys that differ in bits 0, 1, 3 and 4; even and odd ones lie in
// different halves of the banks) nor 32 lanes of a transposed read (64 bytes of four
// neighbouring keys) meet on a bank.
__device__ __forceinline__ int swz(int key) {
  return ((key >> 1) & 1) << 2 | ((key >> 3) & 1) << 1 | ((key >> 4) & 1);
}

__device__ __forceinline__ int rare_thread() { return rare(static_cast<int>(threadIdx.x)); }

// The products by hand: O's accumulators take all 256 accumulation registers, and S's
// go to vector registers (the compiler would keep both in the former, and move O out
// and in for every tile).  A product may follow one that it adds to at once; what
// else touches a sum waits for it, 12 wait states behind a product of 8 passes.  The
// compiler does not see to that here: mfma_settle does, and a test reads the distances
// from the listing.
__device__ __forceinline__ void mfma_acc(f32x16& o, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_first(f32x16& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}
// o = 0 (a product takes 8 bytes of code, 16 moves 128).
__device__ __forceinline__ void mfma_zero(f32x16& o, bf16x8 zero) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %1, 0" : "=a"(o) : "v"(zero));
}
__device__ __forceinline__ void mfma_next(f32x16& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_settle(f32x16& s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }
// The same after three further products: the last of them went out when the pipe had
// been through the first two, 64 cycles after s was done.
__device__ __forceinline__ void mfma_settled(f32x16& s) { asm volatile("s_nop 3" : "+v"(s)); }
__device__ __forceinline__ void settled(f32x16& o) { asm volatile("" : "+a"(o)); }

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
  const Seq first_seqs = seq_of(in, lane);
  const Place place = find_place(in, kCut, lane, first_seqs, &total, [&](int64_t t) {
    share = latent::share_of(t, a.W, kCut);
    return rank * share;
  });
  share = uniform(share);
  pos = rank * share;
  const int64_t end = min(pos + share, total);
  if (threadIdx.x == 0) a.ws_cut[rank].valid = 0;
  if (pos >= end) return;
  int b = __builtin_amdgcn_readfirstlane(place.b);
  int64_t before = uniform(place.before);
  int tree_of = -1;  // the sequence whose ancestor sets are in LDS

  // ---- lane constants
  // direct loads: lane 8 k + c of wave w fetches chunk c of key 8 w + k in every group
  int load_key = 8 * wave + (lane >> 3);
  // S^T operand: row l32, chunk 2 kk + h, which step kk moves by an exclusive or
  int k_rd = operand_key(l32) * 128 + ((h ^ swz(operand_key(l32))) << 4);
  // C^T operand: 16-lane group g reads keys 16 ks + 8 (g / 2) + .. (two reads of
  // 4), dims 32 db + 16 (g % 2) + ..; the same way from ks = 0, db = 0
  const int v_key = 8 * (lane >> 5) + ((lane >> 2) & 3);
  int v_rd = wave * (kCols / 64) * kPlane + v_key * 128 +
             (((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ swz(v_key)) << 4) + (lane & 1) * 8;
  const uint32_t kv_lds = lds_addr(sm.kv[0]);
  while (pos < end) {
    // ---- the unit's piece in this share
    const Seq seq = b < kWave ? first_seqs : seq_of(in, b);
    const int n = __builtin_amdgcn_readlane(seq.n, b % kWave), P = __builtin_amdgcn_readlane(seq.P, b % kWave);
    const int64_t length = kCut.cost + latent::tiles_of(P, n);
    const int64_t all = latent::units_of(n, in.Hq, kCut) * length;
    if (pos >= before + all) {
      before += all;
      ++b;
      continue;
    }
    const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>(latent::quotient(pos - before, length)));
    const int64_t start = before + unit * length;
    const int64_t stop = uniform(min(start + length, end));
    const int t0 = __builtin_amdgcn_readfirstlane(static_cast<int>(latent::tile_at(pos - start, kCut)));
    const int t1 = __builtin_amdgcn_readfirstlane(static_cast<int>(latent::tile_at(stop - start, kCut)));
    if (t1 == t0) {  // (a share that ends within a unit's own cost)
      pos = stop;
      continue;
    }
    const bool whole = t0 == 0 && stop == start + length;
    const int slot = 2 * rank + (t0 == 0);  // (one piece that goes on, one that begins)
    const int r0 = unit * kRows;
    const int valid = min(kRows, n * in.Hq - r0);
    const int last = P + n - 1;
    const bool tree = static_cast<int64_t>(t1) * kKeys > P && tree_of != b;
    __syncthreads();  // the last piece's LDS is free

    // Direct loads.  at(t): where the lane's chunk of its key's first plane lies for
    // tile t (rows past the last are not read: the last one is, again, and never
    // visible).  A paged cache's block ids are read a tile ahead.
    int32_t block = 0;
    auto look_up = [&](int t, int32_t& block) {
      if constexpr (kPaged)
        block = in.block_table[static_cast<int64_t>(b) * in.max_blocks + block_of(a, min(t * kKeys + load_key, last))];
    };
    auto source = [&](uint32_t place) {
      return static_cast<const unsigned char*>(in.cache) +
             (static_cast<uint64_t>(place) * kRowBytes + ((lane & 7) ^ swz(load_key)) * 16);
    };
    auto at = [&](int t, int32_t block) { return source(row_place<kPaged>(a, b, min(t * kKeys + load_key, last), block)); };
    auto issue_plane = [&](int t, const unsigned char* from, auto plane) {
      dma16_at<plane() * 128>(kv_lds + ((t - t0) % kStages) * kTileBytes + wave * 1024 + plane() * kPlane, from);
    };
    auto issue = [&](int t, int32_t block) {
      const unsigned char* from = at(t, block);
      for_each_index<kPlanes>([&](auto g) { issue_plane(t, from, g); });
    };
    int32_t block0 = 0, block1 = 0;
    look_up(t0, block0);
    look_up(t0 + 1, block1);
    look_up(t0 + 2, block);
    // ---- queries: lane holds row l32 of the wave's 32, dims 16 kk + 8 h ..  They come
    // through LDS, in two runs of planes of 64 dims through the wave's part of what the
    // first tile leaves free: loaded from where they lie, 16 bytes of 32 rows an
    // instruction, they took 7100 cycles, and the tile behind them waited.
    bf16x8 qf[kSteps];
    int node;
    constexpr int kRun = (2 * kTileBytes + static_cast<int>(sizeof(sm.p))) / (kWaves * kQPlane);
    static_assert(2 * kRun >= kPlanes && offsetof(Smem<DL>, p) == kStages * kTileBytes, "the queries come in two runs");
    constexpr int kFirst = kRun < kPlanes ? kRun : kPlanes;
    const unsigned char* q_from[2][4];  // row 8 i + lane / 8: its chunk of the first plane, and of the rotated part
    {
      const uint32_t r = r0 + min(32 * wave + l32, valid - 1), heads = rare(in.Hq);
      node = static_cast<int>(r / heads);
      const int head = static_cast<int>(r % heads);
      const int64_t row = static_cast<int64_t>(b) * in.Nmax + node;
      const int64_t ql = 2 * (row * in.ql_row + head * in.ql_head), qr = 2 * (row * in.qr_row + head * in.qr_head);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int of = 8 * i + (lane >> 3), chunk = ((lane & 7) ^ (of >> 1 & 7)) * 16;
        q_from[0][i] = static_cast<const unsigned char*>(in.q_latent) + (__shfl(ql, of, kWave) + chunk);
        q_from[1][i] = static_cast<const unsigned char*>(in.q_rope) + (__shfl(qr, of, kWave) + chunk);
      }
    }
    unsigned char* q_lds = sm.kv[1] + wave * (kFirst * kQPlane);
    auto load_queries = [&](auto from, auto to) {
      for_each_index<to() - from()>([&](auto ix) {
        constexpr int g = from() + ix();
        for_each_index<4>([&](auto i) {
          const uint32_t dst = lds_addr(q_lds) + ix() * kQPlane + i() * 1024;
          if constexpr (g < DL / 64) dma16_at<g * 128>(dst, q_from[0][i()]);
          else dma16_at<0>(dst, q_from[1][i()]);
        });
      });
    };
    auto take_queries = [&](auto from, auto to) {
      wait_vmcnt<0>();
      for_each_index<4 * (to() - from())>([&](auto ix) {
        qf[4 * from() + ix()] = *reinterpret_cast<const bf16x8*>(
            q_lds + (ix() >> 2) * kQPlane + l32 * 128 + (((2 * (ix() & 3) + h) ^ (l32 >> 1 & 7)) << 4));
      });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    using First = std::integral_constant<int, kFirst>;
    using All = std::integral_constant<int, kPlanes>;
    issue(t0, block0);
    load_queries(std::integral_constant<int, 0>{}, First{});

    // ---- ancestor sets (256 bits a node) by pointer doubling: anc(i) |= anc(jump(i)),
    // jump(i) = jump(jump(i)); thread i has node i
    if (tree) {
      tree_of = b;
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
    take_queries(std::integral_constant<int, 0>{}, First{});
    if constexpr (kFirst < kPlanes) {
      load_queries(First{}, All{});
      take_queries(First{}, All{});
    }
    __syncthreads();
    if (t0 + 1 < t1) issue(t0 + 1, block1);

    float m_run = rare(kNoMax), l_run = 0.f;
    f32x16 o[kDB][kGroups];
    bf16x8 zero = bf16x8{};
    asm volatile("s_nop 1" : "+v"(zero));
#pragma unroll
    for (int db = 0; db < kDB; ++db)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        mfma_zero(o[db][g], zero);
      }
    const float c = a.scale_log2;
    auto settle_all = [&] {
      asm volatile("s_nop 15\n\ts_nop 7");
#pragma unroll
      for (int db = 0; db < kDB; ++db)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) settled(o[db][g]);
    };

    // bits base .. base + 31 of a node's visible tree keys (earlier ones are the prefix)
    auto visible = [&](int base) -> uint32_t {
      const auto word = [&](int w) -> uint32_t {
        uint32_t x = w < 0 ? 0xFFFFFFFFu : 0u;
        if (static_cast<uint32_t>(w) < kAncWords) x = sm.anc[w][node];
        return x;
      };
      const int w = base >> 5;
      return __builtin_amdgcn_alignbit(word(w + 1), word(w), base & 31);
    };

    // The weights of the tile whose scores are in s, in pieces of a few instructions that
    // fit beside one of the other products: the maximum, which moves only when a
    // score passes it by 2^kLazyMax, a weight a piece, and what follows from them.
    // (With two products and two weights a piece the vector operations of a piece
    // outlasted the second product: 1250 cycles a tile where the products take 670.)
    //
    // They are rounded to bfloat16, as one factor of the products: outputs are off by 0.0020 of
    // them where their own rounding gives 0.0017.  With what the rounding left as a second
    // part, 32 more products a tile beside 68, the difference was gone and 8 sequences of
    // 128 heads took 731 us instead of 556, 60 nodes of 16 heads over 16384 keys 68 instead of 58,
    // one token of 16 sequences of 128 heads 58 instead of 53.
    float alpha = 1.f, top, neg, ps, p0;
    uint64_t moves;
    u32x4 pk[2];
    constexpr int kPieces = 23;
    auto weigh = [&](auto piece, const f32x16& s, int par) {
      constexpr int i = piece();
      if constexpr (i < 4) {
        if constexpr (i == 0) top = s[0];
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, s[4 * i]), s[4 * i + 1]);
        top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, s[4 * i + 2]), s[4 * i + 3]);
      } else if constexpr (i == 4) {
        top = max_xor32(top);
        top = top > m_run + a.lazy_gap ? top : m_run;
      } else if constexpr (i == 5) {
        neg = fminf(-top * c, __FLT_MAX__);
        alpha = exp2_fast((m_run - top) * c);  // (1 where it has not moved)
        m_run = top;
        ps = 0.f;
      } else if constexpr (i < 22) {
        constexpr int j = (i - 6) / 2, q = j >> 2, r = 4 * q + 8 * ((j >> 1) & 1) + 2 * (j & 1);
        if constexpr ((i - 6) % 2 == 0) {
          p0 = exp2_fast(__builtin_fmaf(s[r], c, neg));
          // (tells the other waves what the rows' sums so far are multiplied by)
          if constexpr (j == 1) moves = __ballot(alpha != 1.f);
          if constexpr (j == 2) {
            if (moves != 0) sm.alpha[par][32 * wave + l32] = alpha;
          }
          if constexpr (j == 3) reinterpret_cast<int*>(&sm.moved[par])[wave] = moves != 0;  // (all lanes the same)
          if constexpr (j == 4) sm.p[par][h][32 * wave + l32] = pk[0];
        } else {
          const float p1 = exp2_fast(__builtin_fmaf(s[r + 1], c, neg));
          // (the sum is that of the rounded weights, the very ones that multiply the values)
          const bf16x2 w = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
          ps = __builtin_amdgcn_fdot2_f32_bf16(w, __builtin_bit_cast(bf16x2, 0x3F803F80u), ps, false);
          asm volatile("" : "+v"(ps));  // (here, not all of them after the last product)
          pk[q][j & 3] = __builtin_bit_cast(uint32_t, w);
        }
      } else {
        sm.p[par][2 + h][32 * wave + l32] = pk[1];
        l_run = l_run * alpha + ps;
      }
    };
    // Hides the keys that the lane's node does not see.  A tree key whose latent part
    // holds a NaN or an infinity (bad) gives NaN to the nodes that see it.
    auto mask = [&](f32x16& s, int t, uint32_t bad) {
      const uint32_t vis = visible(t * kKeys - P) >> (8 * h);
      const uint32_t nan = bad >> (8 * h);
      if (bad != 0) {
        const float none = rare(NAN);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (nan >> acc_key(r)) & 1u ? none : s[r];
      }
      const float hidden = rare(-INFINITY);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (vis >> acc_key(r)) & 1u ? s[r] : hidden;
    };
    auto masked = [&](int t) { return (t + 1) * static_cast<int64_t>(kKeys) > P; };
    // The keys of tile t (landed) whose latent part is not finite; the whole
    // workgroup looks.
    auto find_bad = [&](int t) -> uint32_t {
      const unsigned char* kv = sm.kv[(t - t0) % kStages];
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
      unsigned char* kv = sm.kv[(t - t0) % kStages];
#pragma unroll 1
      for (int e = rare_thread(); e < kKeys * DL / 8; e += kThreads)
        if ((bad >> (e / 8 % kKeys)) & 1u) {
          const uint32_t zero = rare(0u);
          *reinterpret_cast<u32x4*>(kv + e * 16) = u32x4{zero, zero, zero, zero};
        }
      __syncthreads();
    };

    auto load_k = [&](const unsigned char* kv, int kk) {
      return *reinterpret_cast<const bf16x8*>(kv + (k_rd ^ ((kk & 3) << 5)) + (kk >> 2) * kPlane);
    };
    auto load_v = [&](const unsigned char* kv, int db, int ks) {
      const unsigned char* at = kv + (v_rd ^ ((db & 1) << 6 | ks << 4)) + ks * 16 * 128 + (db >> 1) * kPlane;
      const s16x4 lo = lds_read_tr(at), hi = lds_read_tr(at + 4 * 128);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto load_p = [&](int par, int g, int ks) {
      return __builtin_bit_cast(bf16x8, sm.p[par][2 * ks + h][32 * g + l32]);
    };

    // The products of a tile's weights and values, in the order q = 4 ks + g of 16 keys
    // (ks) and 32 rows (g): weights are read three q ahead, values a ks ahead.
    bf16x8 va[kDB], vb[kDB], pf[3];
    auto product = [&](auto ix, const bf16x8(&v)[kDB], int par) {  // of index q * kDB + db
      constexpr int q = ix() / kDB, db = ix() % kDB;
      mfma_acc(o[db][q & 3], v[db], pf[q % 3]);
      if constexpr (db == kDB - 1 && q + 3 < 2 * kGroups) pf[q % 3] = load_p(par, (q + 3) & 3, (q + 3) >> 2);
    };
    constexpr int kHalf = 2 * kDB;  // products of two q
    // The last quarter of a tile's products waits in registers for the next step: it
    // fills the time that the step's first reads take.
    auto last_products = [&](auto beside) {
      for_each_index<kHalf>([&](auto i) {
        product(std::integral_constant<int, 3 * kHalf + i()>{}, vb, 0);
        beside(i);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto load_values = [&](bf16x8(&v)[kDB], const unsigned char* kv, int ks) {
#pragma unroll
      for (int db = 0; db < kDB; ++db) v[db] = load_v(kv, db, ks);
    };
    // Scores of tile t from its first fragments in kf; beside(kk) runs beside product kk.
    bf16x8 kf[kAhead];
    auto first_keys = [&](const unsigned char* kv) {
#pragma unroll
      for (int kk = 0; kk < kAhead; ++kk) kf[kk] = load_k(kv, kk);
    };
    auto scores = [&](f32x16& s, const unsigned char* kv, auto beside) {
      for_each_index<kSteps>([&](auto ix) {
        constexpr int kk = ix();
        if constexpr (kk == 0) mfma_first(s, kf[0], qf[0]);
        else mfma_next(s, kf[kk % kAhead], qf[kk]);
        if constexpr (kk + kAhead < kSteps) kf[kk % kAhead] = load_k(kv, kk + kAhead);
        beside(ix);
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    // ---- the tile loop, software-pipelined by one tile: step t works out the scores and
    // weights of tile t + 1 and multiplies tile t's weights and values.  A quarter of
    // those products runs in front of the scores', and three beside the weights'
    // vector operations.
    uint32_t bad = masked(t0) ? find_bad(t0) : 0;
    {
      f32x16 s;
      const unsigned char* kv = sm.kv[0];
      first_keys(kv);
      scores(s, kv, [](auto) {});
      mfma_settle(s);
      if (masked(t0)) mask(s, t0, bad);
      for_each_index<kPieces>([&](auto i) { weigh(i, s, t0 & 1); });
      // (nothing has been summed up yet that the first maximum could change)
    }
#pragma unroll
    for (int db = 0; db < kDB; ++db) vb[db] = bf16x8{};
    pf[0] = pf[1] = pf[2] = bf16x8{};
    // Tile t + 1 has landed, tile t's weights are in LDS, and everyone is done with
    // tile t - 1.
    auto turn = [&] {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      barrier_only();
    };
    auto catch_up = [&](int t, const i32x4& moved) {
      const int par = t & 1;
      if (bad != 0) clear_bad(t, bad);
      if (t > t0 && __builtin_amdgcn_readfirstlane(moved[0] | moved[1] | moved[2] | moved[3]) != 0) {
        settle_all();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const float al = moved[g] ? sm.alpha[par][32 * g + l32] : 1.f;
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
      asm volatile("" : "+v"(k_rd), "+v"(v_rd), "+v"(l32), "+v"(h), "+v"(load_key));
      const unsigned char* kv = sm.kv[(t + 1 - t0) % kStages];
      const unsigned char* kv_old = sm.kv[(t - t0) % kStages];
      const int par = t & 1;
      turn();
      first_keys(kv);
      const i32x4 moved = sm.moved[par];
      __builtin_amdgcn_sched_barrier(0);
      // (tile t + 2's addresses, a few instructions beside each product)
      int row;
      uint32_t place;
      const unsigned char* from;
      last_products([&](auto i) {
        if constexpr (i() == 0) row = min((t + 2) * kKeys + load_key, last);
        if constexpr (i() == 1) place = row_place<kPaged>(a, b, row, block);
        if constexpr (i() == 2) from = source(place);
        if constexpr (i() == 3) look_up(t + 3, block);
      });
      catch_up(t, moved);
      bad = masked(t + 1) ? find_bad(t + 1) : 0;
      f32x16 s;
      scores(s, kv, [&](auto ix) {
        constexpr int kk = ix();
        // (tile t + 2's direct loads go out one by one; one tile past the piece's last
        // is loaded and not used)
        if constexpr (kk % 3 == 2 && kk / 3 < kPlanes) issue_plane(t + 2, from, std::integral_constant<int, kk / 3>{});
        // (the first values and weights, ahead of their products)
        constexpr int late = kk - (kSteps - kDB - 3);
        if constexpr (late >= 0 && late < kDB) va[late] = load_v(kv_old, late, 0);
        if constexpr (late >= kDB) pf[late - kDB] = load_p(par, late - kDB, 0);
      });
      // (what stands between the scores and their readers)
      constexpr int kApart = 3;
      for_each_index<kApart>([&](auto i) { product(i, va, par); });
      load_values(vb, kv_old, 1);
      __builtin_amdgcn_sched_barrier(0);
      mfma_settled(s);
      __builtin_amdgcn_sched_barrier(0);
      if (masked(t + 1)) mask(s, t + 1, bad);
      __builtin_amdgcn_sched_barrier(0);
      for_each_index<kPieces>([&](auto ix) {
        constexpr int n = 3 * kHalf - kApart, a0 = kApart + ix() * n / kPieces, a1 = kApart + (ix() + 1) * n / kPieces;
        for_each_index<a1 - a0>([&](auto i) {
          constexpr int at = a0 + i();
          if constexpr (at < 2 * kHalf) product(std::integral_constant<int, at>{}, va, par);
          else product(std::integral_constant<int, at>{}, vb, par);
        });
        weigh(ix, s, par ^ 1);
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    {
      const float l = l_run + xor32(l_run);
      // (a piece without a visible key has weight 0 in the merge, and O = 0)
      if (h == 0) sm.row_f[32 * wave + l32] = !whole && l == 0.f ? 0.f : 1.f / l;
      if (!whole && h == 0 && 32 * wave + l32 < valid) {
        PieceRow& row = a.ws_row[static_cast<int64_t>(slot) * kRows + 32 * wave + l32];
        row.m = m_run * c;
        row.l = l;
      }
      if (!whole && t0 == 0 && threadIdx.x == 0)
        a.ws_cut[rank] = CutUnit{b, r0, valid, static_cast<int>(latent::quotient(start + length - 1, share))};
    }
    turn();
    last_products([](auto) {});
    catch_up(t1 - 1, sm.moved[(t1 - 1) & 1]);
    {
      const unsigned char* kv = sm.kv[(t1 - 1 - t0) % kStages];
      const int par = (t1 - 1) & 1;
      load_values(va, kv, 0);
      load_values(vb, kv, 1);
      for_each_index<3>([&](auto g) { pf[g()] = load_p(par, g(), 0); });
      for_each_index<2 * kHalf>([&](auto i) { product(i, va, par); });
      for_each_index<2 * kHalf>([&](auto i) { product(std::integral_constant<int, 2 * kHalf + i()>{}, vb, par); });
    }
    settle_all();

    // ---- results, 32 rows at a time: O / l of a whole unit to `out`, as a piece to the
    // workspace.  (256 workgroups' pieces are 67 MB, which bound this part.)  The sums
    // pass through LDS, in the stages that no wave reads any more (two waves in each), so
    // that a row's dims of a wave go out in one run and the code is that of one row.
    constexpr int kPitch = kCols * 4 + 16;
    unsigned char* stage = sm.kv[(t1 - t0 + (wave >> 1)) % kStages] + (wave & 1) * 32 * kPitch;
    static_assert(2 * 32 * kPitch <= kTileBytes, "rows of two waves fit a tile");
    {
      asm volatile("" : "+v"(l32), "+v"(h));
      const int to_lane = rare(lane);
      constexpr int kLanes = kCols / 8;  // of a row
      const auto put = [&](auto g) {
        f32x4* to = reinterpret_cast<f32x4*>(stage + l32 * kPitch + 16 * h);
#pragma unroll
        for (int db = 0; db < kDB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x16& x = o[db][g()];
            to[8 * db + 2 * q] = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
          }
      };
#pragma unroll 1
      for (int r = 0; r < valid; r += 32) {
        if (r == 0) put(std::integral_constant<int, 0>{});
        else if (r == 32) put(std::integral_constant<int, 1>{});
        else if (r == 64) put(std::integral_constant<int, 2>{});
        else put(std::integral_constant<int, 3>{});
        // (a lane's rows side by side: one after another they wait for themselves)
        constexpr int kEach = 32 * kLanes / kWave, kStep = kWave / kLanes;  // rows a lane, and to the next
        const int first = to_lane / kLanes, piece = to_lane % kLanes;
        const auto sums = [&](int i, int col) {  // dims 4 col .. of the i-th row
          return *reinterpret_cast<const f32x4*>(stage + (first + i * kStep) * kPitch + col * 16) * sm.row_f[r + first + i * kStep];
        };
        if (whole) {
          uint16_t* to = static_cast<uint16_t*>(in.out) +
                         (static_cast<int64_t>(b) * in.Nmax * in.Hq + r0 + r + first) * DL + wave * kCols + piece * 8;
          for_each_index<kEach>([&](auto i) {
            const f32x4 x0 = sums(i(), 2 * piece), x1 = sums(i(), 2 * piece + 1);
            if (r + first + i() * kStep < valid)
              *reinterpret_cast<u32x4*>(to + i() * kStep * DL) =
                  u32x4{pack_bf16x2(x0[0], x0[1]), pack_bf16x2(x0[2], x0[3]), pack_bf16x2(x1[0], x1[1]), pack_bf16x2(x1[2], x1[3])};
          });
        } else {  // (a slot has room for all 128 rows)
          float* to = a.ws_o + (static_cast<int64_t>(slot) * kRows + r + first) * DL + wave * kCols + piece * 4;
          for_each_index<kEach>([&](auto i) {
            *reinterpret_cast<f32x4*>(to + i() * kStep * DL) = sums(i(), piece);
            *reinterpret_cast<f32x4*>(to + i() * kStep * DL + kCols / 2) = sums(i(), kLanes + piece);
          });
        }
      }
    }
    pos = stop;
  }
}

// Joins the pieces of cut unit blockIdx.x (in the order of the shares that they begin in), a
// wave a row, kBatch pieces at a time: lane 16 g + p takes piece p's maximum and sum for the
// weights, then each lane its dims of every piece.  The pieces are asked for before their
// weights are known, and those of the next batch before the last one's are summed up (one token
// of a sequence of 16 heads over 8192 keys 24.4 us a call, 26.4 otherwise; where units have few
// pieces it changes nothing).
//
// Bound: the pieces' bytes where there are many rows (256 workgroups' 67 MB in about 13 us),
// one row's chain of loads where there are few.  (With a workgroup per share that looked
// up whether a cut begins there, and pieces' loads behind their weights, one token of 128
// heads over 4096 keys took 1 us more.)
template <int DL>
__global__ void __launch_bounds__(kThreads) latent_merge_kernel(LatentArgs a) {
  constexpr int kRuns = DL / (4 * kWave);  // of 4 dims a lane, 256 dims apart
  constexpr int kBatch = 8, kGroup = 4;    // pieces, and those whose loads go out together
  static_assert(kBatch % kGroup == 0 && kBatch <= 16, "a batch's pieces lie across 16 lanes");
  const LatentAttn& in = a.in;
  if (halted(in.status)) return;
  const int lane = threadIdx.x % kWave;
  // ---- which share the cut unit begins in
  int x = -1;
  CutUnit cut{};
  int rank = blockIdx.x;  // among the cuts from share `base` on
  for (int base = 0; base < a.W && x < 0; base += 4 * kWave) {
    CutUnit c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = a.ws_cut[min(base + i * kWave + lane, a.W - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t cuts = __ballot(base + i * kWave + lane < a.W && c[i].valid > 0);
      const int below = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(cuts >> 32),
                                                  __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(cuts), 0));
      const uint64_t hit = __ballot((cuts >> lane & 1) != 0 && below == rank);
      if (x < 0 && hit != 0) {
        const int l = __ffsll(static_cast<long long>(hit)) - 1;
        x = base + i * kWave + l;
        cut = CutUnit{__builtin_amdgcn_readlane(c[i].b, l), __builtin_amdgcn_readlane(c[i].r0, l),
                      __builtin_amdgcn_readlane(c[i].valid, l), __builtin_amdgcn_readlane(c[i].last, l)};
      }
      rank -= __popcll(cuts);
    }
  }
  const int row = blockIdx.y * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (x < 0 || row >= cut.valid) return;
  const int pieces = cut.last - x + 1;
  // (the first piece begins in share x, the others go on in the next ones)
  auto slot = [&](int p) { return static_cast<int64_t>(p == 0 ? 2 * x + 1 : 2 * (x + p)) * kRows + row; };
  struct Batch {
    float m, l;
    f32x4 d[kBatch][kRuns];
  };
  auto fetch = [&](Batch& t, int p0) {
    const int count = min(kBatch, pieces - p0);
    t.m = kNoMax;
    t.l = 0.f;
    if (lane % 16 < count) {
      const PieceRow r = a.ws_row[slot(p0 + lane % 16)];
      t.m = r.m;
      t.l = r.l;
    }
#pragma unroll
    for (int g = 0; g < kBatch; g += kGroup)
      if (g < count) {
#pragma unroll
        for (int u = g; u < g + kGroup; ++u)
#pragma unroll
          for (int i = 0; i < kRuns; ++i)
            t.d[u][i] = reinterpret_cast<const f32x4*>(a.ws_o + slot(p0 + min(u, count - 1)) * DL)[i * kWave + lane];
      }
  };
  float M = kNoMax, L = 0.f;
  f32x4 acc[kRuns];
#pragma unroll
  for (int i = 0; i < kRuns; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](const Batch& t, int p0) {
    const int count = min(kBatch, pieces - p0);
    const float m = t.l != 0.f ? t.m : kNoMax;
    const float m_new = fmaxf(M, row_reduce(m, [](float u, float v) { return fmaxf(u, v); }));
    const float old = exp2_fast(M - m_new), w = t.l != 0.f ? exp2_fast(m - m_new) * t.l : 0.f;
    L = L * old + row_reduce(w, [](float u, float v) { return u + v; });
    M = m_new;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) acc[i] *= old;
#pragma unroll
    for (int g = 0; g < kBatch; g += kGroup)
      if (g < count) {
#pragma unroll
        for (int u = g; u < g + kGroup; ++u) {
          const float wu = __shfl(w, u, 16);
          // (a piece of weight 0 is added too: it has 0, or NaN where an infinity stood
          // behind weights of 0, which has to reach the output however the row is cut)
          if (u < count) {
#pragma unroll
            for (int i = 0; i < kRuns; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][e] = __builtin_fmaf(wu, t.d[u][i][e], acc[i][e]);
          }
        }
      }
  };
  Batch t0, t1;
  fetch(t0, 0);
  for (int p = 0; p < pieces; p += 2 * kBatch) {
    if (p + kBatch < pieces) fetch(t1, p + kBatch);
    add(t0, p);
    if (p + 2 * kBatch < pieces) fetch(t0, p + 2 * kBatch);
    if (p + kBatch < pieces) add(t1, p + kBatch);
  }
  const float inv = 1.f / L;
  uint16_t* out = static_cast<uint16_t*>(in.out) + (static_cast<int64_t>(cut.b) * in.Nmax * in.Hq + cut.r0 + row) * DL;
#pragma unroll
  for (int i = 0; i < kRuns; ++i)
    reinterpret_cast<uint2*>(out)[i * kWave + lane] =
        make_uint2(pack_bf16x2(acc[i][0] * inv, acc[i][1] * inv), pack_bf16x2(acc[i][2] * inv, acc[i][3] * inv));
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
  __shared__ int32_t parents_s[LTD_MAX_NODES];
  __shared__ int path_len_s;
  if (halted(a.status)) return;
  const int i = blockIdx.x, b = blockIdx.z;
  if (i >= a.n_nodes[b]) return;
  const int t = threadIdx.x, lane = t % kWave, w = t / kWave;
  const int head = blockIdx.y * kWaves + w;
  const bool live = head < a.Hq;
  const int P = max(a.prefix_len[b], 0);
  if (t <= i) parents_s[t] = a.parents[static_cast<int64_t>(b) * a.Nmax + t];
  const int64_t row = static_cast<int64_t>(b) * a.Nmax + i;
  for (int e = lane; e < DK; e += kWave) {
    float v = 0.f;
    if (live)
      v = e < DL ? static_cast<const float*>(a.q_latent)[row * a.ql_row + head * a.ql_head + e]
                 : static_cast<const float*>(a.q_rope)[row * a.qr_row + head * a.qr_head + e - DL];
    q_s[w][e] = v;
  }
  __syncthreads();
  if (t == 0) path_len_s = root_path(parents_s, i, path_s);
  __syncthreads();
  const int n_keys = P + path_len_s;
  float m = -INFINITY, l = 0.f;
  float acc[DL / kWave];
#pragma unroll
  for (int e = 0; e < DL / kWave; ++e) acc[e] = 0.f;
  const float c = a.scale;
  // Eight threads load a key, into registers a tile ahead: the loads run beside the last
  // tile's products.
  constexpr int kPerKey = kThreads / kKeys, kLoads = kQuads / kPerKey;
  static_assert(kQuads % kPerKey == 0, "whole loads");
  const int my_key = t / kPerKey, my_col = t % kPerKey * 4;
  f32x4 next[kLoads];
  auto load = [&](int base) {
    const int kt = min(base + my_key, n_keys - 1);
    const int r = kt < P ? kt : P + path_s[kt - P];
    const float* src = static_cast<const float*>(a.cache) + cache_row(a.block_table, b, 0, r, 1, DK, a.kv_rows, a.max_blocks) + my_col;
    for_each_index<kLoads>([&](auto j) { next[j()] = *reinterpret_cast<const f32x4*>(src + j() * kPerKey * 4); });
  };
  load(0);
  for (int base = 0; base < n_keys; base += kKeys) {
    const int cnt = min(kKeys, n_keys - base);
    for_each_index<kLoads>([&](auto j) { *reinterpret_cast<f32x4*>(&x_s[my_key][my_col + j() * kPerKey * 4]) = next[j()]; });
    __syncthreads();
    if (base + kKeys < n_keys) load(base + kKeys);
    const int key = lane & 31, half = lane >> 5;
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
    const float* xr = &x_s[min(key, cnt - 1)][half * (DK / 2)];
    const float* qr = &q_s[w][half * (DK / 2)];
#pragma unroll 8
    for (int e = 0; e < DK / 2; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(xr + e), q = *reinterpret_cast<const float4*>(qr + e);
      s4[0] = __builtin_fmaf(x.x, q.x, s4[0]);
      s4[1] = __builtin_fmaf(x.y, q.y, s4[1]);
      s4[2] = __builtin_fmaf(x.z, q.z, s4[2]);
      s4[3] = __builtin_fmaf(x.w, q.w, s4[3]);
    }
    float s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
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
    // (a row past the last key is the last one again, of weight 0)
#pragma unroll 8
    for (int k = 0; k < kKeys; ++k) {
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
  hipError_t rc;
  const bool few = a.in.Nmax * static_cast<int64_t>(a.in.Hq) <= latent::kFewRows;
  if (few) {
    rc = launch_latent_few(&a, DL, stream);
  } else {
    if (a.in.block_table)
      hipLaunchKernelGGL((latent_attn_kernel<DL, true>), dim3(a.W), dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((latent_attn_kernel<DL, false>), dim3(a.W), dim3(kThreads), 0, stream, a);
    rc = hipGetLastError();
  }
  if (rc != hipSuccess || a.W < 2) return rc;
  // At most so many units are cut.
  const latent::Cut cut = few ? latent::kFew : latent::kMany;
  const int64_t units = a.in.B * latent::units_of(a.in.Nmax, a.in.Hq, cut);
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.W - 1, units)), cut.rows / kWaves);
  hipLaunchKernelGGL((latent_merge_kernel<DL>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t latent_attn_workspace_bytes(const LatentAttn& s, int d_latent, int dtype, int cus) {
  if (dtype == LTD_DTYPE_F32 || s.B == 0) return 0;
  const size_t W = grid_of(s, cus);
  return 2 * W * kRows * (d_latent * sizeof(float) + sizeof(PieceRow)) + W * sizeof(CutUnit);
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
  a.ws_cut = reinterpret_cast<CutUnit*>(a.ws_o + static_cast<int64_t>(2) * a.W * kRows * d_latent);
  a.ws_row = reinterpret_cast<PieceRow*>(a.ws_cut + a.W);
  a.scale_log2 = s.scale * kLog2e;
  a.lazy_gap = kLazyMax / a.scale_log2;
  a.block = latent::row_divisor(s.kv_rows);
  return d_latent == 512 ? launch_bf16<512>(a, stream) : launch_bf16<256>(a, stream);
}

}  // namespace ltd
