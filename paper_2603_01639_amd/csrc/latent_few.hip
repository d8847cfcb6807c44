// Tree attention over a latent cache for calls of up to 16 stacked query rows a sequence
// (one token, or a few nodes, of a few heads), in bf16 on the matrix cores.
//
// The cache's bytes bound these calls, so the split follows the stream: the four waves
// of a workgroup take every fourth tile of 16 keys of its share, each with a double
// buffer of its own in LDS that direct loads fill, rows in registers, and no barrier
// until the share ends.
//   S^T[key][row] = X Q^T         (v_mfma_f32_16x16x32_bf16, 18 a tile)
//   O^T[dim][row] += C^T P^T      (the same with both parts of 16 weights, 32 a tile)
// A lane's four accumulators of S^T are four keys of its row and as they are, in two parts,
// its operand P^T; C^T comes from the same tile by transposed reads, each value twice.  The
// waves' results are joined through LDS at the end.
//
// 16 heads, this kernel and the one for many rows (which pads them to 128), both with
// the merge, in a graph: one token of a sequence over 1000 keys 17.8 us, 18.9; of 16
// sequences 21, 22; of 16 over 1024 to 8192 keys 33, 40; of 16 over 8192 keys 47, 55; of 128
// over 2048 keys 79, 100.  With 32 rows, in two units that each read the cache, 16
// sequences over 8192 keys took 58 us where the other kernel takes 55, hence the rule.
// 16 sequences over 1024 to 8192 keys (85 MB) take 25 to 26 us before the merge, half of it the
// stream at 6 TB/s, the rest the search, the first loads and the join.
#include "latent_attn.hpp"

namespace ltd {
namespace {

constexpr int kKeys = 16;            // of a tile
constexpr int kPlane = kKeys * 128;  // 64 dims of a tile in LDS

// A tile's 16-byte chunks within a plane trade places by their key: neither 16 lanes of
// an S^T operand's read (one chunk of 16 keys; even and odd ones lie in different halves
// of the banks) nor 32 lanes of a transposed read (32 bytes of eight keys) meet on a bank.
__device__ __forceinline__ int swz(int key) {
  return ((key >> 1) & 1) << 1 | ((key >> 2) & 1) << 2 | ((key >> 3) & 1);
}

// The products by hand, sums in vector registers (the compiler would keep them in the
// accumulation registers and move all of O out and in for every tile).  What else reads a
// sum waits: 16 wait states are more than a product takes.
__device__ __forceinline__ void mfma_s(f32x4& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_first(f32x4& s, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_settle(f32x4& s) { asm volatile("s_nop 15" : "+v"(s)); }
__device__ __forceinline__ void settled(f32x4& o) { asm volatile("" : "+v"(o)); }

template <int DL>
struct Smem {
  static constexpr int kTileBytes = (DL + kRopeDims) / 64 * kPlane;
  union {
    alignas(16) unsigned char kv[kWaves][2][kTileBytes];
    f32x4 o[kWaves][16][DL / 4];  // the waves' results of 16 rows
  };
  float m[kWaves][16], l[kWaves][16];
  int32_t ids[kWaves][2][kWave];  // block ids of the tile that follows a buffer's, key i % 16 at i
};

template <int DL, bool kPaged>
__global__ void __launch_bounds__(kThreads, 1) latent_few_kernel(LatentArgs a) {
  constexpr latent::Cut kCut = latent::kFew;
  constexpr int kTilesPer = latent::kKeyTile / kKeys;  // tiles here of one in the cut
  constexpr int DK = DL + kRopeDims;
  constexpr int kRowBytes = DK * 2;
  constexpr int kPlanes = DK / 64;
  constexpr int kTileBytes = kPlanes * kPlane;
  constexpr int kSteps = DK / 32;   // k-steps of S^T
  constexpr int kBlocks = DL / 16;  // 16-dim blocks of O^T
  __shared__ Smem<DL> sm;
  const LatentAttn& in = a.in;
  if (halted(in.status)) return;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane & 15, quad = lane >> 4;

  int64_t total, share;
  const int rank = a.W % 8 == 0 ? static_cast<int>(blockIdx.x % 8) * (a.W / 8) + static_cast<int>(blockIdx.x / 8)
                                : static_cast<int>(blockIdx.x);
  const Seq first_seqs = seq_of(in, lane);
  const Place place = find_place(in, kCut, lane, first_seqs, &total, [&](int64_t t) {
    share = latent::share_of(t, a.W, kCut);
    return rank * share;
  });
  share = uniform(share);
  int64_t pos = rank * share;
  const int64_t end = min(pos + share, total);
  if (threadIdx.x == 0) a.ws_cut[rank].valid = 0;
  if (pos >= end) return;
  int b = __builtin_amdgcn_readfirstlane(place.b);
  int64_t before = uniform(place.before);

  // ---- lane constants.  Direct loads: lane 8 k + c fetches chunk c of keys k and k + 8.
  const int load_key = lane >> 3;
  const int off0 = ((lane & 7) ^ swz(load_key)) * 16, off1 = ((lane & 7) ^ swz(load_key + 8)) * 16;
  // S^T operand: key l16, chunk 4 kk + quad (k-steps in turn take a plane's first and last half)
  const int k_rd = l16 * 128 + ((quad ^ swz(l16)) << 4);
  // C^T operand: keys 4 quad + .., 16 dims from 16 block on
  const int v_key = 4 * quad + (l16 >> 2);
  const int v_rd = v_key * 128 + ((((l16 & 3) >> 1) ^ swz(v_key)) << 4) + (l16 & 1) * 8;
  const uint32_t ring = lds_addr(sm.kv[wave][0]), ids = lds_addr(sm.ids[wave][0]);
  const float c = a.scale_log2;

  while (pos < end) {
    // ---- the unit's piece in this share
    const Seq seq = b < kWave ? first_seqs : seq_of(in, b);
    const int n = __builtin_amdgcn_readlane(seq.n, b % kWave), P = __builtin_amdgcn_readlane(seq.P, b % kWave);
    const int64_t length = kCut.cost + latent::tiles_of(P, n);
    if (n == 0 || pos >= before + length) {
      if (n != 0) before += length;
      ++b;
      continue;
    }
    const int64_t start = before;  // (its one unit)
    const int64_t stop = uniform(min(start + length, end));
    const int t0 = __builtin_amdgcn_readfirstlane(static_cast<int>(latent::tile_at(pos - start, kCut))) * kTilesPer;
    const int t1 = __builtin_amdgcn_readfirstlane(static_cast<int>(latent::tile_at(stop - start, kCut))) * kTilesPer;
    const bool whole = t0 == 0 && stop == start + length;
    const int slot = 2 * rank + (t0 == 0);  // (one piece that goes on, one that begins)
    const int valid = n * in.Hq;
    const int last = P + n - 1;
    pos = stop;
    if (t1 == t0) continue;  // (a share that ends within a unit's own cost)

    // a tile's direct loads, by the block ids of the lane's two keys; behind them those of the
    // ids of the tile that will follow in the buffer, so that one wait covers both
    const auto table_at = [&](int key) {
      return in.block_table + (static_cast<int64_t>(b) * in.max_blocks + block_of(a, min(key, last)));
    };
    auto issue = [&](int t, int buffer, int id0, int id1) {
      const unsigned char* from[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        from[k] = static_cast<const unsigned char*>(in.cache) +
                  (static_cast<uint64_t>(row_place<kPaged>(a, b, min(t * kKeys + load_key + 8 * k, last), k == 0 ? id0 : id1)) * kRowBytes +
                   (k == 0 ? off0 : off1));
      const uint32_t dst = ring + buffer * kTileBytes;
      for_each_index<kPlanes>([&](auto g) {
        dma16_at<g() * 128>(dst + g() * kPlane, from[0]);
        dma16_at<g() * 128>(dst + g() * kPlane + 1024, from[1]);
      });
      if constexpr (kPaged) dma4(ids + buffer * kWave * 4, table_at((t + 2 * kWaves) * kKeys + l16));
    };
    constexpr int kLoads = 2 * kPlanes + (kPaged ? 1 : 0);

    // ---- the queries (lane: row l16, dims 32 kk + 8 quad ..) and the tree's links, then the
    // first two of the wave's tiles, which are t0 + wave and every fourth from there
    bf16x8 qf[kSteps];
    int node;
    {
      const uint32_t r = min(l16, valid - 1), heads = in.Hq;
      node = static_cast<int>(r / heads);
      const int head = static_cast<int>(r % heads);
      const int64_t row = static_cast<int64_t>(b) * in.Nmax + node;
      const uint16_t* ql = static_cast<const uint16_t*>(in.q_latent) + row * in.ql_row + head * in.ql_head + 8 * quad;
      const uint16_t* qr = static_cast<const uint16_t*>(in.q_rope) + row * in.qr_row + head * in.qr_head + 8 * quad;
#pragma unroll
      for (int kk = 0; kk < DL / 32; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(ql + 32 * kk);
#pragma unroll
      for (int kk = 0; kk < kRopeDims / 32; ++kk) qf[DL / 32 + kk] = *reinterpret_cast<const bf16x8*>(qr + 32 * kk);
    }
    int par = -1;
    if (lane < n) par = min(in.parents[static_cast<int64_t>(b) * in.Nmax + lane], lane - 1);
    int first_ids[2][2] = {{0, 0}, {0, 0}};
    if constexpr (kPaged) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        first_ids[i / 2][i % 2] = *table_at((t0 + wave + i / 2 * kWaves) * kKeys + load_key + 8 * (i % 2));
    }
    // (asked for before the tiles: a later wait for one of these would wait for tiles too)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(qf[kk]));
    asm volatile("" : "+v"(par));
    if (t0 + wave < t1) issue(t0 + wave, 0, first_ids[0][0], first_ids[0][1]);
    if (t0 + wave + kWaves < t1) issue(t0 + wave + kWaves, 1, first_ids[1][0], first_ids[1][1]);
    // the lane's node's ancestors: at most 16 nodes, whose links lie across the wave
    uint32_t anc = 0;
    if (t1 * static_cast<int64_t>(kKeys) > P) {
      int j = node;
      while (__ballot(j >= 0) != 0) {  // (every link goes down, so at most n steps)
        if (j >= 0) anc |= 1u << j;
        const int up = __shfl(par, max(j, 0), kWave);
        j = j > 0 ? up : -1;
      }
    }

    float m_run = kNoMax, l_run = 0.f;
    f32x4 o[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    int buffer = 0;
#pragma unroll 1
    for (int t = t0 + wave; t < t1; t += kWaves, buffer ^= 1) {
      if (t + kWaves < t1) wait_vmcnt<kLoads>();
      else wait_vmcnt<0>();
      unsigned char* kv = sm.kv[wave][buffer];
      // A tree key whose latent part holds a NaN or an infinity: the nodes that see it get
      // NaN, and for the others its values, which 0 would multiply, are cleared.
      const bool masked = (t + 1) * static_cast<int64_t>(kKeys) > P;
      uint32_t bad = 0;
      if (masked) {
        uint32_t any = 0;  // bits of keys: 64 lanes look at 128 bytes of eight of them at a time
#pragma unroll 1
        for (int e = 0; e < kKeys * DL * 2 / 16 / kWave; ++e) {
          const int at = (e * kWave + lane) * 16;
          const u32x4 x = *reinterpret_cast<const u32x4*>(kv + at);
          uint32_t hit = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) hit |= ((x[j] & 0x7F80u) == 0x7F80u) | ((x[j] & 0x7F800000u) == 0x7F800000u);
          if (hit) any |= 1u << (at / 128 % kKeys);
        }
        any |= lane_xor<1>(any, lane);
        any |= lane_xor<2>(any, lane);
        any |= lane_xor<4>(any, lane);
        any |= lane_xor<8>(any, lane);
        any |= lane_xor<16>(any, lane);
        any |= lane_xor<32>(any, lane);
        bad = __builtin_amdgcn_readfirstlane(any);
      }
      f32x4 s;
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kv + (k_rd ^ ((kk & 1) << 6)) + (kk >> 1) * kPlane);
        if (kk == 0) mfma_first(s, kf, qf[0]);
        else mfma_s(s, kf, qf[kk]);
      }
      mfma_settle(s);
      if (masked) {
        // bit j: tree key t * 16 - P + 4 quad + j (earlier ones are the prefix, later ones none)
        const int base = t * kKeys - P + 4 * quad;
        const uint32_t vis = base >= 16 ? 0u : base >= 0 ? anc >> base
                             : base > -16 ? (anc << -base) | ((1u << -base) - 1u) : 0xFFFFFFFFu;
        const uint32_t nan = bad >> (4 * quad);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = !((vis >> j) & 1u) ? -INFINITY : (nan >> j) & 1u ? NAN : s[j];
      }
      float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[0], s[1]),
                                                __builtin_elementwise_maximum(s[2], s[3]));
      top = rows_reduce(top, [](float x, float y) { return __builtin_elementwise_maximum(x, y); });
      const float m_new = top > m_run + a.lazy_gap ? top : m_run;
      const float neg = fminf(-m_new * c, __FLT_MAX__);
      if (__ballot(m_new != m_run) != 0) {
        const float alpha = exp2_fast((m_run - m_new) * c);
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) o[d] *= alpha;
        m_run = m_new;
      }
      // Weights in two parts, rounded and what that left, 16 bits in all: a product of 32
      // factors takes the time of one of 16, and with one part the outputs' error was 0.0019
      // of them where their own rounding gives 0.0017 (one token of 16 sequences of 16 heads 32.1
      // us a call, with one part 32.6).
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float p0 = exp2_fast(__builtin_fmaf(s[2 * j], c, neg)), p1 = exp2_fast(__builtin_fmaf(s[2 * j + 1], c, neg));
        w[j] = pack_bf16x2(p0, p1);
        w[2 + j] = pack_bf16x2(p0 - __builtin_bit_cast(float, w[j] << 16), p1 - __builtin_bit_cast(float, w[j] & 0xFFFF0000u));
      }
      // (the sum is that of the very weights that multiply the values)
      const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t two = w[j];
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, l_run, false);
      }
      bf16x8 pf = __builtin_bit_cast(bf16x8, w);
      if (bad != 0) {
#pragma unroll 1
        for (int e = 0; e < kKeys * DL * 2 / 16 / kWave; ++e) {
          const int at = (e * kWave + lane) * 16;
          if ((bad >> (at / 128 % kKeys)) & 1u) *reinterpret_cast<u32x4*>(kv + at) = u32x4{0, 0, 0, 0};
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      }
      for_each_index<kBlocks / 4>([&](auto plane) {
        bf16x8 vf[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const s16x4 v = lds_read_tr(kv + (v_rd ^ (d << 5)) + plane() * kPlane);
          vf[d] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v, v, 0, 1, 2, 3, 0, 1, 2, 3));
        }
        // (a product reads what vector operations wrote two wait states later)
        asm volatile("s_nop 1" : "+v"(vf[0]), "+v"(vf[1]), "+v"(vf[2]), "+v"(vf[3]), "+v"(pf));
#pragma unroll
        for (int d = 0; d < 4; ++d) mfma_s(o[4 * plane() + d], vf[d], pf);
      });
      if (t + 2 * kWaves < t1) {
        const int id0 = kPaged ? sm.ids[wave][buffer][load_key] : 0, id1 = kPaged ? sm.ids[wave][buffer][load_key + 8] : 0;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the buffer's last reads are done
        issue(t + 2 * kWaves, buffer, id0, id1);
      }
    }

    // ---- the waves' results joined
    asm volatile("s_nop 15");
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) settled(o[d]);
    const int jl = rare(lane), row16 = jl & 15, part = jl >> 4;
    l_run = rows_reduce(l_run, [](float x, float y) { return x + y; });
    if (part == 0) {
      sm.m[wave][row16] = m_run * c;
      sm.l[wave][row16] = l_run;
    }
    __syncthreads();  // (all waves are done with their tiles, too)
    float M = kNoMax * __FLT_MAX__, L = 0.f;  // (-inf)
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (sm.l[w][row16] != 0.f) M = fmaxf(M, sm.m[w][row16]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (sm.l[w][row16] != 0.f) L += exp2_fast(sm.m[w][row16] - M) * sm.l[w][row16];
    // (a wave without a visible key has weight 0, as has such a piece, and O = 0, or NaN where
    // an infinity stood behind weights of 0)
    const float f = l_run == 0.f && (L != 0.f || !whole) ? 0.f : exp2_fast(m_run * c - M) / L;
    if (!whole && wave == 0 && part == 0 && row16 < valid)
      a.ws_row[static_cast<int64_t>(slot) * kRows + row16] = PieceRow{M, L};
    if (!whole && t0 == 0 && threadIdx.x == 0)
      a.ws_cut[rank] = CutUnit{b, 0, valid, static_cast<int>(latent::quotient(start + length - 1, share))};
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
      sm.o[wave][row16][(4 * d + part) ^ (row16 & 7)] = o[d] * f;
    __syncthreads();
    const auto sum_of = [&](int row, int col) {  // dims 4 col ..
      f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x += sm.o[w][row][col ^ (row & 7)];
      return x;
    };
    if (whole) {
      uint16_t* out = static_cast<uint16_t*>(in.out) + static_cast<int64_t>(b) * in.Nmax * in.Hq * DL;
#pragma unroll 2
      for (int e = rare(static_cast<int>(threadIdx.x)); e < valid * (DL / 8); e += kThreads) {
        const int row = e / (DL / 8), col = e % (DL / 8);
        const f32x4 x0 = sum_of(row, 2 * col), x1 = sum_of(row, 2 * col + 1);
        *reinterpret_cast<u32x4*>(out + static_cast<int64_t>(row) * DL + col * 8) =
            u32x4{pack_bf16x2(x0[0], x0[1]), pack_bf16x2(x0[2], x0[3]), pack_bf16x2(x1[0], x1[1]), pack_bf16x2(x1[2], x1[3])};
      }
    } else {
      float* out = a.ws_o + static_cast<int64_t>(slot) * kRows * DL;
#pragma unroll 2
      for (int e = rare(static_cast<int>(threadIdx.x)); e < valid * (DL / 4); e += kThreads)
        *reinterpret_cast<f32x4*>(out + e * 4) = sum_of(e / (DL / 4), e % (DL / 4));
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_latent_few(const void* args, int d_latent, hipStream_t stream) {
  const LatentArgs& a = *static_cast<const LatentArgs*>(args);
  const bool paged = a.in.block_table != nullptr;
  const dim3 grid(a.W), threads(kThreads);
  if (d_latent == 512) {
    if (paged) hipLaunchKernelGGL((latent_few_kernel<512, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((latent_few_kernel<512, false>), grid, threads, 0, stream, a);
  } else {
    if (paged) hipLaunchKernelGGL((latent_few_kernel<256, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((latent_few_kernel<256, false>), grid, threads, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace ltd
