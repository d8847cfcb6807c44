// The matrix-core attention over an 8-bit cache: the tile loop's kernels (attn_mfma.hpp)
// instantiated for it, and the short units' own.
#include <cstddef>

#include "attn_mfma.hpp"
#include "few_plan.hpp"

namespace ltd {
namespace {

// ---- units of at most 32 stacked rows over an 8-bit cache (decoding, short
// trees).  Such calls are bound by the cache's bytes.  A (sequence, kv head) is
// cut into splits of one length, the tree's keys joining the last, one for a
// workgroup of four waves; two workgroups share a compute unit.  The length is
// worked out on the GPU from the call's own lengths (few_plan.hpp).  Every wave
// takes all of the unit's rows and its own 32-key blocks (block i: wave i mod 4),
// from loads to P.V, with no barrier until the waves' results are joined.  Its
// blocks move straight into two slots of LDS of its own, refilled as soon as they
// are read: 8 to 16 KiB requested per wave, 64 to 128 per compute unit (with the
// next block in registers, which are free only part of a block's time, 16
// sequences of 1024 to 8192 keys, 64/8 heads, one node: 44.6 us a call instead of
// 42.2; of now 39.5 the kernel takes about 35, 154 MB at 4.4 TB/s, and the merge 4).
//
// K lies in LDS as the S^T operand takes it: lane l finds the codes of key
// sigma(l & 31), 16 dims in every 32, where its own load put them (Q's fragments
// have their dims in the same order), and widens them.  V's rows lie as in the
// cache, 16-byte chunks swizzled; ds_read_b64_tr_b8 hands each lane 8 keys of one
// dim, widened next.  A fragment of 8 keys lies in one scale block in every
// full block; in a range's last partial block and the tree's (32 nodes at most,
// one block) each key's V scale multiplies its weights instead, an exact power
// of two.
constexpr int kFewWaves = 4;
constexpr int kFewThreads = kFewWaves * kWave;
constexpr int kFewBlocks = 512;  // paged block ids a split may span
constexpr int kFewSlots = 2;     // blocks a wave has in LDS or on the way

// A wave's slot: K's codes by lane, V's rows, the scale bytes (a word each) of
// every lane's K row and of V (full block: keys 16 (l / 32) .., else key l & 31).
template <int HD>
struct FewSlot {
  unsigned char k[32 * HD];
  unsigned char v[32 * HD];
  uint32_t ks[kWave];
  uint32_t vs[kWave];
};
template <int HD>
struct FewSmem {
  union {
    FewSlot<HD> slot[kFewWaves][kFewSlots];
    float o[kFewWaves][kFewRows][HD];  // the waves' results
  };
  uint16_t q[kFewRows][HD];  // 16-byte chunk c of row r at c ^ (r & 7)
  float ml[kFewWaves][kFewRows][2];
  int32_t blk[kFewBlocks];  // row groups (id * Hkv + g) of the split's pages
};

// What a workgroup of the grid works on: split `split` of `n_splits` of
// sequence b and kv head g; w is its place among the call's splits (b major,
// then g, then split), and the unit's first split's place is w - split.  b < 0:
// the call has fewer splits.  more: they come in rounds.
struct FewWork {
  int b, g, split, n_splits, P, split_keys;
  bool more;
};

// Every wave works it out on its own (lane l holds sequence c * 64 + l of chunk
// c; one sequence takes a scalar load and no scans).
__device__ __forceinline__ FewWork few_find(const MfmaArgs& a, int w) {
  const int lane = __lane_id();
  FewWork r{-1, 0, 0, 0, 0, 0, false};
  if (a.B == 1) {
    r.P = min(max(a.prefix_len[0], 0), a.max_prefix);
    const few::Length len = few::one_length(r.P, a.Hkv, a.W, a.few_width, a.max_prefix);
    r.split_keys = len.keys;
    r.more = len.rounds > 1;
    r.n_splits = max((r.P + r.split_keys - 1) / r.split_keys, 1);
    r.g = w / r.n_splits;
    r.split = w - r.g * r.n_splits;
    r.b = r.g < a.Hkv ? 0 : -1;
    return r;
  }
  auto length = [&](int b) { return b < a.B ? min(max(a.prefix_len[b], 0), a.max_prefix) : 0; };
  const int P0 = length(lane);
  int64_t T = readlane_i64(wave_scan_i64(P0), kWave - 1);
  for (int c0 = kWave; c0 < a.B; c0 += kWave) T += readlane_i64(wave_scan_i64(length(c0 + lane)), kWave - 1);
  const few::Length len = few::batch_length(T, a.Hkv, a.B * a.Hkv, a.W, a.few_width, a.max_prefix, [&](int keys) {
    float n = 0.f;  // (below 2^24: exact)
    for (int c0 = 0; c0 < a.B; c0 += kWave) {
      const int P = c0 == 0 ? P0 : length(c0 + lane);
      n += c0 + lane < a.B ? static_cast<float>(max((P + keys - 1) / keys, 1)) : 0.f;
    }
    return __builtin_amdgcn_readfirstlane(static_cast<int>(wave_sum_dpp(n))) * a.Hkv;
  });
  const int sk = len.keys;
  r.split_keys = sk;
  r.more = len.rounds > 1;
  int before = 0;  // splits of the sequences before this chunk
  for (int c0 = 0; c0 < a.B; c0 += kWave) {
    const int P = c0 == 0 ? P0 : length(c0 + lane);
    const int n = c0 + lane < a.B ? max((P + sk - 1) / sk, 1) : 0;  // splits per head
    const int upto = static_cast<int>(wave_scan_i64(n * a.Hkv)) + before;
    const int start = upto - n * a.Hkv;
    const uint64_t hit = __ballot(start <= w && w < upto);
    if (hit != 0) {
      const int l = __ffsll(static_cast<long long>(hit)) - 1;
      r.b = c0 + l;
      r.P = __builtin_amdgcn_readlane(P, l);
      r.n_splits = __builtin_amdgcn_readlane(n, l);
      const int at = w - __builtin_amdgcn_readlane(start, l);
      r.g = at / r.n_splits;
      r.split = at - r.g * r.n_splits;
      return r;
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return r;
}

// The split at place slot_id; whether the workgroup may have another, a grid on.
template <int HD, bool kPaged, bool kLoop>
__device__ __forceinline__ bool attend_few(const MfmaArgs& a, FewSmem<HD>& sm, int slot_id) {
  const FewWork fw = few_find(a, slot_id);
  if (fw.b < 0) return false;
  const int b = fw.b, g = fw.g, P = fw.P;
  const int n = min(max(a.n_nodes[b], 1), a.Nmax);
  const bool has_tree = fw.split == fw.n_splits - 1;
  const bool final_out = fw.n_splits == 1;
  const int valid_rows = a.G * n;
  const int key_begin = fw.split * fw.split_keys;
  const int n_pre = min(fw.split_keys, P - key_begin);
  if (fw.split == 0 && threadIdx.x == 0)
    reinterpret_cast<FewDesc*>(a.ws_desc)[b * a.Hkv + g] = FewDesc{slot_id, fw.n_splits};
  // (an opaque copy of the thread's index: otherwise the compiler keeps what
  // follows from it alone in registers from one split to the next)
  int tid = threadIdx.x;
  if constexpr (kLoop) asm volatile("" : "+v"(tid));
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lane = tid % kWave;
  const int h = lane >> 5, l32 = lane & 31;
  constexpr int kKC = HD / 32;                // 16-code chunks of a lane's K
  constexpr int kVRow = HD / 16;              // lanes of a V row
  constexpr int kVKeys = kWave / kVRow;       // keys of a V load
  constexpr int kVC = 32 / kVKeys;            // V loads of a block
  constexpr int kLoads = kKC + kVC + 2;       // loads of a block
  constexpr int kRowBytes = HD;               // a V row in LDS
  const int n_full = n_pre / 32;              // full prefix blocks
  const int n_blocks = (n_pre + 31) / 32;     // ... and a partial one
  const int n_all = n_blocks + (has_tree ? 1 : 0);

  // ---- Q's rows (rows past the unit's repeat its last) and, for a paged cache,
  // the split's row groups
  constexpr int kQRowChunks = HD / 8;
  constexpr int kQLoads = kFewRows * kQRowChunks / kFewThreads;  // 16-byte chunks a thread: 2 or 1
#pragma unroll
  for (int j = 0; j < kQLoads; ++j) {
    const int x = j * kFewThreads + tid;
    const int r = x / kQRowChunks, qr = min(r, valid_rows - 1);
    const int node = node_of(a, qr);
    const uint16_t* src = a.q +
        ((static_cast<int64_t>(b) * a.Nmax + node) * a.Hq + g * a.G + (qr - node * a.G)) * HD +
        ((x % kQRowChunks) ^ (r & 7)) * 8;
    dma16(lds_addr(&sm.q[0][0]) + (j * kFewThreads + wave * kWave) * 16, src);
  }
  const int first_blk = kPaged ? key_begin / a.kv_rows : 0;
  if constexpr (kPaged) {
    const int n_blk = (key_begin + n_pre + (has_tree ? n : 0) - 1) / a.kv_rows - first_blk + 1;
    const int32_t* bt = a.block_table + static_cast<int64_t>(b) * a.max_blocks + first_blk;
    for (int j = tid; j < n_blk; j += kFewThreads) sm.blk[j] = bt[j] * a.Hkv + g;
    __syncthreads();
  }
  auto place = [&](int row, int64_t& rg, int& in) {
    if (!kPaged) {
      rg = static_cast<int64_t>(b) * a.Hkv + g;
      in = row;
    } else if (a.kv_shift >= 0) {
      rg = sm.blk[(row >> a.kv_shift) - first_blk];
      in = row & (a.kv_rows - 1);
    } else {
      const int blk = row / a.kv_rows;
      rg = sm.blk[blk - first_blk];
      in = row - blk * a.kv_rows;
    }
  };
  // Byte offsets of a row's codes and of its scale byte; `uniform` rows go
  // through scalar registers.
  auto offsets = [&](int row, bool uniform, int64_t& at, int64_t& st) {
    int64_t rg;
    int in;
    place(row, rg, in);
    if (uniform) {
      rg = __builtin_amdgcn_readfirstlane(static_cast<int>(rg));
      in = __builtin_amdgcn_readfirstlane(in);
    }
    at = (rg * a.kv_rows + in) * HD;
    st = rg * a.scale_per_page + (in >> a.scale_shift);
  };
  // V in LDS: chunk c of key k at c ^ f(k), so that the 8 keys x 16 dims of a
  // transposed read spread over the banks.
  const auto v_swz = [](int key) { return HD == 128 ? (key >> 1) & 3 : (key >> 2) & 3; };
  const unsigned char* kbase = reinterpret_cast<const unsigned char*>(a.k);
  const unsigned char* vbase = reinterpret_cast<const unsigned char*>(a.v);
  const int k_key = sigma(l32);
  const uint32_t slot0_lds = lds_addr(&sm.slot[wave][0]);
  int v_off[kVC];  // the lane's chunk of each V load, within its row
#pragma unroll
  for (int j = 0; j < kVC; ++j) v_off[j] = ((lane % kVRow) ^ v_swz(j * kVKeys + lane / kVRow)) * 16;
  // Requests block i (wave-uniform) into slot s.
  auto load = [&](int i, int s) {
    const uint32_t k_lds = slot0_lds + s * sizeof(FewSlot<HD>);
    const uint32_t v_lds = k_lds + offsetof(FewSlot<HD>, v);
    const uint32_t s_lds = k_lds + offsetof(FewSlot<HD>, ks);
    if (i < n_full) {
      // 32 keys from a multiple of 32: each half lies in one page and one scale block
      const int row = key_begin + 32 * i;
      int64_t at0, at1, st0, st1;
      offsets(row, true, at0, st0);
      offsets(row + 16, true, at1, st1);
      const int up = k_key >> 4;
      const unsigned char* kp = kbase + (up ? at1 : at0) + (k_key & 15) * HD + h * 16;
#pragma unroll
      for (int j = 0; j < kKC; ++j) dma16(k_lds + j * 1024, kp + 32 * j);
#pragma unroll
      for (int j = 0; j < kVC; ++j) {
        const int first = j * kVKeys;  // (its keys share a half)
        dma16(v_lds + j * 1024, vbase + (first >= 16 ? at1 : at0) + ((first & 15) + lane / kVRow) * HD + v_off[j]);
      }
      dma1(s_lds, a.ks + (up ? st1 : st0));
      dma1(s_lds + sizeof(uint32_t) * kWave, a.vs + (h ? st1 : st0));
      return;
    }
    const bool tree = i == n_blocks;
    const int row = tree ? P : key_begin + 32 * i;
    const int last = (tree ? n : n_pre - 32 * i) - 1;  // keys past the range read its last row, masked out
    int64_t at, st;
    offsets(row + min(k_key, last), false, at, st);
#pragma unroll
    for (int j = 0; j < kKC; ++j) dma16(k_lds + j * 1024, kbase + at + h * 16 + 32 * j);
    dma1(s_lds, a.ks + st);
#pragma unroll
    for (int j = 0; j < kVC; ++j) {
      offsets(row + min(j * kVKeys + lane / kVRow, last), false, at, st);
      dma16(v_lds + j * 1024, vbase + at + v_off[j]);
    }
    offsets(row + min(l32, last), false, at, st);
    dma1(s_lds + sizeof(uint32_t) * kWave, a.vs + st);
  };
  const int mine = wave < n_all ? (n_all - wave + kFewWaves - 1) / kFewWaves : 0;  // this wave's blocks
#pragma unroll
  for (int s = 0; s < kFewSlots; ++s)
    if (s < mine) load(wave + s * kFewWaves, s);
  // (Q has landed once no more than those loads are outstanding)
  if (mine >= 2) wait_vmcnt<2 * kLoads>();
  else if (mine == 1) wait_vmcnt<kLoads>();
  else wait_vmcnt<0>();
  barrier_only();

  // ---- Q: lane holds row l32, chunk j's 16 dims 32 j + 16 h .. as two k-steps
  const bool qvalid = l32 < valid_rows;
  const int qnode = node_of(a, min(l32, valid_rows - 1));
  bf16x8 qf[kKC][2];
#pragma unroll
  for (int j = 0; j < kKC; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      qf[j][e] = *reinterpret_cast<const bf16x8*>(&sm.q[l32][((4 * j + 2 * h + e) ^ (l32 & 7)) * 8]);

  // ---- the ancestors of row l32's node, by doubling over the links (lane =
  // node; at most 32 of them), in the wave that takes the tree's block
  uint32_t anc = 0;
  if (has_tree && wave == n_blocks % kFewWaves) {
    int jump = lane > 0 && lane < n ? a.parents[static_cast<int64_t>(b) * a.Nmax + lane] : -1;
    uint32_t set = lane < n ? 1u << (lane & 31) : 0u;
    for (int r = 0; r < 5; ++r) {
      const int j = min(max(jump, 0), kWave - 1);  // (a malformed link stays in the wave)
      const uint32_t other = __shfl(set, j, kWave);
      const int next = __shfl(jump, j, kWave);
      if (jump >= 0) {
        set |= other;
        jump = next;
      }
    }
    anc = __shfl(set, qnode, kWave);
  }

  float m_run = kNoMax, l_run = 0.f;
  f32x16 o_acc[HD / 32];
#pragma unroll
  for (int db = 0; db < HD / 32; ++db) o_acc[db] = f32x16{};
  const float c = a.scale_log2;
  uint32_t nan_keys = 0;  // tree rows with a NaN code in V
  // transposed read: 16-lane group q, lane s of it: key 16 (q / 2) + 8 kk + s / 2, dims 32 db + 16 (q % 2) + 8 (s % 2)
  const int tq = lane >> 4, ts = lane & 15;
  int v_rd[2][HD / 32];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk)
#pragma unroll
    for (int db = 0; db < HD / 32; ++db) {
      const int key = 16 * (tq >> 1) + 8 * kk + (ts >> 1);
      v_rd[kk][db] = key * kRowBytes + (((2 * db + (tq & 1)) ^ v_swz(key)) << 4) + 8 * (ts & 1);
    }

#pragma unroll 1
  for (int it = 0; it < mine; ++it) {
    const int i = wave + it * kFewWaves;
    const bool full = i < n_full;
    const bool tree = has_tree && i == n_blocks;
    FewSlot<HD>& sl = sm.slot[wave][it % kFewSlots];
    if (it + 1 < mine) wait_vmcnt<kLoads>();
    else wait_vmcnt<0>();
    if (tree) {  // NaN codes in V leave the product (see attend)
#pragma unroll
      for (int j = 0; j < kVC; ++j) {
        u32x4* at = reinterpret_cast<u32x4*>(sl.v + j * 1024) + lane;
        u32x4 codes = *at;
        const bool bad = q8_clear_nan(codes);
        const uint64_t hit = __ballot(bad);
        if (bad) *at = codes;
        for (int k = 0; k < kVKeys && hit != 0; ++k)
          if ((hit >> (k * kVRow)) & ((1u << kVRow) - 1)) nan_keys |= 1u << (j * kVKeys + k);
      }
    }
    const uint32_t ks = sl.ks[lane];
    const float v_scale = full ? q8_scale(static_cast<int>(sl.vs[lane])) : 1.f;
    f32x16 s = {};
#pragma unroll
    for (int j = 0; j < kKC; ++j) {
      u32x4 w[2];
      q8_to_bf16(reinterpret_cast<const u32x4*>(sl.k)[j * kWave + lane], ks, w);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[e]), qf[j][e], s, 0, 0, 0);
    }
    if (!full) {
      const int left = tree ? n : n_pre - 32 * i;
      uint32_t vis = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
      if (tree) vis &= anc;
      vis >>= 16 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((vis >> r) & 1u)) s[r] = -INFINITY;
    }
    // softmax, as in attend
    float tmax = __builtin_elementwise_maximum(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2)
      tmax = __builtin_elementwise_maximum(__builtin_elementwise_maximum(tmax, s[r]), s[r + 1]);
    tmax = max_xor32(tmax);
    const float m_new = tmax > m_run + a.lazy_gap ? tmax : m_run;
    const float neg = fminf(-m_new * c, __FLT_MAX__);  // (no visible key yet: see attend)
    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
    float ps = 0.f;
    float p[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = exp2_fast(__builtin_fmaf(s[r], c, neg));
    bf16x8 pf[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 pk;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x2 w = __builtin_convertvector((f32x2){p[8 * kk + 2 * j], p[8 * kk + 2 * j + 1]}, bf16x2);
        ps = __builtin_amdgcn_fdot2_f32_bf16(w, ones, ps, false);
        pk[j] = __builtin_bit_cast(uint32_t, w);
      }
      pf[kk] = __builtin_bit_cast(bf16x8, pk);
    }
    if (!full) {
      // each key's scale onto its rounded weight (the sum has the weight itself)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        u32x4 pk = __builtin_bit_cast(u32x4, pf[kk]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t* sc = sl.vs + 16 * h + 8 * kk + 2 * j;
          pk[j] = pack_bf16x2(bf16_to_f32(static_cast<uint16_t>(pk[j] & 0xFFFFu)) * q8_scale(static_cast<int>(sc[0])),
                              bf16_to_f32(static_cast<uint16_t>(pk[j] >> 16)) * q8_scale(static_cast<int>(sc[1])));
        }
        pf[kk] = __builtin_bit_cast(bf16x8, pk);
      }
    }
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
      const float alpha = exp2_fast((m_run - m_new) * c);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < HD / 32; ++db) o_acc[db] *= alpha;
    }
    l_run += ps;
    m_run = m_new;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < HD / 32; ++db) {
        const i32x2 codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)as_lds(sl.v + v_rd[kk][db]));
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t cw = static_cast<uint32_t>(codes[j]);
          w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(cw, v_scale, false));
          w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(cw, v_scale, true));
        }
        o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf[kk], o_acc[db], 0, 0, 0);
      }
    if (it + kFewSlots < mine) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this block's LDS reads are done
      load(i + kFewSlots * kFewWaves, it % kFewSlots);
    }
  }
  if ((anc & nan_keys) != 0) {
#pragma unroll
    for (int db = 0; db < HD / 32; ++db) o_acc[db] = f32x16{} + __builtin_nanf("");
  }

  // ---- the waves' results joined through LDS: O as [wave][row][HD] float,
  // 16-byte chunk c of row r at c ^ r (and the row's chunks are a multiple of
  // 16), max and sum beside.
  const float lsum = l_run + xor32(l_run);
  constexpr int kChunks = HD / 4;
  __syncthreads();  // every wave is done with its V
  if (qvalid) {
    float* o_lds = sm.o[wave][l32];
#pragma unroll
    for (int db = 0; db < HD / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 v = {o_acc[db][4 * j], o_acc[db][4 * j + 1], o_acc[db][4 * j + 2], o_acc[db][4 * j + 3]};
        *reinterpret_cast<f32x4*>(o_lds + 4 * ((db * 8 + 2 * j + h) ^ (l32 & (kChunks - 1)))) = v;
      }
    if (h == 0) {
      sm.ml[wave][l32][0] = m_run;
      sm.ml[wave][l32][1] = lsum;
    }
  }
  __syncthreads();
  // 16 lanes take a row, 8 (or 4) of its dims each: 16 rows at a time.
  constexpr int kPer = HD / 16;
  const int col = lane % 16;
  for (int r = wave * 4 + lane / 16; r < valid_rows; r += kFewWaves * 4) {
    float mw[kFewWaves], lw[kFewWaves], M = kNoMax;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      mw[w] = sm.ml[w][r][0];
      lw[w] = sm.ml[w][r][1];
      M = fmaxf(M, mw[w]);
    }
    float sum = 0.f, o[kPer] = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = lw[w] > 0.f ? exp2_fast((mw[w] - M) * c) : 0.f;
      sum += f * lw[w];
#pragma unroll
      for (int e = 0; e < kPer / 4; ++e) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(
            &sm.o[w][r][4 * ((col * (kPer / 4) + e) ^ (r & (kChunks - 1)))]);
#pragma unroll
        for (int x = 0; x < 4; ++x) o[4 * e + x] += f * v[x];
      }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    uint32_t out[kPer / 2];
    uint16_t* dst;
    if (final_out) {
#pragma unroll
      for (int e = 0; e < kPer / 2; ++e) out[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
      const int node = node_of(a, r);
      dst = a.out + ((static_cast<int64_t>(b) * a.Nmax + node) * a.Hq + g * a.G + (r - node * a.G)) * HD;
    } else {
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) top = fmaxf(top, fabsf(o[e]));
      top = fmaxf(top, dpp<0xB1>(top));  // (over the row's 16 lanes, as in wave_reduce)
      top = fmaxf(top, dpp<0x4E>(top));
      top = fmaxf(top, dpp<0x141>(top));
      top = fmaxf(top, dpp<0x140>(top)) * inv;
      const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 14, 1), 253);  // (PartRow's factor)
      const float down = inv * q8_scale(254 - ex);
#pragma unroll
      for (int e = 0; e < kPer / 2; ++e) out[e] = pack_f16x2(o[2 * e] * down, o[2 * e + 1] * down);
      const int64_t row = static_cast<int64_t>(slot_id) * kFewRows + r;
      dst = a.ws_o + row * kD;
      if (col == 0) {
        const f32x4 ml = {sum > 0.f ? M * c : -INFINITY, sum, q8_scale(ex), 0.f};
        *reinterpret_cast<f32x4*>(a.ws_ml + row * 4) = ml;
      }
    }
    if constexpr (kPer == 8)
      *reinterpret_cast<u32x4*>(dst + col * 8) = (u32x4){out[0], out[1], out[2], out[3]};
    else
      *reinterpret_cast<uint2*>(dst + col * 4) = make_uint2(out[0], out[1]);
  }
  return fw.more;
}

// kLoop: the launch's bounds allow more splits than workgroups, which the call's own
// lengths may or may not make.  (One sequence of 128 keys:
// 7.1 us a call without the loop, 7.25 with it; of 16384 keys 16.8 and 17.0.)
template <int HD, bool kPaged, bool kLoop>
__global__ void __launch_bounds__(kFewThreads, 2) attn_few_kernel(MfmaArgs a) {
  __shared__ __attribute__((aligned(16))) FewSmem<HD> sm;
  if (halted(a.status)) return;
  if constexpr (!kLoop) {
    attend_few<HD, kPaged, false>(a, sm, blockIdx.x);
  } else {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host's pass copies no structure out of an address space)
    // (The arguments are read anew for each split: kept from one to the next, they
    // and what follows from them take more scalar registers than there are, 40.4 us
    // a call where this takes 38.7.)
    typedef const __attribute__((address_space(4))) MfmaArgs KernArgs;
    KernArgs* args = (KernArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    for (int slot_id = blockIdx.x;; slot_id += gridDim.x) {
      asm volatile("" : "+s"(args));
      const MfmaArgs now = *args;
      if (!attend_few<HD, kPaged, true>(now, sm, slot_id)) return;
      __syncthreads();  // every wave is done with the results in LDS
    }
#endif
  }
}

static_assert((few::kMaxKeys + 2 * kKT + kFewRows) / 16 + 2 <= kFewBlocks, "a split's block ids fit");
static_assert(few::kKeyTile == kKT && few::kMinKeys == 32 * kFewWaves && few::kMostSplits == kMaxMergeSplits,
              "the plan's constants");

}  // namespace

hipError_t launch_attn_mfma_q8(const AttnShape& s, const AttnPlan& p, const void* q,
                               const void* k_cache, const void* v_cache, const int32_t* block_table,
                               const int32_t* prefix_len, const int32_t* parents,
                               const int32_t* n_nodes, void* out, float scale, void* workspace,
                               const KvScales& scales, const int32_t* status, hipStream_t stream) {
  MfmaArgs a = make_args(s, q, k_cache, v_cache, block_table, prefix_len, parents, n_nodes, out, scale, workspace,
                         status);
  a.ks = scales.k;
  a.vs = scales.v;
  a.scale_per_page = (s.kv_rows + s.scale_rows - 1) / s.scale_rows;
  while ((1 << a.scale_shift) < s.scale_rows) ++a.scale_shift;
  if (!p.few) return launch_tiles<true>(s, p, a, workspace, stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.row_tiles = 1;
  a.tile_rows = kFewRows;
  a.W = p.few_target;
  a.few_width = p.few_width;
  const size_t slots = static_cast<size_t>(p.few_slots) * kFewRows;
  a.ws_ml = reinterpret_cast<float*>(ws + slots * kD * 2);
  a.ws_desc = reinterpret_cast<MergeDesc*>(ws + slots * part_row_bytes(s));
  const auto launch_paged = [&](auto d, auto paged) {
    if (p.few_wide)
      hipLaunchKernelGGL((attn_few_kernel<d(), paged(), true>), dim3(p.grid), dim3(kFewThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((attn_few_kernel<d(), paged(), false>), dim3(p.grid), dim3(kFewThreads), 0, stream, a);
  };
  const auto launch_few = [&](auto d) {
    if (a.block_table) launch_paged(d, std::true_type{});
    else launch_paged(d, std::false_type{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.max_splits == 1) return e;  // one split a unit: the output is final
    hipLaunchKernelGGL((attn_split_merge_kernel<d(), false, true, true>),
                       dim3(s.B * s.Hkv, (a.G * s.Nmax + 3) / 4), dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  return s.d == 64 ? launch_few(std::integral_constant<int, 64>{}) : launch_few(std::integral_constant<int, 128>{});
}

}  // namespace ltd
