// What latent attention's kernels share: their arguments, the pieces of cut units, and
// the search for a workgroup's share.
#pragma once

#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "latent_plan.hpp"
#include "mfma_tiles.hpp"

namespace ltd {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = latent::kRows;
constexpr int kRopeDims = 64;
constexpr int kAncWords = LTD_MAX_NODES / 32;  // 256 bits a node

// A row's reference maximum moves when a score passes it by 2^16: weights up to that and
// their sums have as many bits in float32 and bfloat16 as small ones, and moving it
// costs every accumulator of the row.  (At 2^8 two tiles in ten of 128 rows moved some
// row's, 1400 cycles a tile; 8 sequences of 128 heads 774 us, 650 without.)
constexpr float kLazyMax = 16.f;
constexpr float kNoMax = -__FLT_MAX__;

// A piece's row beside its O / l, which is float32 as every sum here: the maximum (log2 units)
// and the sum.  (Half the bytes, in float16 under powers of two and rounded towards 0, moved
// outputs by up to an eighth of their own rounding step: one token of 16 sequences of 128 heads
// over 1024 to 8192 keys took 48.1 us so, takes 53.8 us; 60 nodes of 16 heads over 16384 56.6 and
// 60.9; 8 sequences' trees of 128 heads are as fast.)
struct PieceRow {
  float m, l;
};
// A unit that was cut: its rows, and the workgroups that have the other pieces.
struct CutUnit {
  int b, r0, valid, last;
};

struct LatentArgs {
  LatentAttn in;
  float* ws_o;       // [2 W][128][DL]: pieces' O / l
  PieceRow* ws_row;  // [2 W][128]
  CutUnit* ws_cut;   // [W]: the cut unit that begins in a workgroup's share (valid 0: none)
  int W;         // workgroups
  float scale_log2, lazy_gap;
  latent::RowDivisor block;  // of kv_rows
};

// x, made anew: constants of rare branches, and what they and a piece's end derive from
// the thread's index, would be hoisted out of the loops into registers that these do
// not have.
template <typename T>
__device__ __forceinline__ T rare(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Where a place of the laid-out units falls.
struct Place {
  int b;
  int64_t before;  // length before sequence b
};

// Nodes and prefix of sequence b (none past the batch; what is out of range is clamped).
struct Seq {
  int n, P;
};
__device__ __forceinline__ Seq seq_of(const LatentAttn& a, int b) {
  if (b >= a.B) return Seq{0, 0};
  return Seq{min(max(a.n_nodes[b], 0), a.Nmax), max(a.prefix_len[b], 0)};
}
__device__ __forceinline__ int64_t seq_length(const LatentAttn& a, const Seq& s, const latent::Cut& c) {
  return s.n > 0 ? latent::length_of(s.P, s.n, a.Hq, c) : 0;
}

// x moved between lanes by DPP (0 where there is none to take).
template <int kCtrl, int kRowMask>
__device__ __forceinline__ int64_t dpp64(int64_t x) {
  const uint64_t u = static_cast<uint64_t>(x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), kCtrl, kRowMask, 0xF, kRowMask == 0xF);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), kCtrl, kRowMask, 0xF, kRowMask == 0xF);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t v) {  // inclusive
  v += dpp64<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += dpp64<0x112, 0xF>(v);
  v += dpp64<0x114, 0xF>(v);
  v += dpp64<0x118, 0xF>(v);
  v += dpp64<0x142, 0xA>(v);  // row_bcast 15 into rows 1 and 3
  v += dpp64<0x143, 0xC>(v);  // row_bcast 31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ int64_t read_lane(int64_t v, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), l);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint64_t>(v) >> 32), l);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// The length of all sequences' units, and the sequence that place pos(length) falls
// into (B past the end); every wave works it out by itself.  seq: sequence `lane`.
template <class Pos>
__device__ __forceinline__ Place find_place(const LatentAttn& a, const latent::Cut& c, int lane, const Seq& seq,
                                            int64_t* total_out, Pos pos) {
  const int64_t mine = seq_length(a, seq, c), upto = wave_scan(mine);
  const int64_t first = read_lane(upto, kWave - 1);
  int64_t total = first;
  for (int b0 = kWave; b0 < a.B; b0 += kWave) total += read_lane(wave_scan(seq_length(a, seq_of(a, b0 + lane), c)), kWave - 1);
  *total_out = total;
  const int64_t at = pos(total);
  if (at < first) {
    const int l = __ffsll(static_cast<long long>(__ballot(at < upto))) - 1;
    return Place{l, read_lane(upto - mine, l)};
  }
  int64_t before = first;
  for (int b0 = kWave; b0 < a.B; b0 += kWave) {
    const int64_t here = seq_length(a, seq_of(a, b0 + lane), c), past = wave_scan(here) + before;
    const uint64_t hit = __ballot(at < past);
    if (hit != 0) {
      const int l = __ffsll(static_cast<long long>(hit)) - 1;
      return Place{b0 + l, read_lane(past - here, l)};
    }
    before = read_lane(past, kWave - 1);
  }
  return Place{a.B, total};
}

// A direct load of 16 bytes a lane (lane i's land at lds + 16 i) from kOff bytes past
// p.  (The instruction's offset moves its place in LDS as well, so that is taken back.)
template <int kOff>
__device__ __forceinline__ void dma16_at(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off offset:%2"
               ::"s"(lds - kOff), "v"(p), "n"(kOff)
               : "memory");
}

// A row's block.
__device__ __forceinline__ int block_of(const LatentArgs& a, int row) {
  return static_cast<int>(__umulhi(2u * static_cast<uint32_t>(row), a.block.magic) >> a.block.shift);
}
// Its place among the cache's rows, which are counted in 32 bits: 2^31 of them pass any
// memory.
template <bool kPaged>
__device__ __forceinline__ uint32_t row_place(const LatentArgs& a, int b, int row, int32_t block) {
  return kPaged ? block * a.in.kv_rows + (row - block_of(a, row) * a.in.kv_rows) : b * a.in.kv_rows + row;
}

}  // namespace

// latent_few.hip: the kernel for up to 16 stacked rows a sequence (args: a LatentArgs).
hipError_t launch_latent_few(const void* args, int d_latent, hipStream_t stream);

}  // namespace ltd
