// The 8-bit KV cache's writes: appending rows (a prompt's or a draft tree's)
// and moving the accepted rows next to the prefix (arXiv 2603.01639, section
// 3.2: the candidates after the first mismatch are discarded).
//
// A scale block is scale_rows rows of one kv head, K or V.  Both kernels give a
// block to one workgroup (or part of one), which alone reads and writes its
// scale byte, so a block whose scale grows can encode its older rows again
// without any exchange with others.
//
// Append: a block's threads hold 16 dims of a row each, take the largest
// magnitude of the new rows by a reduction over the block, and encode from
// registers: the input is read once.  Bound: HBM, (elem + 1) bytes per element.
#include <type_traits>

#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "q8.hpp"
#include "q8_rows.hpp"

namespace ltd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// 16 consecutive elements as floats.
template <typename T>
struct Raw16;
template <>
struct Raw16<uint16_t> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const uint16_t* p) {
    w[0] = reinterpret_cast<const u32x4*>(p)[0];
    w[1] = reinterpret_cast<const u32x4*>(p)[1];
  }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t x = w[i >> 3][(i >> 1) & 3];
    return __uint_as_float((i & 1) ? (x & 0xFFFF0000u) : (x << 16));
  }
};
template <>
struct Raw16<float> {
  f32x4 w[4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const f32x4*>(p)[i];
  }
  __device__ __forceinline__ float get(int i) const { return w[i >> 2][i & 3]; }
};

struct AppendArgs {
  const void* x[2];      // K and V rows
  unsigned char* c[2];   // codes
  uint8_t* s[2];         // scale bytes
  const int32_t* block_table;
  const int32_t* prefix_len;
  const int32_t* n_rows;
  const int32_t* status;
  int64_t row_stride;
  int Nmax, Hkv, kv_rows, max_blocks, scale_per_page, units;  // units = blocks a sequence may touch
};

// Threads of a block of `pieces` 16-dim pieces: two a thread (one each: prompts
// of 1024 to 8192 rows in 16-row blocks 106.4 us instead of 100.9; four each in
// fp32 23.2 instead of 20.6), within a wave and a workgroup.
constexpr int unit_threads(int pieces) {
  const int t = pieces / 2 < kWave ? kWave : pieces / 2;
  return t < kThreads ? t : kThreads;
}

template <typename T, int HD, int SR>
__global__ void __launch_bounds__(kThreads) kv_append_q8_kernel(AppendArgs a) {
  constexpr int kPieces = SR * HD / 16;                       // 16-dim pieces of a block
  constexpr int kUnitThreads = unit_threads(kPieces);
  constexpr int kIter = kPieces / kUnitThreads;
  constexpr int kUnits = kThreads / kUnitThreads;             // blocks per workgroup
  constexpr int kUnitWaves = kUnitThreads / kWave;
  constexpr int kLanes = HD / 16;                             // threads of a row
  constexpr int kRowStep = kUnitThreads / kLanes;             // rows of an iteration
  __shared__ float wave_max_s[kThreads / kWave];
  if (halted(a.status)) return;
  const int per_seq = (a.units + kUnits - 1) / kUnits;
  const int b = blockIdx.x / per_seq;
  const int g = blockIdx.y >> 1, which = blockIdx.y & 1;
  const int t = threadIdx.x % kUnitThreads;
  const int unit = (blockIdx.x % per_seq) * kUnits + threadIdx.x / kUnitThreads;
  const int P = max(a.prefix_len[b], 0);
  const int n = min(a.n_rows[b], a.Nmax);
  // The unit's rows [r0, r1) of the logical cache: blocks never cross a page
  // (a page holds whole blocks), so they follow one another.
  const int r0 = append_block(P, n, unit, SR);
  const int64_t end = static_cast<int64_t>(P) + n;
  const bool work = r0 >= 0;
  const int lane = t % kLanes;
  Raw16<T> x[kIter];
  float amax = 0.f;
  // (the old scale byte is read by every thread ahead of the barrier, after
  // which one of them may replace it)
  uint8_t* scale = nullptr;
  unsigned char* rows = nullptr;  // this thread's piece of the block's first row
  int e_old = 0;
  if (work) {
    const Q8Row at = q8_row(a.block_table, b, r0, a.kv_rows, a.max_blocks);
    const int64_t head = at.page * a.Hkv + g;
    scale = a.s[which] + head * a.scale_per_page + at.row / SR;
    rows = a.c[which] + (head * a.kv_rows + at.row) * HD + lane * 16;
    if (r0 < P) e_old = *scale;
    const T* src = static_cast<const T*>(a.x[which]) + static_cast<int64_t>(b) * a.Nmax * a.row_stride +
                   g * HD + lane * 16;
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
      const int r = r0 + t / kLanes + k * kRowStep;
      if (r >= P && r < end) x[k].load(src + static_cast<int64_t>(r - P) * a.row_stride);
    }
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
      const int r = r0 + t / kLanes + k * kRowStep;
      if (r >= P && r < end) {
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(x[k].get(i)));  // (NaN is passed over)
      }
    }
  }
  amax = wave_max_dpp(amax);
  if constexpr (kUnitWaves > 1) {
    if (threadIdx.x % kWave == 0) wave_max_s[threadIdx.x / kWave] = amax;
    __syncthreads();
    const int w0 = threadIdx.x / kUnitThreads * kUnitWaves;
#pragma unroll
    for (int w = 0; w < kUnitWaves; ++w) amax = fmaxf(amax, wave_max_s[w0 + w]);
  }
  if (!work) return;
  const int e = max(q8_needed_byte(amax), e_old);  // (e_old is 0 in a block without rows that stay)
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);  // 2^(127 - e)
  const float shift = q8_shift(e_old, e);
#pragma unroll
  for (int k = 0; k < kIter; ++k) {
    const int r = r0 + t / kLanes + k * kRowStep;
    u32x4* dst = reinterpret_cast<u32x4*>(rows + static_cast<int64_t>(r - r0) * HD);
    u32x4 w;
    if (r >= P && r < end) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = q8_encode4(x[k].get(4 * j) * inv, x[k].get(4 * j + 1) * inv, x[k].get(4 * j + 2) * inv,
                          x[k].get(4 * j + 3) * inv);
      *dst = w;
    } else if (r < P && e != e_old) {
      w = *dst;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = q8_rescale4(w[j], shift);
      *dst = w;
    }
  }
  if (t == 0 && e != e_old) *scale = static_cast<uint8_t>(e);
}

struct CompactArgs {
  unsigned char* c[2];
  uint8_t* s[2];
  const int32_t* block_table;
  const int32_t* prefix_len;
  int32_t* new_prefix_len;
  const int32_t* accepted_nodes;
  const int32_t* n_accepted;
  const int32_t* status;
  int64_t layer_stride, scale_stride;
  int Nmax, Hkv, kv_rows, max_blocks, scale_per_page;
};

// As many threads as a block has pieces: most moves fill only part of one, and
// small workgroups leave room for more of them (16 sequences, 20 layers of 8 kv
// heads, 8 accepted rows, 16-row blocks: 13.4 us with 256 threads, 9.7 with 128).
constexpr int compact_threads(int hd, int sr) { return sr * hd / 16 < kThreads ? sr * hd / 16 : kThreads; }

// Compaction: a workgroup per (sequence, layer, kv head, K or V) fills the
// destination blocks one after another.  Every source of a block (row P +
// path[j], path[j] >= j) is read, with its scale byte, before the block or its
// byte is written, and lies in this block or a later one, so no source has been
// overwritten and no byte it needs has changed.
template <int HD, int SR>
__global__ void __launch_bounds__(kThreads) kv_compact_q8_kernel(CompactArgs a) {
  constexpr int kLanes = HD / 16;
  constexpr int kRowStep = compact_threads(HD, SR) / kLanes;  // rows of a pass
  constexpr int kIter = (SR + kRowStep - 1) / kRowStep;
  __shared__ int top_s;
  if (halted(a.status)) return;
  const int b = blockIdx.x;
  const int y = blockIdx.y;  // ((layer * Hkv) + g) * 2 + which
  const int which = y & 1;
  const int g = (y >> 1) % a.Hkv;
  const int layer = (y >> 1) / a.Hkv;
  const int32_t* path = a.accepted_nodes + static_cast<int64_t>(b) * a.Nmax;
  const int P = a.prefix_len[b];
  const int n = a.n_accepted[b];
  unsigned char* codes = a.c[which] + layer * a.layer_stride;
  uint8_t* scales = a.s[which] + layer * a.scale_stride;
  const int rj = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  for (int r0 = P / SR * SR; r0 < P + n; r0 += SR) {
    const Q8Row at = q8_row(a.block_table, b, r0, a.kv_rows, a.max_blocks);
    const int64_t head = at.page * a.Hkv + g;
    uint8_t* scale = scales + head * a.scale_per_page + at.row / SR;
    unsigned char* rows = codes + (head * a.kv_rows + at.row) * HD + lane * 16;
    const int e_own = *scale;
    if (threadIdx.x == 0) top_s = r0 < P ? e_own : 0;
    __syncthreads();
    u32x4 w[kIter];
    int e_src[kIter];  // 0: no row here; the row's scale byte otherwise
    bool moves[kIter];
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
      const int r = r0 + rj + k * kRowStep;
      e_src[k] = 0;
      moves[k] = false;
      if (rj + k * kRowStep < SR && r >= P && r < P + n) {
        const int pj = path[r - P];
        const Q8Row from = q8_row(a.block_table, b, P + pj, a.kv_rows, a.max_blocks);
        const int64_t fh = from.page * a.Hkv + g;
        e_src[k] = scales[fh * a.scale_per_page + from.row / SR];
        moves[k] = pj != r - P;
        w[k] = *reinterpret_cast<const u32x4*>(codes + (fh * a.kv_rows + from.row) * HD + lane * 16);
        if (lane == 0) atomicMax(&top_s, e_src[k]);
      }
    }
    __syncthreads();
    const int e = top_s;
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
      const int r = r0 + rj + k * kRowStep;
      if (rj + k * kRowStep >= SR) continue;
      u32x4* dst = reinterpret_cast<u32x4*>(rows + static_cast<int64_t>(r - r0) * HD);
      if (r < P) {  // a row that stays, of the block's own scale
        if (e == e_own) continue;
        w[k] = *dst;
        e_src[k] = e_own;
      } else if (e_src[k] == 0 || (!moves[k] && e_src[k] == e)) {
        continue;
      }
      if (e_src[k] != e) {
        const float shift = q8_shift(e_src[k], e);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[k][j] = q8_rescale4(w[k][j], shift);
      }
      *dst = w[k];
    }
    if (threadIdx.x == 0 && e != e_own) *scale = static_cast<uint8_t>(e);
    __syncthreads();  // top_s is reused
  }
  if (y == 0 && threadIdx.x == 0) a.new_prefix_len[b] = P + n;
}

// The append's data-dependent checks: one workgroup over every sequence, the
// code of the lowest failing one.
__global__ void __launch_bounds__(kThreads) validate_append_kernel(
    const int32_t* block_table, const int32_t* prefix_len, const int32_t* n_rows, int B, int Nmax,
    int kv_rows, int max_blocks, int num_blocks, int32_t* status) {
  __shared__ int best;
  if (threadIdx.x == 0) best = 0x7FFFFFFF;
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += kThreads) {
    const int n = n_rows[b], P = prefix_len[b];
    const int64_t capacity = min(
        block_table ? static_cast<int64_t>(kv_rows) * max_blocks : static_cast<int64_t>(kv_rows),
        static_cast<int64_t>(LTD_MAX_LENGTH));
    int code = 0;
    if (n < 0 || n > Nmax) {
      code = LTD_STATUS_BAD_NNODES;
    } else if (P < 0 || static_cast<int64_t>(P) + n > capacity) {
      code = LTD_STATUS_BAD_PREFIX;
    } else if (block_table && n > 0) {
      for (int j = P / kv_rows; j <= (P + n - 1) / kv_rows && code == 0; ++j) {
        const int32_t blk = block_table[static_cast<int64_t>(b) * max_blocks + j];
        if (blk < 0 || blk >= num_blocks) code = LTD_STATUS_BAD_BLOCK;
      }
    }
    if (code != 0) {
      atomicMin(&best, (b << 8) | code);
      break;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) *status = best == 0x7FFFFFFF ? 0 : (best & 0xFF);
}

// launch(head size, scale rows), as compile-time constants.
template <class Launch>
void pick_block(int d, int scale_rows, Launch launch) {
  const auto with_rows = [&](auto hd) {
    if (scale_rows == 16) launch(hd, std::integral_constant<int, 16>{});
    else if (scale_rows == 32) launch(hd, std::integral_constant<int, 32>{});
    else if (scale_rows == 64) launch(hd, std::integral_constant<int, 64>{});
    else launch(hd, std::integral_constant<int, 128>{});
  };
  if (d == 64) with_rows(std::integral_constant<int, 64>{});
  else with_rows(std::integral_constant<int, 128>{});
}

}  // namespace

hipError_t launch_validate_append(const int32_t* block_table, const int32_t* prefix_len,
                                  const int32_t* n_rows, int B, int Nmax, int kv_rows,
                                  int max_blocks, int num_blocks, int32_t* status,
                                  hipStream_t stream) {
  hipLaunchKernelGGL(validate_append_kernel, dim3(1), dim3(kThreads), 0, stream, block_table,
                     prefix_len, n_rows, B, Nmax, kv_rows, max_blocks, num_blocks, status);
  return hipGetLastError();
}

hipError_t launch_append_q8(const void* k_new, const void* v_new, int64_t row_stride,
                            void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                            const int32_t* block_table, const int32_t* prefix_len,
                            const int32_t* n_rows, int B, int Nmax, int Hkv, int d, int kv_rows,
                            int max_blocks, int scale_rows, int dtype, const int32_t* status,
                            hipStream_t stream) {
  AppendArgs a{};
  a.x[0] = k_new;
  a.x[1] = v_new;
  a.c[0] = static_cast<unsigned char*>(k_cache);
  a.c[1] = static_cast<unsigned char*>(v_cache);
  a.s[0] = k_scale;
  a.s[1] = v_scale;
  a.block_table = block_table;
  a.prefix_len = prefix_len;
  a.n_rows = n_rows;
  a.status = status;
  a.row_stride = row_stride;
  a.Nmax = Nmax;
  a.Hkv = Hkv;
  a.kv_rows = kv_rows;
  a.max_blocks = max_blocks;
  a.scale_per_page = (kv_rows + scale_rows - 1) / scale_rows;
  a.units = append_units(Nmax, scale_rows);
  pick_block(d, scale_rows, [&](auto hd, auto sr) {
    constexpr int kUnits = kThreads / unit_threads(sr() * hd() / 16);
    const dim3 grid(static_cast<unsigned>(B) * ((a.units + kUnits - 1) / kUnits), Hkv * 2);
    if (dtype == LTD_DTYPE_F32)
      hipLaunchKernelGGL((kv_append_q8_kernel<float, hd(), sr()>), grid, dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((kv_append_q8_kernel<uint16_t, hd(), sr()>), grid, dim3(kThreads), 0, stream, a);
  });
  return hipGetLastError();
}

hipError_t launch_compact_q8(void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                             const int32_t* block_table, const int32_t* prefix_len,
                             int32_t* new_prefix_len, const int32_t* accepted_nodes,
                             const int32_t* n_accepted, int B, int Nmax, int Hkv, int d,
                             int kv_rows, int max_blocks, int scale_rows, int num_layers,
                             int64_t layer_stride, int64_t scale_stride, const int32_t* status,
                             hipStream_t stream) {
  CompactArgs a{};
  a.c[0] = static_cast<unsigned char*>(k_cache);
  a.c[1] = static_cast<unsigned char*>(v_cache);
  a.s[0] = k_scale;
  a.s[1] = v_scale;
  a.block_table = block_table;
  a.prefix_len = prefix_len;
  a.new_prefix_len = new_prefix_len;
  a.accepted_nodes = accepted_nodes;
  a.n_accepted = n_accepted;
  a.status = status;
  a.layer_stride = layer_stride;
  a.scale_stride = scale_stride;
  a.Nmax = Nmax;
  a.Hkv = Hkv;
  a.kv_rows = kv_rows;
  a.max_blocks = max_blocks;
  a.scale_per_page = (kv_rows + scale_rows - 1) / scale_rows;
  const dim3 grid(B, num_layers * Hkv * 2);
  pick_block(d, scale_rows, [&](auto hd, auto sr) {
    hipLaunchKernelGGL((kv_compact_q8_kernel<hd(), sr()>), grid, dim3(compact_threads(hd(), sr())), 0, stream, a);
  });
  return hipGetLastError();
}

}  // namespace ltd
