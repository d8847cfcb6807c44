// The latent cache's writes: appending a prompt's or a draft tree's rows, and
// moving the accepted rows next to the prefix (arXiv 2603.01639, section 3.2: the
// candidates after the first mismatch are discarded).
//
// A cache row holds one token's latent part (d_latent dims, the key and value
// of every head) and its rotated part (d_rope dims, key alone).
//
// Append: a wave takes two or four rows of a sequence, whose loads all go out first.  A row's
// latent part lies across the wave, so that its mean square is a wave reduction
// over registers; two angles a lane pass through LDS to the lanes that hold the
// rotated parts.  A row is read and written once.  Bound: HBM, or the launch for a
// tree's rows.
#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "rope.hpp"

namespace ltd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kRopeDims = 64;  // d_rope
constexpr int kPairs = kRopeDims / 2;

template <typename T>
struct Piece {  // 16 bytes
  static constexpr int N = 16 / sizeof(T);
  typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
  V v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const V*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<V*>(p) = v; }
  __device__ __forceinline__ float get(int i) const { return static_cast<float>(v[i]); }
};

constexpr int kWaves = kThreads / kWave;

template <typename T, int DL, int kRowsAtOnce>
__global__ void __launch_bounds__(kThreads) latent_append_kernel(LatentAppendArgs a) {
  constexpr int kGroupRows = kWaves * kRowsAtOnce;
  constexpr int N = Piece<T>::N;
  constexpr int D = DL + kRopeDims;
  constexpr int kPieces = DL / N;                       // of the latent part
  constexpr int kIter = (kPieces + kWave - 1) / kWave;  // a lane's
  __shared__ float2 turn_s[kWaves][kRowsAtOnce][kPairs];
  if (halted(a.status)) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // The rotated parts: a lane has a piece of neighbouring pairs, or two pieces, the first
  // and the second values of its pairs.
  const int per_row = a.interleaved ? kRopeDims / N : kPairs / N;
  const int turn_row = lane / per_row, turn_piece = lane % per_row;
  const double freq = a.freq[lane % kPairs];
  const int groups = (a.Nmax + kGroupRows - 1) / kGroupRows;  // of rows, a sequence
  const uint32_t all = static_cast<uint32_t>(a.B) * groups;
  for (uint32_t group = blockIdx.x; group < all; group += gridDim.x) {
    const int b = static_cast<int>(group / groups);
    const int i0 = static_cast<int>(group % groups) * kGroupRows + wave * kRowsAtOnce;
    const int n = min(a.n_rows[b], a.Nmax), P = a.prefix_len[b];
    const int rows = min(kRowsAtOnce, n - i0);  // (the same for the wave)
    if (rows > 0) {
      const T* src = static_cast<const T*>(a.x) + (static_cast<int64_t>(b) * a.Nmax + i0) * a.x_row;
      Piece<T> c[kRowsAtOnce][kIter], r0, r1;
#pragma unroll
      for (int r = 0; r < kRowsAtOnce; ++r)
#pragma unroll
        for (int k = 0; k < kIter; ++k)
          if (r < rows && lane + k * kWave < kPieces) c[r][k].load(src + r * a.x_row + (lane + k * kWave) * N);
      const bool turns = turn_row < rows;
      if (turns) {
        r0.load(src + turn_row * a.x_row + DL + turn_piece * N);
        if (!a.interleaved) r1.load(src + turn_row * a.x_row + DL + kPairs + turn_piece * N);
      }
      // the rows' places in the cache and their angles
      T* dst[kRowsAtOnce];
#pragma unroll
      for (int r = 0; r < kRowsAtOnce; ++r)
        dst[r] = static_cast<T*>(a.cache) +
                 cache_row(a.block_table, b, 0, P + i0 + min(r, rows - 1), 1, D, a.kv_rows, a.max_blocks);
#pragma unroll
      for (int r = 0; r < kRowsAtOnce; r += kWave / kPairs) {
        const int row = r + lane / kPairs, i = i0 + min(row, rows - 1);
        const int64_t pos = static_cast<int64_t>(P) + (a.depth ? a.depth[static_cast<int64_t>(b) * a.Nmax + i] : i);
        turn_s[wave][row][lane % kPairs] = rope_turn(pos, freq, a.m);
      }
#pragma unroll
      for (int r = 0; r < kRowsAtOnce; ++r) {
        if (r >= rows) break;
        if (a.weight) {
          float ss = 0.f;
#pragma unroll
          for (int k = 0; k < kIter; ++k)
            if (lane + k * kWave < kPieces)
#pragma unroll
              for (int e = 0; e < N; ++e) ss = __builtin_fmaf(c[r][k].get(e), c[r][k].get(e), ss);
          ss = wave_sum_dpp(ss);
          const float rs = 1.f / __builtin_sqrtf(ss * (1.f / DL) + a.eps);
#pragma unroll
          for (int k = 0; k < kIter; ++k)
            if (lane + k * kWave < kPieces) {
              Piece<T> w;
              w.load(static_cast<const T*>(a.weight) + (lane + k * kWave) * N);
#pragma unroll
              for (int e = 0; e < N; ++e) c[r][k].v[e] = static_cast<T>(c[r][k].get(e) * rs * w.get(e));
            }
        }
#pragma unroll
        for (int k = 0; k < kIter; ++k)
          if (lane + k * kWave < kPieces) c[r][k].store(dst[r] + (lane + k * kWave) * N);
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      if (turns) {
        T* to = dst[0];
#pragma unroll
        for (int r = 1; r < kRowsAtOnce; ++r)
          if (turn_row == r) to = dst[r];
        const float2* t = turn_s[wave][turn_row] + turn_piece * (a.interleaved ? N / 2 : N);
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const float p0 = r0.get(2 * e), p1 = r0.get(2 * e + 1);
            r0.v[2 * e] = static_cast<T>(p0 * t[e].x - p1 * t[e].y);
            r0.v[2 * e + 1] = static_cast<T>(p1 * t[e].x + p0 * t[e].y);
          }
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float p0 = r0.get(e), p1 = r1.get(e);
            r0.v[e] = static_cast<T>(p0 * t[e].x - p1 * t[e].y);
            r1.v[e] = static_cast<T>(p1 * t[e].x + p0 * t[e].y);
          }
          r1.store(to + DL + kPairs + turn_piece * N);
        }
        r0.store(to + DL + turn_piece * N);
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // (the angles are replaced)
    }
  }
}

// Compaction: one workgroup per (sequence, layer); rows move in ascending passes
// that read all their sources before the first write.  Row j comes from P +
// path[j], path[j] >= j, so a later pass's sources lie past every destination
// already written.
constexpr int kMoves = 4;  // 16-byte pieces of a pass that a thread holds

__global__ void __launch_bounds__(kThreads) latent_compact_kernel(LatentCompactArgs a) {
  if (halted(a.status)) return;
  const int b = blockIdx.x, layer = blockIdx.y;
  const int32_t* path = a.accepted_nodes + static_cast<int64_t>(b) * a.Nmax;
  const int P = a.prefix_len[b];
  const int n = a.n_accepted[b];
  unsigned char* base = static_cast<unsigned char*>(a.cache) + layer * a.layer_stride_bytes;
  const int per_row = a.row_bytes / 16;
  const int rows = kThreads * kMoves / per_row;  // of a pass
  for (int j0 = 0; j0 < n; j0 += rows) {
    u32x4 v[kMoves];
    int64_t to[kMoves];
#pragma unroll
    for (int k = 0; k < kMoves; ++k) {
      const int e = threadIdx.x + k * kThreads;
      const int j = j0 + e / per_row, col = e % per_row;
      to[k] = -1;
      if (e / per_row < rows && j < n) {
        const int pj = path[j];
        if (pj != j) {
          const int64_t from = cache_row(a.block_table, b, 0, P + pj, 1, a.row_bytes, a.kv_rows, a.max_blocks);
          to[k] = cache_row(a.block_table, b, 0, P + j, 1, a.row_bytes, a.kv_rows, a.max_blocks) + col * 16;
          v[k] = *reinterpret_cast<const u32x4*>(base + from + col * 16);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kMoves; ++k)
      if (to[k] >= 0) *reinterpret_cast<u32x4*>(base + to[k]) = v[k];
    __syncthreads();
  }
  if (layer == 0 && threadIdx.x == 0) a.new_prefix_len[b] = P + n;
}

}  // namespace

namespace {

template <typename T, int kRowsAtOnce>
hipError_t launch_append(const LatentAppendArgs& a, int d_latent, hipStream_t stream) {
  constexpr int kGroupRows = kWaves * kRowsAtOnce;
  const int64_t groups = static_cast<int64_t>(a.B) * ((a.Nmax + kGroupRows - 1) / kGroupRows);
  const dim3 grid(static_cast<unsigned>(groups < (1 << 20) ? groups : (1 << 20)));
  if (d_latent == 512) hipLaunchKernelGGL((latent_append_kernel<T, 512, kRowsAtOnce>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((latent_append_kernel<T, 256, kRowsAtOnce>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// Rows a wave: two where that leaves fewer than eight waves a SIMD, which are not all
// filled anyhow (60 rows 3.2 us, with four 4.0), four past that (16 prompts of 1024 to
// 8192 rows 41.3 us, with two 42.8).
template <typename T>
hipError_t launch_append(const LatentAppendArgs& a, int d_latent, hipStream_t stream) {
  if (static_cast<int64_t>(a.B) * a.Nmax < 16384) return launch_append<T, 2>(a, d_latent, stream);
  return launch_append<T, 4>(a, d_latent, stream);
}

}  // namespace

hipError_t launch_latent_append(const LatentAppendArgs& a, int d_latent, int dtype, hipStream_t stream) {
  return dtype == LTD_DTYPE_F32 ? launch_append<float>(a, d_latent, stream) : launch_append<__bf16>(a, d_latent, stream);
}

hipError_t launch_latent_compact(const LatentCompactArgs& a, int B, int num_layers, hipStream_t stream) {
  hipLaunchKernelGGL(latent_compact_kernel, dim3(B, num_layers), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ltd
