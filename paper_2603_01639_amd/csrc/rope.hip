// Rotary positions of queries and keys.
//
// Pair j of a head's rotated dims (first, second) = (x0, x1) at position
// p = P_b + depth turns by the angle p * f_j:
//   y0 = m (x0 cos - x1 sin),  y1 = m (x1 cos + x0 sin).
// A workgroup takes a few rows: its first loads go out, their angles' cosines and sines
// are computed once into LDS (every head of a row shares them), and the heads are
// streamed through, one 16-byte chunk of first and one of second values a step (a
// chunk of neighbouring pairs in the interleaved layout), so every element is read
// and written once.  Bound: HBM; a tree's rows, the launch.
#include "ltd_device.hpp"
#include "ltd_launch.hpp"
#include "rope.hpp"

namespace ltd {
namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 2048;  // angles in LDS
constexpr int kAhead = 4;     // chunks a thread has in flight
constexpr int kSteps = 4;     // times that, of a workgroup's rows

template <typename T>
__device__ __forceinline__ float widen(T x);
template <>
__device__ __forceinline__ float widen<float>(float x) { return x; }
template <>
__device__ __forceinline__ float widen<__bf16>(__bf16 x) { return static_cast<float>(x); }

// N elements moved at once.
template <typename T, int N>
struct Chunk {
  T v[N];
  __device__ __forceinline__ void load(const T* p) { *this = *reinterpret_cast<const Chunk*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Chunk*>(p) = *this; }
} __attribute__((aligned(sizeof(T) * N)));

// N elements a chunk.  kInter: neighbouring pairs, all within a chunk.  kLoose: a
// chunk is one element of a half, or one pair, of any alignment (what is only
// copied goes by single elements).
template <typename T, int N, bool kInter, bool kLoose>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a) {
  __shared__ float2 turn_s[kTurns];
  if (halted(a.status)) return;
  const int half = a.rot / 2;
  const int groups = (a.Nmax + a.rows - 1) / a.rows;  // of rows, a sequence
  const int heads = a.H[0] + a.H[1];
  const int turning = kInter ? a.rot / N : half / N;  // items of a head that turn ...
  constexpr int kCopy = kLoose ? 1 : N;
  const int per_head = turning + (a.copies ? (a.d - a.rot) / kCopy : 0);  // ... and that are copied
  const uint32_t total = static_cast<uint32_t>(a.B) * groups;
  for (uint32_t group = blockIdx.x; group < total; group += gridDim.x) {
    const int b = static_cast<int>(group / groups);
    const int i0 = static_cast<int>(group % groups) * a.rows;
    const int rows = min(a.rows, min(a.n_rows[b], a.Nmax) - i0);
    if (rows <= 0) continue;  // (the same for the whole workgroup)
    const int64_t row0 = static_cast<int64_t>(b) * a.Nmax + i0;
    const int64_t P = a.prefix_len[b];
    // The thread's next item: row, head and piece, moved on without divisions.
    int r = threadIdx.x / (heads * per_head), hh = threadIdx.x / per_head % heads, p = threadIdx.x % per_head;
    Chunk<T, N> x0[kAhead], x1[kAhead];
    T* to[kAhead];
    int j0[kAhead];  // the chunk's first angle; -1: a copy; -2: none
    auto load = [&] {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        j0[u] = -2;
        if (r < rows) {
          const int which = hh >= a.H[0];
          const int h = which ? hh - a.H[0] : hh;
          const T* x = static_cast<const T*>(a.x[which]) + (row0 + r) * a.x_row[which] + h * a.x_head[which];
          int at;  // first element
          if (p < turning) {
            at = a.off + p * N;
            j0[u] = r * half + (kInter ? p * (N / 2) : p * N);
          } else {
            at = (p - turning) * kCopy;
            if (at >= a.off) at += a.rot;
            j0[u] = -1;
          }
          to[u] = static_cast<T*>(a.y[which]) + (row0 + r) * a.y_row[which] + h * a.y_head[which] + at;
          if constexpr (kLoose) {
            x0[u].v[0] = x[at];
            if (kInter && j0[u] >= 0) x0[u].v[N - 1] = x[at + 1];
            if (!kInter && j0[u] >= 0) x1[u].v[0] = x[at + half];
          } else {
            x0[u].load(x + at);
            if (!kInter && j0[u] >= 0) x1[u].load(x + at + half);
          }
          p += a.step_p;
          hh += a.step_head;
          if (p >= per_head) {
            p -= per_head;
            ++hh;
          }
          while (hh >= heads) {
            hh -= heads;
            ++r;
          }
        }
      }
    };
    load();
    for (int e = threadIdx.x; e < rows * half; e += kThreads) {
      const int row = e / half, j = e % half;
      const int64_t pos = P + (a.depth ? a.depth[row0 + row] : i0 + row);
      turn_s[e] = rope_turn(pos, a.freq[j], a.m);
    }
    __syncthreads();
    while (j0[0] != -2) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (j0[u] == -2) continue;
        if (j0[u] >= 0) {
          if constexpr (kInter) {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
              const float2 t = turn_s[j0[u] + e / 2];
              const float p0 = widen(x0[u].v[e]), p1 = widen(x0[u].v[e + 1]);
              x0[u].v[e] = static_cast<T>(p0 * t.x - p1 * t.y);
              x0[u].v[e + 1] = static_cast<T>(p1 * t.x + p0 * t.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const float2 t = turn_s[j0[u] + e];
              const float p0 = widen(x0[u].v[e]), p1 = widen(x1[u].v[e]);
              x0[u].v[e] = static_cast<T>(p0 * t.x - p1 * t.y);
              x1[u].v[e] = static_cast<T>(p1 * t.x + p0 * t.y);
            }
          }
        }
        if constexpr (kLoose) {
          to[u][0] = x0[u].v[0];
          if (kInter && j0[u] >= 0) to[u][1] = x0[u].v[N - 1];
          if (!kInter && j0[u] >= 0) to[u][half] = x1[u].v[0];
        } else {
          x0[u].store(to[u]);
          if (!kInter && j0[u] >= 0) x1[u].store(to[u] + half);
        }
      }
      load();
    }
    __syncthreads();  // the angles are replaced
  }
}

// Node counts in [0, Nmax], positions in [0, LTD_MAX_LENGTH).
__global__ void __launch_bounds__(kThreads) validate_rows_kernel(const int32_t* prefix_len,
                                                                 const int32_t* depth,
                                                                 const int32_t* n_rows, int B,
                                                                 int Nmax, int32_t* status) {
  __shared__ int best;
  if (threadIdx.x == 0) best = 0x7FFFFFFF;
  __syncthreads();
  for (int b = 0; b < B; ++b) {
    const int n = n_rows[b];
    const int64_t P = prefix_len[b];
    if (n < 0 || n > Nmax) {
      if (threadIdx.x == 0) atomicMin(&best, (b << 8) | LTD_STATUS_BAD_NNODES);
      continue;
    }
    bool bad = P < 0 || P + n > LTD_MAX_LENGTH;
    if (depth)
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const int dep = depth[static_cast<int64_t>(b) * Nmax + i];
        bad |= dep < 0 || P + dep >= LTD_MAX_LENGTH;
      }
    if (bad) atomicMin(&best, (b << 8) | LTD_STATUS_BAD_PREFIX);
  }
  __syncthreads();
  if (threadIdx.x == 0) *status = best == 0x7FFFFFFF ? 0 : (best & 0xFF);
}

template <typename T, int N, bool kLoose>
void launch_typed(RopeArgs a, hipStream_t stream) {
  const int turning = a.interleaved ? a.rot / (kLoose ? 2 : N) : a.rot / 2 / N;
  const int per_head = turning + (a.copies ? (a.d - a.rot) / (kLoose ? 1 : N) : 0);
  a.step_p = kThreads % per_head;
  a.step_head = kThreads / per_head;
  // Rows a workgroup: a few steps of every thread where there are rows for many
  // workgroups, one row otherwise.
  const int64_t all = static_cast<int64_t>(a.B) * a.Nmax;
  const int64_t row_items = static_cast<int64_t>(a.H[0] + a.H[1]) * per_head;
  int64_t rows = all < 8192 ? 1 : (kSteps * kAhead * kThreads + row_items - 1) / row_items;
  const int64_t most = kTurns / (a.rot / 2);
  a.rows = static_cast<int>(rows < most ? rows : most);
  const int64_t groups = static_cast<int64_t>(a.B) * ((a.Nmax + a.rows - 1) / a.rows);
  const int grid = static_cast<int>(groups < (1 << 20) ? groups : (1 << 20));
  if (a.interleaved)
    hipLaunchKernelGGL((rope_kernel<T, kLoose ? 2 : N, true, kLoose>), dim3(grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((rope_kernel<T, N, false, kLoose>), dim3(grid), dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_validate_rows(const int32_t* prefix_len, const int32_t* depth,
                                const int32_t* n_rows, int B, int Nmax, int32_t* status,
                                hipStream_t stream) {
  hipLaunchKernelGGL(validate_rows_kernel, dim3(1), dim3(kThreads), 0, stream, prefix_len, depth,
                     n_rows, B, Nmax, status);
  return hipGetLastError();
}

hipError_t launch_rope(RopeArgs a, int dtype, hipStream_t stream) {
  const int elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
  const int N = 16 / elem;
  // 16-byte chunks where every chunk of every row and head is aligned.
  bool wide = a.d % N == 0 && a.off % N == 0 && (a.interleaved ? a.rot : a.rot / 2) % N == 0;
  a.copies = 0;
  for (int w = 0; w < 2; ++w) {
    if (a.H[w] == 0) continue;
    wide = wide && reinterpret_cast<uintptr_t>(a.x[w]) % 16 == 0 && reinterpret_cast<uintptr_t>(a.y[w]) % 16 == 0 &&
           a.x_row[w] % N == 0 && a.x_head[w] % N == 0 && a.y_row[w] % N == 0 && a.y_head[w] % N == 0;
    if (a.x[w] != a.y[w]) a.copies = 1;  // (in place the other dims stay where they are)
  }
  if (dtype == LTD_DTYPE_F32) {
    if (wide) launch_typed<float, 4, false>(a, stream);
    else launch_typed<float, 1, true>(a, stream);
  } else {
    if (wide) launch_typed<__bf16, 8, false>(a, stream);
    else launch_typed<__bf16, 1, true>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace ltd
