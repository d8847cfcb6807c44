// A request's sampling rules on the target's logits at every tree node:
// penalties for tokens that occurred, biases and the grammar's mask, written
// out (ltd_tree_process_logits) or reduced to each node's argmax without being
// written (ltd_tree_accept_processed); and the table of occurrences the
// penalties read (ltd_token_counts).
//
// A workgroup takes a chunk of the vocabulary (16 tokens a thread) and a few
// nodes of one sequence.  What the nodes share is set up once: which of a
// thread's tokens have a count or a bias, and, per node, which draft tokens of
// its root path lie in the chunk (a short list in LDS).  Then it streams the
// nodes' rows, with the next node's logits in flight.  Most tokens are touched
// by no rule and pass through.
//
// Bound: HBM, 4 bytes read per logit (none for a group of 4 tokens that the
// mask forbids) and, when written, 4 more.
#include <type_traits>

#include "ltd_device.hpp"
#include "ltd_launch.hpp"

#pragma clang fp contract(off)  // every step of a rule is rounded, as documented

namespace ltd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
// (a row starts at any multiple of 4 bytes; the hardware takes 16-byte accesses there)
typedef f32x4 f32x4_any __attribute__((aligned(4)));

constexpr int kVec = 4;           // 16-byte groups of a thread
constexpr int kNodesMax = 8;      // nodes of a workgroup at most
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
  int Nmax, Voc, max_bias, chunks, nodes, groups;  // nodes a workgroup, node groups a sequence
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

// kArgmax: reduce to the chunk's argmax key; else write the row.  kInPlace: out
// is logits, and groups of 4 that no rule touches are neither read nor written.
template <int kThreads, bool kArgmax, bool kInPlace>
__global__ void __launch_bounds__(kThreads) rules_kernel(RuleArgs a) {
  constexpr int kChunk = kThreads * 4 * kVec;
  __shared__ int32_t par_s[LTD_MAX_NODES], tok_s[LTD_MAX_NODES];
  __shared__ uint16_t path_s[kNodesMax][LTD_MAX_NODES];  // chunk offsets of the path's tokens
  __shared__ int path_len_s[kNodesMax];
  __shared__ int32_t bias_tok_s[LTD_MAX_BIAS];
  __shared__ float bias_val_s[LTD_MAX_BIAS];
  __shared__ float bias_sum_s[LTD_MAX_BIAS];
  __shared__ int bias_here_s;
  __shared__ unsigned long long best_s[kNodesMax];
  const int chunk = blockIdx.x % a.chunks;
  const int group = blockIdx.x / a.chunks;
  const int b = group / a.groups;
  const int i0 = group % a.groups * a.nodes;
  if (halted(a.status)) return;
  const int tid = threadIdx.x;
  const int n = min(a.n_nodes[b], a.Nmax);
  if (i0 >= n) return;
  const int i1 = min(i0 + a.nodes, n);
  const int lo = chunk * kChunk;
  const int hi = min(a.Voc, lo + kChunk);
  const int64_t seq = static_cast<int64_t>(b) * a.Nmax;
  const int words = (a.Voc + 31) / 32;

  for (int j = tid; j < n; j += kThreads) {
    par_s[j] = a.parents[seq + j];
    tok_s[j] = a.tokens[seq + j];
  }
  const int nb = a.max_bias > 0 ? min(max(a.n_bias[b], 0), a.max_bias) : 0;
  for (int j = tid; j < nb; j += kThreads) {
    bias_tok_s[j] = a.bias_tokens[static_cast<int64_t>(b) * a.max_bias + j];
    bias_val_s[j] = a.bias_values[static_cast<int64_t>(b) * a.max_bias + j];
  }
  if (tid == 0) bias_here_s = 0;
  if (tid < kNodesMax) {
    path_len_s[tid] = 0;
    best_s[tid] = 0;
  }
  Penalty pen{1.f, 0.f, 0.f};
  uint32_t cnt[kVec][4] = {};
  if (a.penalties != nullptr) {
    pen = Penalty{a.penalties[3 * b], a.penalties[3 * b + 1], a.penalties[3 * b + 2]};
    if (a.counts != nullptr) {
      const int32_t* row = a.counts + static_cast<int64_t>(b) * a.Voc;
#pragma unroll
      for (int u = 0; u < kVec; ++u)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int v = lo + (u * kThreads + tid) * 4 + c;
          if (v < hi) cnt[u][c] = static_cast<uint32_t>(row[v]);
        }
    }
  }
  __syncthreads();
  // The first entry of each biased token in this chunk gets the sum of its
  // entries, in list order.
  for (int j = tid; j < nb; j += kThreads) {
    const int t = bias_tok_s[j];
    if (t < lo || t >= hi) continue;
    float sum = bias_val_s[j];
    bool first = true;
    for (int k = 0; k < nb; ++k)
      if (bias_tok_s[k] == t && k != j) {
        if (k < j) first = false;
        else sum = sum + bias_val_s[k];
      }
    bias_sum_s[j] = sum;
    if (first) bias_here_s = 1;
  }
  // Root paths: one wave a node lists the draft tokens that lie in the chunk
  // (parents clamped below their child, so the walk ends whatever they hold).
  if (a.penalties != nullptr) {
    for (int k = tid / kWave; k < i1 - i0; k += kThreads / kWave) {
      if (tid % kWave == 0) {
        int len = 0;
        for (int j = i0 + k; j > 0;) {
          const int t = tok_s[j];
          if (t >= lo && t < hi) path_s[k][len++] = static_cast<uint16_t>(t - lo);
          j = min(max(par_s[j], 0), j - 1);
        }
        path_len_s[k] = len;
      }
    }
  }
  __syncthreads();
  float bias[kVec][4] = {};
  uint32_t biased = 0;  // bit 4u + c
  if (bias_here_s > 0) {
    for (int j = 0; j < nb; ++j) {
      const int o = bias_tok_s[j] - lo;
      if (o < 0 || o >= hi - lo || ((o >> 2) % kThreads) != tid) continue;
      const int slot = (o >> 2) / kThreads * 4 + (o & 3);
      if ((biased >> slot) & 1u) continue;  // (its first entry holds the sum)
      biased |= 1u << slot;
      const float s = bias_sum_s[j];
#pragma unroll
      for (int u = 0; u < kVec; ++u)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (slot == 4 * u + c) bias[u][c] = s;
    }
  }
  uint32_t touched = biased;
#pragma unroll
  for (int u = 0; u < kVec; ++u)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (cnt[u][c] != 0) touched |= 1u << (4 * u + c);

  for (int i = i0; i < i1; ++i) {
    const float* row = a.logits + (seq + i) * a.Voc;
    float* orow = kArgmax ? nullptr : a.out + (seq + i) * a.Voc;
    // Draft tokens of the root path: extra counts, 8 bits a token (a path has
    // at most 255 tokens below the root).
    uint32_t extra[kVec] = {};
    const int len = path_len_s[i - i0];
    for (int k = 0; k < len; ++k) {
      const int o = path_s[i - i0][k];
      if (((o >> 2) % kThreads) == tid) {
        const int u = (o >> 2) / kThreads;
#pragma unroll
        for (int w = 0; w < kVec; ++w)
          if (w == u) extra[w] += 1u << (8 * (o & 3));
      }
    }
    float vm = -INFINITY;
    int bi = 0x7FFFFFFF;
#pragma unroll
    for (int u = 0; u < kVec; ++u) {
      const int v = lo + (u * kThreads + tid) * 4;
      if (v >= hi) continue;
      uint32_t ok = 0xFu;
      if (a.mask != nullptr) ok = (a.mask[(seq + i) * words + (v >> 5)] >> (v & 31)) & 0xFu;
      const bool acts = ((touched >> (4 * u)) & 0xFu) != 0 || extra[u] != 0;
      const bool full = v + 4 <= hi;
      if (kInPlace && ok == 0xFu && !acts) continue;
      float x[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = -INFINITY;
      if (ok != 0) {
        if (full) {
          const f32x4 y = *reinterpret_cast<const f32x4_any*>(row + v);
#pragma unroll
          for (int c = 0; c < 4; ++c) x[c] = y[c];
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (v + c < hi) x[c] = row[v + c];
        }
        if (acts) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            x[c] = apply_rule(x[c], cnt[u][c] + ((extra[u] >> (8 * c)) & 0xFFu), pen,
                              (biased >> (4 * u + c)) & 1u, bias[u][c]);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (!((ok >> c) & 1u)) x[c] = -INFINITY;
      }
      if constexpr (kArgmax) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (v + c < hi && (x[c] > vm || bi == 0x7FFFFFFF)) {
            vm = x[c];
            bi = v + c;
          }
      } else if (full) {
        *reinterpret_cast<f32x4_any*>(orow + v) = (f32x4){x[0], x[1], x[2], x[3]};
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (v + c < hi) orow[v + c] = x[c];
      }
    }
    if constexpr (kArgmax) {
      uint64_t best = bi == 0x7FFFFFFF ? 0 : pack_key(vm, bi);
      best = wave_max_u64(best, tid % kWave);
      if (tid % kWave == 0) atomicMax(&best_s[i - i0], static_cast<unsigned long long>(best));
    }
  }
  if constexpr (kArgmax) {
    __syncthreads();
    if (tid < i1 - i0) a.partial[(seq + i0 + tid) * a.chunks + chunk] = best_s[tid];
  }
}

// ---- the table of occurrences

constexpr int kCountThreads = 256;

__global__ void __launch_bounds__(kCountThreads) counts_reset_kernel(int32_t* __restrict__ counts, int64_t total) {
  const int64_t v = static_cast<int64_t>(blockIdx.x) * kCountThreads + threadIdx.x;
  if (v < total) counts[v] = 0;
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
    const int64_t total = static_cast<int64_t>(B) * Voc;
    hipLaunchKernelGGL(counts_reset_kernel, dim3(static_cast<unsigned>((total + kCountThreads - 1) / kCountThreads)),
                       dim3(kCountThreads), 0, stream, counts, total);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (T > 0)
    hipLaunchKernelGGL(counts_add_kernel, dim3((T + kCountThreads - 1) / kCountThreads, B), dim3(kCountThreads), 0,
                       stream, tokens, n_tokens, T, Voc, prompt ? 1 : 0, counts);
  return hipGetLastError();
}

hipError_t launch_rules(const LogitRules& r, int B, int Nmax, int Voc, float* out, void* partial,
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
  a.nodes = 4;
  a.groups = (Nmax + a.nodes - 1) / a.nodes;
  const auto launch = [&](auto threads, auto argmax, auto in_place) {
    constexpr int kChunk = threads() * 4 * kVec;
    a.chunks = (Voc + kChunk - 1) / kChunk;
    hipLaunchKernelGGL((rules_kernel<threads(), argmax(), in_place()>),
                       dim3(static_cast<unsigned>(a.chunks) * a.groups * B), dim3(threads()), 0, stream, a);
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
