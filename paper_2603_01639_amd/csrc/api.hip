// The C ABI of ltd_verify (declared in ltd_verify.h): argument checks, launch
// plans and kernel dispatch.  No allocation, no synchronisation.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "ltd_launch.hpp"
#include "ltd_verify.h"
#include "runs.hpp"

namespace {

constexpr int kMaxDevices = 64;

int device_cu_count() {
  static std::once_flag once[kMaxDevices];
  static int cus[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
  std::call_once(once[dev], [dev] {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        n <= 0)
      n = 256;
    cus[dev] = n;
  });
  return cus[dev];
}

bool attn_args_ok(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix, int dtype) {
  (void)d;
  (void)dtype;
  return B >= 0 && Nmax >= 1 && Nmax <= LTD_MAX_NODES && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 &&
         max_prefix >= 0;
}

bool attn_supported(int d, int dtype) {
  return (dtype == LTD_DTYPE_F32 || dtype == LTD_DTYPE_BF16) && (d == 64 || d == 128);
}

ltd::AttnShape make_shape(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix, int kv_rows,
                          int max_blocks, int dtype) {
  return ltd::AttnShape{B, Nmax, Hq, Hkv, d, max_prefix, kv_rows, max_blocks, dtype, 0};
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// An 8-bit cache's geometry: what the kernels implement.
bool q8_supported(int d, int kv_rows, int scale_rows, bool paged) {
  return (d == 64 || d == 128) &&
         (scale_rows == 16 || scale_rows == 32 || scale_rows == 64 || scale_rows == 128) &&
         (!paged || kv_rows % scale_rows == 0);
}

ltd::AttnShape make_q8_shape(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix, int kv_rows,
                             int max_blocks, int dtype, int scale_rows) {
  ltd::AttnShape s = make_shape(B, Nmax, Hq, Hkv, d, max_prefix, kv_rows, max_blocks, dtype);
  s.scale_rows = scale_rows;
  return s;
}

}  // namespace

extern "C" {

const char* ltd_version(void) { return "ltd_verify 0.1 (gfx950)"; }

size_t ltd_tree_verify_attn_workspace_size(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix,
                                           int dtype) {
  if (!attn_args_ok(B, Nmax, Hq, Hkv, d, max_prefix, dtype) || !attn_supported(d, dtype)) return 0;
  // The largest need over the layouts: a contiguous cache, and a paged one
  // with one-row blocks (the smallest blocks shorten the split plan's splits
  // the most, and send a batch from the stream plan to the split plan).
  const ltd::AttnShape contiguous =
      make_shape(B, Nmax, Hq, Hkv, d, max_prefix, max_prefix + Nmax, 0, dtype);
  const ltd::AttnShape tiny_blocks = make_shape(B, Nmax, Hq, Hkv, d, max_prefix, 1, 1, dtype);
  const int cus = device_cu_count();
  return std::max(ltd::plan_attention(contiguous, cus).workspace_bytes,
                  ltd::plan_attention(tiny_blocks, cus).workspace_bytes);
}

int ltd_tree_verify_attn_grid(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix, int dtype,
                              int kv_rows, int paged) {
  if (!attn_args_ok(B, Nmax, Hq, Hkv, d, max_prefix, dtype) || !attn_supported(d, dtype) ||
      kv_rows < 1)
    return -1;
  const ltd::AttnShape s =
      make_shape(B, Nmax, Hq, Hkv, d, max_prefix, kv_rows, paged ? 1 : 0, dtype);
  return ltd::attention_grid(ltd::plan_attention(s, device_cu_count()));
}

int ltd_tree_verify_attn(const void* q, const void* k_cache, const void* v_cache,
                         const int32_t* block_table, const int32_t* prefix_len,
                         const int32_t* parents, const int32_t* n_nodes, void* out, int B, int Nmax,
                         int Hq, int Hkv, int d, int max_prefix, int kv_rows, int max_blocks,
                         int num_blocks, float scale, int dtype, void* workspace,
                         size_t workspace_bytes, int validate, int32_t* status, void* stream) {
  if (!attn_args_ok(B, Nmax, Hq, Hkv, d, max_prefix, dtype) || kv_rows < 1) return LTD_EINVAL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return LTD_EINVAL;
  if (!attn_supported(d, dtype)) return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!q || !k_cache || !v_cache || !prefix_len || !parents || !n_nodes || !out) return LTD_EINVAL;
  const ltd::AttnShape s = make_shape(B, Nmax, Hq, Hkv, d, max_prefix, kv_rows, max_blocks, dtype);
  const ltd::AttnPlan plan = ltd::plan_attention(s, device_cu_count());
  if (plan.workspace_bytes > 0 && (!workspace || workspace_bytes < plan.workspace_bytes))
    return LTD_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(block_table, prefix_len, parents, n_nodes, B, Nmax, max_prefix,
                                  kv_rows, max_blocks, num_blocks, true, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_attention(s, plan, q, k_cache, v_cache, block_table, prefix_len, parents,
                            n_nodes, out, scale, workspace, ltd::KvScales{},
                            validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

size_t ltd_tree_accept_workspace_size(int B, int Nmax, int Voc) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1) return 0;
  return ltd::accept_workspace_bytes(B, Nmax, Voc);
}

int ltd_tree_accept(const float* logits, const int32_t* draft_tokens, const int32_t* parents,
                    const int32_t* n_nodes, int B, int Nmax, int Voc, int32_t* pred,
                    int32_t* accepted_nodes, int32_t* out_tokens, int32_t* n_accepted,
                    void* workspace, size_t workspace_bytes, int validate, int32_t* status,
                    void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!logits || !draft_tokens || !parents || !n_nodes || !pred || !accepted_nodes ||
      !out_tokens || !n_accepted)
    return LTD_EINVAL;
  const size_t need = ltd::accept_workspace_bytes(B, Nmax, Voc);
  if (!workspace || workspace_bytes < need) return LTD_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(nullptr, nullptr, parents, n_nodes, B, Nmax, 0, 1, 0, 0, false,
                                  status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_accept(logits, draft_tokens, parents, n_nodes, B, Nmax, Voc, pred,
                         accepted_nodes, out_tokens, n_accepted, workspace,
                         validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

size_t ltd_tree_accept_noalloc_max_bytes(void) { return ltd::accept_noalloc_scratch_bytes(); }

int ltd_tree_accept_noalloc(const float* logits, const int32_t* draft_tokens,
                            const int32_t* parents, const int32_t* n_nodes, int B, int Nmax,
                            int Voc, int32_t* pred, int32_t* accepted_nodes, int32_t* out_tokens,
                            int32_t* n_accepted, int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!logits || !draft_tokens || !parents || !n_nodes || !pred || !accepted_nodes ||
      !out_tokens || !n_accepted)
    return LTD_EINVAL;
  if (ltd::accept_workspace_bytes(B, Nmax, Voc) > ltd::accept_noalloc_scratch_bytes())
    return LTD_EWORKSPACE;
  void* scratch = ltd::accept_noalloc_scratch();
  if (!scratch) return LTD_EHIP;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(nullptr, nullptr, parents, n_nodes, B, Nmax, 0, 1, 0, 0, false,
                                  status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_accept(logits, draft_tokens, parents, n_nodes, B, Nmax, Voc, pred,
                         accepted_nodes, out_tokens, n_accepted, scratch,
                         validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_kv_compact(void* k_cache, void* v_cache, const int32_t* block_table,
                   const int32_t* prefix_len, int32_t* new_prefix_len,
                   const int32_t* accepted_nodes, const int32_t* n_accepted, int B, int Nmax,
                   int Hkv, int d, int kv_rows, int max_blocks, int num_blocks, int num_layers,
                   int64_t layer_stride_elems, int dtype, int validate, int32_t* status,
                   void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Hkv < 1 || d < 1 || kv_rows < 1 ||
      num_layers < 1 || layer_stride_elems < 0)
    return LTD_EINVAL;
  if (dtype != LTD_DTYPE_F32 && dtype != LTD_DTYPE_BF16) return LTD_EUNSUPPORTED;
  const int elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
  const int row_bytes = d * elem;
  if (row_bytes % 16 != 0 || row_bytes > 16 * 256) return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!k_cache || !v_cache || !prefix_len || !new_prefix_len || !accepted_nodes || !n_accepted)
    return LTD_EINVAL;
  if (new_prefix_len == prefix_len) return LTD_EINVAL;
  if (num_layers > 1 && layer_stride_elems == 0) return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_path(block_table, prefix_len, accepted_nodes, n_accepted, B, Nmax,
                                  kv_rows, max_blocks, num_blocks, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_compact(k_cache, v_cache, block_table, prefix_len, new_prefix_len,
                          accepted_nodes, n_accepted, B, Nmax, Hkv, row_bytes, kv_rows, max_blocks,
                          num_layers, layer_stride_elems * elem, validate ? status : nullptr,
                          st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_select_candidates(const float* scores, const int32_t* pool_parents,
                          const int32_t* pool_tokens, const int32_t* pool_size,
                          const int32_t* n_select, int B, int Vpool, int Nmax, int32_t* selected,
                          int32_t* parents, int32_t* tokens, int32_t* depth, int32_t* n_nodes,
                          int validate, int32_t* status, void* stream) {
  if (B < 0 || Vpool < 1 || Vpool > LTD_MAX_POOL || Nmax < 1 || Nmax > LTD_MAX_NODES)
    return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!scores || !pool_parents || !pool_tokens || !pool_size || !n_select || !parents ||
      !tokens || !n_nodes)
    return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_pool(scores, pool_parents, pool_size, n_select, B, Vpool, Nmax,
                                  status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_select(scores, pool_parents, pool_tokens, pool_size, n_select, B, Vpool, Nmax,
                         selected, parents, tokens, depth, n_nodes, validate ? status : nullptr,
                         st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

size_t ltd_tree_accept_sampling_workspace_size(int B, int Nmax, int Voc) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1 ||
      ltd::sampling_chunks(Voc) > LTD_SAMPLING_MAX_CHUNKS)
    return 0;
  return ltd::sampling_workspace_bytes(B, Nmax, Voc);
}

int ltd_tree_accept_sampling(const float* logits, const float* draft_probs,
                             const int32_t* draft_tokens, const int32_t* parents,
                             const int32_t* n_nodes, const float* uniforms, int B, int Nmax,
                             int Voc, float temperature, int32_t* accepted_nodes,
                             int32_t* out_tokens, int32_t* n_accepted, void* workspace,
                             size_t workspace_bytes, int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1 ||
      ltd::sampling_chunks(Voc) > LTD_SAMPLING_MAX_CHUNKS || !(temperature > 0.f) ||
      !std::isfinite(temperature))
    return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!logits || !draft_probs || !draft_tokens || !parents || !n_nodes || !uniforms ||
      !accepted_nodes || !out_tokens || !n_accepted)
    return LTD_EINVAL;
  if (!workspace || workspace_bytes < ltd::sampling_workspace_bytes(B, Nmax, Voc))
    return LTD_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(nullptr, nullptr, parents, n_nodes, B, Nmax, 0, 1, 0, 0, false,
                                  status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_sampling(logits, draft_probs, draft_tokens, parents, n_nodes, uniforms, B, Nmax,
                           Voc, temperature, accepted_nodes, out_tokens, n_accepted, workspace,
                           validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

namespace {
bool expand_args_ok(int B, int F, int Voc, int W) {
  return B >= 0 && F >= 1 && W >= 1 && W <= LTD_EXPAND_MAX_W && Voc >= W &&
         ltd::expand_chunks(Voc) <= LTD_EXPAND_MAX_CHUNKS && F * W <= LTD_EXPAND_MAX_CHILDREN;
}
}  // namespace

size_t ltd_draft_expand_workspace_size(int B, int F, int Voc, int W) {
  if (!expand_args_ok(B, F, Voc, W)) return 0;
  return ltd::expand_workspace_bytes(B, F, Voc, W);
}

int ltd_draft_expand(const float* logits, const int32_t* frontier, int B, int F, int Voc, int W,
                     int W_next, float* scores, int32_t* pool_parents, int32_t* pool_tokens,
                     int32_t* pool_size, int Vpool, int32_t* new_frontier, void* workspace,
                     size_t workspace_bytes, int validate, int32_t* status, void* stream) {
  if (Voc < 1 || F < 1 || W < 1 || F > LTD_EXPAND_MAX_CHILDREN || !expand_args_ok(B, F, Voc, W) ||
      W_next < 1 || W_next > F * W || Vpool < 1)
    return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!logits || !frontier || !scores || !pool_parents || !pool_tokens || !pool_size ||
      !new_frontier)
    return LTD_EINVAL;
  if (!workspace || workspace_bytes < ltd::expand_workspace_bytes(B, F, Voc, W))
    return LTD_EWORKSPACE;
  if (ltd::launch_expand(logits, frontier, B, F, Voc, W, W_next, scores, pool_parents,
                         pool_tokens, pool_size, Vpool, new_frontier, workspace, status,
                         validate != 0, static_cast<hipStream_t>(stream)) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

size_t ltd_policy_workspace_size(int B, int h1, int h2) {
  if (B < 0 || h1 < 1 || h1 > LTD_POLICY_MAX_HIDDEN || h2 < 0 || h2 > LTD_POLICY_MAX_HIDDEN)
    return 0;
  return ltd::policy_workspace_bytes(B, h1, h2);
}

int ltd_policy_forward(int layout, const float* scores, const int32_t* pool_size, int Vpool,
                       const int32_t* depth, const int32_t* ctx_len, float pad, int B, int in_dim,
                       const float* w1, const float* b1, int h1, const float* w2, const float* b2,
                       int h2, const float* wo, const float* bo, int n_out, int action_offset,
                       int action_scale, float* logits, int32_t* action, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if ((layout != LTD_POLICY_SIZE && layout != LTD_POLICY_DEPTH) || B < 0 || Vpool < 1 ||
      in_dim < 3 || in_dim > LTD_POLICY_MAX_IN || h1 < 1 || h1 > LTD_POLICY_MAX_HIDDEN || h2 < 0 ||
      h2 > LTD_POLICY_MAX_HIDDEN || n_out < 1 || n_out > LTD_POLICY_MAX_OUT)
    return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!scores || !pool_size || !depth || !ctx_len || !w1 || !b1 || !wo || !bo || !logits ||
      !action || (h2 > 0 && (!w2 || !b2)))
    return LTD_EINVAL;
  if (!workspace || workspace_bytes < ltd::policy_workspace_bytes(B, h1, h2))
    return LTD_EWORKSPACE;
  if (ltd::launch_policy(layout, scores, pool_size, Vpool, depth, ctx_len, pad, B, in_dim, w1, b1,
                         h1, w2, b2, h2, wo, bo, n_out, action_offset, action_scale, logits, action,
                         workspace, static_cast<hipStream_t>(stream)) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_kv_append_q8(const void* k_new, const void* v_new, int64_t new_row_stride, void* k_cache,
                     void* v_cache, uint8_t* k_scale, uint8_t* v_scale, const int32_t* block_table,
                     const int32_t* prefix_len, const int32_t* n_rows, int B, int Nmax, int Hkv,
                     int d, int kv_rows, int max_blocks, int num_blocks, int scale_rows, int dtype,
                     int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Hkv < 1 || d < 1 || kv_rows < 1) return LTD_EINVAL;
  if (dtype != LTD_DTYPE_F32 && dtype != LTD_DTYPE_BF16) return LTD_EUNSUPPORTED;
  if (!q8_supported(d, kv_rows, scale_rows, block_table != nullptr)) return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (Nmax > LTD_MAX_LENGTH) return LTD_EUNSUPPORTED;
  if (new_row_stride < static_cast<int64_t>(Hkv) * d) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !k_scale || !v_scale || !prefix_len || !n_rows)
    return LTD_EINVAL;
  const int64_t row_bytes = new_row_stride * (dtype == LTD_DTYPE_F32 ? 4 : 2);
  if (!aligned16(k_new) || !aligned16(v_new) || row_bytes % 16 != 0 || !aligned16(k_cache) ||
      !aligned16(v_cache))
    return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_append(block_table, prefix_len, n_rows, B, Nmax, kv_rows, max_blocks,
                                    num_blocks, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_append_q8(k_new, v_new, new_row_stride, k_cache, v_cache, k_scale, v_scale,
                            block_table, prefix_len, n_rows, B, Nmax, Hkv, d, kv_rows, max_blocks,
                            scale_rows, dtype, validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

size_t ltd_tree_verify_attn_q8_workspace_size(int B, int Nmax, int Hq, int Hkv, int d,
                                              int max_prefix, int dtype) {
  if (!attn_args_ok(B, Nmax, Hq, Hkv, d, max_prefix, dtype) || !attn_supported(d, dtype) ||
      max_prefix > LTD_MAX_LENGTH)
    return 0;
  // The largest need over the layouts, as for a 16-bit cache; an 8-bit one's
  // smallest blocks hold 16 rows.
  const int cus = device_cu_count();
  const ltd::AttnShape contiguous =
      make_q8_shape(B, Nmax, Hq, Hkv, d, max_prefix, max_prefix + Nmax, 0, dtype, 16);
  const ltd::AttnShape small_blocks =
      make_q8_shape(B, Nmax, Hq, Hkv, d, max_prefix, 16, 1, dtype, 16);
  return std::max(ltd::plan_attention(contiguous, cus).workspace_bytes,
                  ltd::plan_attention(small_blocks, cus).workspace_bytes);
}

int ltd_tree_verify_attn_q8(const void* q, const void* k_cache, const void* v_cache,
                            const uint8_t* k_scale, const uint8_t* v_scale,
                            const int32_t* block_table, const int32_t* prefix_len,
                            const int32_t* parents, const int32_t* n_nodes, void* out, int B,
                            int Nmax, int Hq, int Hkv, int d, int max_prefix, int kv_rows,
                            int max_blocks, int num_blocks, int scale_rows, float scale, int dtype,
                            void* workspace, size_t workspace_bytes, int validate, int32_t* status,
                            void* stream) {
  if (!attn_args_ok(B, Nmax, Hq, Hkv, d, max_prefix, dtype) || kv_rows < 1) return LTD_EINVAL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return LTD_EINVAL;
  if (!attn_supported(d, dtype) || !q8_supported(d, kv_rows, scale_rows, block_table != nullptr) ||
      max_prefix > LTD_MAX_LENGTH)
    return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!q || !k_cache || !v_cache || !k_scale || !v_scale || !prefix_len || !parents || !n_nodes ||
      !out)
    return LTD_EINVAL;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out))
    return LTD_EINVAL;
  const ltd::AttnShape s = make_q8_shape(B, Nmax, Hq, Hkv, d, max_prefix, kv_rows,
                                         block_table ? max_blocks : 0, dtype, scale_rows);
  const ltd::AttnPlan plan = ltd::plan_attention(s, device_cu_count());
  if (plan.workspace_bytes > 0 &&
      (!workspace || !aligned16(workspace) || workspace_bytes < plan.workspace_bytes))
    return LTD_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(block_table, prefix_len, parents, n_nodes, B, Nmax, max_prefix,
                                  kv_rows, max_blocks, num_blocks, true, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_attention(s, plan, q, k_cache, v_cache, block_table, prefix_len, parents,
                            n_nodes, out, scale, workspace, ltd::KvScales{k_scale, v_scale},
                            validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_kv_compact_q8(void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                      const int32_t* block_table, const int32_t* prefix_len,
                      int32_t* new_prefix_len, const int32_t* accepted_nodes,
                      const int32_t* n_accepted, int B, int Nmax, int Hkv, int d, int kv_rows,
                      int max_blocks, int num_blocks, int scale_rows, int num_layers,
                      int64_t layer_stride_elems, int64_t scale_stride_elems, int validate,
                      int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Hkv < 1 || d < 1 || kv_rows < 1 ||
      num_layers < 1 || layer_stride_elems < 0 || scale_stride_elems < 0)
    return LTD_EINVAL;
  if (!q8_supported(d, kv_rows, scale_rows, block_table != nullptr)) return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !prefix_len || !new_prefix_len ||
      !accepted_nodes || !n_accepted)
    return LTD_EINVAL;
  if (new_prefix_len == prefix_len) return LTD_EINVAL;
  if (num_layers > 1 && (layer_stride_elems == 0 || scale_stride_elems == 0)) return LTD_EINVAL;
  if (!aligned16(k_cache) || !aligned16(v_cache) ||
      (num_layers > 1 && layer_stride_elems % 16 != 0))
    return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_path(block_table, prefix_len, accepted_nodes, n_accepted, B, Nmax,
                                  kv_rows, max_blocks, num_blocks, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_compact_q8(k_cache, v_cache, k_scale, v_scale, block_table, prefix_len,
                             new_prefix_len, accepted_nodes, n_accepted, B, Nmax, Hkv, d, kv_rows,
                             max_blocks, scale_rows, num_layers, layer_stride_elems,
                             scale_stride_elems, validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_token_counts(const int32_t* tokens, const int32_t* n_tokens, int B, int T, int Voc,
                     int prompt, int reset, int32_t* counts, void* stream) {
  if (B < 0 || T < 0 || Voc < 1) return LTD_EINVAL;
  if (T > LTD_MAX_LENGTH || Voc > LTD_MAX_LENGTH) return LTD_EUNSUPPORTED;
  if (B == 0) return LTD_OK;
  if (!counts || (T > 0 && (!tokens || !n_tokens))) return LTD_EINVAL;
  if (ltd::launch_token_counts(tokens, n_tokens, B, T, Voc, prompt != 0, reset != 0, counts,
                               static_cast<hipStream_t>(stream)) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

namespace {
// The scalar and pointer checks of a call with sampling rules (LTD_OK, or the
// code to return); the caller has dealt with an empty batch.
int rules_ok(const ltd::LogitRules& r) {
  if (!r.logits || !r.tokens || !r.parents || !r.n_nodes) return LTD_EINVAL;
  if (r.max_bias > 0 && (!r.bias_tokens || !r.bias_values || !r.n_bias)) return LTD_EINVAL;
  return LTD_OK;
}
}  // namespace

int ltd_tree_process_logits(const float* logits, const int32_t* draft_tokens,
                            const int32_t* parents, const int32_t* n_nodes, const int32_t* counts,
                            const float* penalties, const int32_t* bias_tokens,
                            const float* bias_values, const int32_t* n_bias, const uint32_t* mask,
                            int B, int Nmax, int Voc, int max_bias, float* out, int validate,
                            int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1 || max_bias < 0 ||
      max_bias > LTD_MAX_BIAS)
    return LTD_EINVAL;
  if (Voc > LTD_MAX_LENGTH) return LTD_EUNSUPPORTED;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  const ltd::LogitRules r{logits,      draft_tokens, parents, n_nodes, counts, penalties,
                          bias_tokens, bias_values,  n_bias,  mask,    max_bias};
  const int rc = rules_ok(r);
  if (rc != LTD_OK) return rc;
  if (!out) return LTD_EINVAL;
  const uintptr_t in_at = reinterpret_cast<uintptr_t>(logits), out_at = reinterpret_cast<uintptr_t>(out);
  if (in_at != out_at && (in_at < out_at ? out_at - in_at : in_at - out_at) / sizeof(float) <
                             static_cast<uint64_t>(B) * Nmax * Voc)
    return LTD_EINVAL;  // (a workgroup would read rows that another has written)
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_rules(parents, n_nodes, penalties, n_bias, B, Nmax, max_bias, status,
                                   st) != hipSuccess)
      return LTD_EHIP;
  }
  if (ltd::launch_rules(r, B, Nmax, Voc, out, nullptr, device_cu_count(),
                        validate ? status : nullptr, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

int ltd_tree_accept_processed(const float* logits, const int32_t* draft_tokens,
                              const int32_t* parents, const int32_t* n_nodes,
                              const int32_t* counts, const float* penalties,
                              const int32_t* bias_tokens, const float* bias_values,
                              const int32_t* n_bias, const uint32_t* mask, int B, int Nmax,
                              int Voc, int max_bias, int32_t* pred, int32_t* accepted_nodes,
                              int32_t* out_tokens, int32_t* n_accepted, void* workspace,
                              size_t workspace_bytes, int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || Voc < 1 || max_bias < 0 ||
      max_bias > LTD_MAX_BIAS)
    return LTD_EINVAL;
  if (Voc > LTD_MAX_LENGTH) return LTD_EUNSUPPORTED;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  const ltd::LogitRules r{logits,      draft_tokens, parents, n_nodes, counts, penalties,
                          bias_tokens, bias_values,  n_bias,  mask,    max_bias};
  const int rc = rules_ok(r);
  if (rc != LTD_OK) return rc;
  if (!pred || !accepted_nodes || !out_tokens || !n_accepted) return LTD_EINVAL;
  if (!workspace || workspace_bytes < ltd::accept_workspace_bytes(B, Nmax, Voc))
    return LTD_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_rules(parents, n_nodes, penalties, n_bias, B, Nmax, max_bias, status,
                                   st) != hipSuccess)
      return LTD_EHIP;
  }
  const int32_t* halt = validate ? status : nullptr;
  if (ltd::launch_rules(r, B, Nmax, Voc, nullptr, workspace, device_cu_count(), halt, st) !=
      hipSuccess)
    return LTD_EHIP;
  if (ltd::launch_accept_scan(workspace, draft_tokens, parents, n_nodes, B, Nmax, Voc, pred,
                              accepted_nodes, out_tokens, n_accepted, halt, st) != hipSuccess)
    return LTD_EHIP;
  return LTD_OK;
}

namespace {

bool dtype_known(int dtype) { return dtype == LTD_DTYPE_F32 || dtype == LTD_DTYPE_BF16; }
bool latent_supported(int d_latent, int d_rope) {
  return (d_latent == 256 || d_latent == 512) && d_rope == LTD_LATENT_ROPE;
}

}  // namespace

namespace {
// Whether the heads of `rows` rows lie apart: whole rows one after another, or whole heads.
bool heads_apart(int64_t rows, int64_t heads, int d, int64_t row, int64_t head) {
  if (row < 0 || head < 0) return false;
  const bool inner = heads == 1 || head >= d, outer = rows == 1 || row >= d;
  return inner && outer &&
         (rows == 1 || heads == 1 || row >= static_cast<__int128>(heads - 1) * head + d ||
          head >= static_cast<__int128>(rows - 1) * row + d);
}

// The bytes from a tensor's first element to its last one's end: `rows` rows of `heads` runs
// of d elements.
struct Span {
  __int128 from, to;
};
Span span_of(const void* p, int64_t rows, int64_t row, int64_t heads, int64_t head, int d, int elem) {
  const __int128 base = static_cast<__int128>(reinterpret_cast<uintptr_t>(p));
  const __int128 by_row = static_cast<__int128>(rows - 1) * row, by_head = static_cast<__int128>(heads - 1) * head;
  const __int128 low = (by_row < 0 ? by_row : 0) + (by_head < 0 ? by_head : 0);
  const __int128 high = (by_row > 0 ? by_row : 0) + (by_head > 0 ? by_head : 0) + d;
  return {base + low * elem, base + high * elem};
}
bool meet(const Span& x, const Span& y) { return x.from < y.to && y.from < x.to; }
}  // namespace

int ltd_tree_rope(const void* q, int64_t q_row_stride, int64_t q_head_stride, void* q_out,
                  int64_t q_out_row_stride, int64_t q_out_head_stride, const void* k,
                  int64_t k_row_stride, int64_t k_head_stride, void* k_out,
                  int64_t k_out_row_stride, int64_t k_out_head_stride, const double* inv_freq,
                  const int32_t* prefix_len, const int32_t* depth, const int32_t* n_rows, int B,
                  int Nmax, int Hq, int Hk, int d, int rot_offset, int rot_dim, int interleaved,
                  float mscale, int dtype, int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || Hq < 1 || Hk < 0 || d < 1 || rot_dim < 2 || rot_dim % 2 != 0 ||
      rot_offset < 0 || static_cast<int64_t>(rot_offset) + rot_dim > d || !std::isfinite(mscale))
    return LTD_EINVAL;
  if (!dtype_known(dtype) || d > LTD_ROPE_MAX_DIM || Nmax > LTD_MAX_LENGTH ||
      (static_cast<int64_t>(Hq) + Hk) * d > (1 << 24) || static_cast<int64_t>(B) * Nmax >= INT32_MAX)
    return LTD_EUNSUPPORTED;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!q || !q_out || (Hk > 0 && (!k || !k_out)) || !inv_freq || !prefix_len || !n_rows)
    return LTD_EINVAL;
  // (in place means the same places)
  if (q == q_out && (q_row_stride != q_out_row_stride || q_head_stride != q_out_head_stride))
    return LTD_EINVAL;
  if (Hk > 0 && k == k_out && (k_row_stride != k_out_row_stride || k_head_stride != k_out_head_stride))
    return LTD_EINVAL;
  const int64_t rows = static_cast<int64_t>(B) * Nmax;
  if (!heads_apart(rows, Hq, d, q_out_row_stride, q_out_head_stride) ||
      (Hk > 0 && !heads_apart(rows, Hk, d, k_out_row_stride, k_out_head_stride)))
    return LTD_EINVAL;
  // (workgroups write heads at times when others still read theirs)
  const auto runs = [&](const void* p, int64_t row, int H, int64_t head) {
    const int64_t elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
    return ltd::Runs{reinterpret_cast<uintptr_t>(p), rows, static_cast<ltd::Wide>(row) * elem, H, static_cast<ltd::Wide>(head) * elem, d * elem};
  };
  const ltd::Runs q_in = runs(q, q_row_stride, Hq, q_head_stride), q_to = runs(q_out, q_out_row_stride, Hq, q_out_head_stride);
  if (q != q_out && ltd::runs_meet(q_in, q_to)) return LTD_EINVAL;
  if (Hk > 0) {
    const ltd::Runs k_in = runs(k, k_row_stride, Hk, k_head_stride), k_to = runs(k_out, k_out_row_stride, Hk, k_out_head_stride);
    if ((k != k_out && ltd::runs_meet(k_in, k_to)) || ltd::runs_meet(q_to, k_in) || ltd::runs_meet(k_to, q_in) ||
        ltd::runs_meet(q_to, k_to))
      return LTD_EINVAL;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_rows(prefix_len, depth, n_rows, B, Nmax, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  ltd::RopeArgs a{};
  a.x[0] = q;
  a.x[1] = k;
  a.y[0] = q_out;
  a.y[1] = k_out;
  a.x_row[0] = q_row_stride;
  a.x_row[1] = k_row_stride;
  a.x_head[0] = q_head_stride;
  a.x_head[1] = k_head_stride;
  a.y_row[0] = q_out_row_stride;
  a.y_row[1] = k_out_row_stride;
  a.y_head[0] = q_out_head_stride;
  a.y_head[1] = k_out_head_stride;
  a.H[0] = Hq;
  a.H[1] = Hk;
  a.freq = inv_freq;
  a.prefix_len = prefix_len;
  a.depth = depth;
  a.n_rows = n_rows;
  a.status = validate ? status : nullptr;
  a.B = B;
  a.Nmax = Nmax;
  a.d = d;
  a.off = rot_offset;
  a.rot = rot_dim;
  a.interleaved = interleaved != 0;
  a.m = mscale;
  return ltd::launch_rope(a, dtype, st) == hipSuccess ? LTD_OK : LTD_EHIP;
}

int ltd_latent_append(const void* kv_new, int64_t new_row_stride, const void* norm_weight,
                      float norm_eps, const double* inv_freq, int interleaved, float mscale,
                      void* cache, const int32_t* block_table, const int32_t* prefix_len,
                      const int32_t* depth, const int32_t* n_rows, int B, int Nmax, int d_latent,
                      int d_rope, int kv_rows, int max_blocks, int num_blocks, int dtype,
                      int validate, int32_t* status, void* stream) {
  if (B < 0 || Nmax < 1 || kv_rows < 1 || !(norm_eps >= 0.f) || !std::isfinite(norm_eps) ||
      !std::isfinite(mscale))
    return LTD_EINVAL;
  if (!dtype_known(dtype) || !latent_supported(d_latent, d_rope) || Nmax > LTD_MAX_LENGTH ||
      static_cast<int64_t>(B) * Nmax >= INT32_MAX)
    return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (new_row_stride < d_latent + d_rope) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!kv_new || !inv_freq || !cache || !prefix_len || !n_rows) return LTD_EINVAL;
  if (!aligned16(kv_new) || new_row_stride * (dtype == LTD_DTYPE_F32 ? 4 : 2) % 16 != 0 ||
      !aligned16(cache) || !aligned16(norm_weight))
    return LTD_EINVAL;
  const int D = d_latent + d_rope, elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
  if (meet(span_of(kv_new, static_cast<int64_t>(B) * Nmax, new_row_stride, 1, 0, D, elem),
           span_of(cache, static_cast<int64_t>(block_table ? num_blocks : B) * kv_rows, D, 1, 0, D, elem)))
    return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_append(block_table, prefix_len, n_rows, B, Nmax, kv_rows, max_blocks,
                                    num_blocks, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  const ltd::LatentAppendArgs a{kv_new, new_row_stride, norm_weight, inv_freq, cache, block_table, prefix_len, depth,
                                n_rows, validate ? status : nullptr, B, Nmax, kv_rows, max_blocks,
                                interleaved != 0, mscale, norm_eps};
  return ltd::launch_latent_append(a, d_latent, dtype, st) == hipSuccess ? LTD_OK : LTD_EHIP;
}

namespace {
bool latent_attn_args_ok(int B, int Nmax, int Hq, int max_prefix) {
  return B >= 0 && Nmax >= 1 && Nmax <= LTD_MAX_NODES && Hq >= 1 && max_prefix >= 0;
}
}  // namespace

size_t ltd_tree_verify_attn_latent_workspace_size(int B, int Nmax, int Hq, int d_latent,
                                                  int d_rope, int max_prefix, int dtype) {
  if (!latent_attn_args_ok(B, Nmax, Hq, max_prefix) || !dtype_known(dtype) ||
      !latent_supported(d_latent, d_rope) || max_prefix > LTD_MAX_LENGTH || Hq > LTD_LATENT_MAX_HEADS)
    return 0;
  ltd::LatentAttn s{};
  s.B = B;
  s.Nmax = Nmax;
  s.Hq = Hq;
  s.max_prefix = max_prefix;
  return ltd::latent_attn_workspace_bytes(s, d_latent, dtype, device_cu_count());
}

int ltd_tree_verify_attn_latent(const void* q_latent, int64_t ql_row_stride,
                                int64_t ql_head_stride, const void* q_rope, int64_t qr_row_stride,
                                int64_t qr_head_stride, const void* cache,
                                const int32_t* block_table, const int32_t* prefix_len,
                                const int32_t* parents, const int32_t* n_nodes, void* out, int B,
                                int Nmax, int Hq, int d_latent, int d_rope, int max_prefix,
                                int kv_rows, int max_blocks, int num_blocks, float scale,
                                int dtype, void* workspace, size_t workspace_bytes, int validate,
                                int32_t* status, void* stream) {
  if (!latent_attn_args_ok(B, Nmax, Hq, max_prefix) || kv_rows < 1) return LTD_EINVAL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return LTD_EINVAL;
  if (!dtype_known(dtype) || !latent_supported(d_latent, d_rope) || max_prefix > LTD_MAX_LENGTH ||
      Hq > LTD_LATENT_MAX_HEADS || (dtype == LTD_DTYPE_F32 && B > 65535))
    return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!q_latent || !q_rope || !cache || !prefix_len || !parents || !n_nodes || !out)
    return LTD_EINVAL;
  if (!aligned16(cache) || !aligned16(out)) return LTD_EINVAL;
  if (dtype == LTD_DTYPE_BF16 &&
      (!aligned16(q_latent) || !aligned16(q_rope) || ql_row_stride % 8 != 0 ||
       ql_head_stride % 8 != 0 || qr_row_stride % 8 != 0 || qr_head_stride % 8 != 0))
    return LTD_EINVAL;
  const ltd::LatentAttn s{q_latent, q_rope, ql_row_stride, ql_head_stride, qr_row_stride, qr_head_stride, cache,
                          block_table, prefix_len, parents, n_nodes, out, validate ? status : nullptr, B, Nmax, Hq,
                          max_prefix, kv_rows, max_blocks, scale};
  const int cus = device_cu_count();
  const size_t need = ltd::latent_attn_workspace_bytes(s, d_latent, dtype, cus);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return LTD_EWORKSPACE;
  // (several workgroups read a row's queries, at times when others have their outputs)
  const int64_t rows = static_cast<int64_t>(B) * Nmax;
  const int elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
  const Span to = span_of(out, rows, static_cast<int64_t>(Hq) * d_latent, Hq, d_latent, d_latent, elem);
  if (meet(to, span_of(q_latent, rows, ql_row_stride, Hq, ql_head_stride, d_latent, elem)) ||
      meet(to, span_of(q_rope, rows, qr_row_stride, Hq, qr_head_stride, d_rope, elem)))
    return LTD_EINVAL;
  // (nor may outputs or pieces be written where keys, queries or each other lie)
  const int D = d_latent + d_rope;
  const Span keys = span_of(cache, static_cast<int64_t>(block_table ? num_blocks : B) * kv_rows, D, 1, 0, D, elem);
  if (meet(to, keys)) return LTD_EINVAL;
  if (need > 0) {
    const __int128 at = static_cast<__int128>(reinterpret_cast<uintptr_t>(workspace));
    const Span pieces{at, at + need};
    if (meet(pieces, to) || meet(pieces, keys) || meet(pieces, span_of(q_latent, rows, ql_row_stride, Hq, ql_head_stride, d_latent, elem)) ||
        meet(pieces, span_of(q_rope, rows, qr_row_stride, Hq, qr_head_stride, d_rope, elem)))
      return LTD_EINVAL;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_tree(block_table, prefix_len, parents, n_nodes, B, Nmax, max_prefix,
                                  kv_rows, max_blocks, num_blocks, true, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  return ltd::launch_latent_attn(s, d_latent, dtype, workspace, cus, st) == hipSuccess ? LTD_OK : LTD_EHIP;
}

int ltd_latent_compact(void* cache, const int32_t* block_table, const int32_t* prefix_len,
                       int32_t* new_prefix_len, const int32_t* accepted_nodes,
                       const int32_t* n_accepted, int B, int Nmax, int d_latent, int d_rope,
                       int kv_rows, int max_blocks, int num_blocks, int num_layers,
                       int64_t layer_stride_elems, int dtype, int validate, int32_t* status,
                       void* stream) {
  if (B < 0 || Nmax < 1 || Nmax > LTD_MAX_NODES || kv_rows < 1 || num_layers < 1 ||
      num_layers > 65535 || layer_stride_elems < 0)
    return LTD_EINVAL;
  if (!dtype_known(dtype) || !latent_supported(d_latent, d_rope)) return LTD_EUNSUPPORTED;
  if (block_table && (max_blocks < 1 || num_blocks < 1)) return LTD_EINVAL;
  if (validate && !status) return LTD_EINVAL;
  if (B == 0) return LTD_OK;
  if (!cache || !prefix_len || !new_prefix_len || !accepted_nodes || !n_accepted) return LTD_EINVAL;
  if (new_prefix_len == prefix_len) return LTD_EINVAL;
  const int elem = dtype == LTD_DTYPE_F32 ? 4 : 2;
  if (!aligned16(cache) ||
      (num_layers > 1 && (layer_stride_elems == 0 || layer_stride_elems * elem % 16 != 0)))
    return LTD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validate) {
    if (ltd::launch_validate_path(block_table, prefix_len, accepted_nodes, n_accepted, B, Nmax,
                                  kv_rows, max_blocks, num_blocks, status, st) != hipSuccess)
      return LTD_EHIP;
  }
  const ltd::LatentCompactArgs a{cache, block_table, prefix_len, new_prefix_len, accepted_nodes, n_accepted,
                                 validate ? status : nullptr, layer_stride_elems * elem, Nmax,
                                 (d_latent + d_rope) * elem, kv_rows, max_blocks};
  return ltd::launch_latent_compact(a, B, num_layers, st) == hipSuccess ? LTD_OK : LTD_EHIP;
}

}  // extern "C"
