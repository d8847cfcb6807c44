"""ltd_verify: the tree-verification step of Learning-to-Draft speculative
decoding (arXiv 2603.01639, section 3.2) as hand-written HIP kernels for
MI355X (gfx950), behind the C ABI declared in ``include/ltd_verify.h``.

This module is the thin Python binding: it marshals torch device tensors to
raw pointers and calls ``libltdverify.so`` through ctypes.  Every step of the
path runs in the library's kernels; torch only provides device memory and the
current stream.  There is no fallback: if the library is missing, importing
the binding's calls raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libltdverify.so")

LTD_OK = 0
LTD_EINVAL = -1
LTD_EUNSUPPORTED = -2
LTD_EWORKSPACE = -3
LTD_EHIP = -4

DTYPE_F32 = 0
DTYPE_BF16 = 1

STATUS_OK = 0
STATUS_BAD_NNODES = 1
STATUS_BAD_PARENT = 2
STATUS_BAD_PREFIX = 3
STATUS_BAD_BLOCK = 4
STATUS_BAD_PATH = 5
STATUS_BAD_SCORE = 6
STATUS_BAD_RULE = 7

MAX_NODES = 256
MAX_BIAS = 1024
MAX_LENGTH = 1 << 30
MAX_POOL = 1024
POLICY_SIZE = 0
POLICY_DEPTH = 1

EXPORTED = (
    "ltd_tree_verify_attn_workspace_size",
    "ltd_tree_verify_attn",
    "ltd_tree_accept_workspace_size",
    "ltd_tree_accept",
    "ltd_kv_compact",
    "ltd_tree_verify_attn_grid",
    "ltd_version",
    "ltd_select_candidates",
    "ltd_policy_workspace_size",
    "ltd_policy_forward",
    "ltd_draft_expand_workspace_size",
    "ltd_draft_expand",
    "ltd_tree_accept_sampling_workspace_size",
    "ltd_tree_accept_sampling",
    "ltd_tree_accept_noalloc_max_bytes",
    "ltd_tree_accept_noalloc",
    "ltd_kv_append_q8",
    "ltd_tree_verify_attn_q8_workspace_size",
    "ltd_tree_verify_attn_q8",
    "ltd_kv_compact_q8",
    "ltd_token_counts",
    "ltd_tree_process_logits",
    "ltd_tree_accept_processed",
)


class LtdError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} returned {code}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded HIP library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python paper_2603_01639_amd/build.py` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        f32 = ctypes.c_float
        L.ltd_tree_verify_attn_workspace_size.argtypes = [i32] * 7
        L.ltd_tree_verify_attn_workspace_size.restype = sz
        L.ltd_tree_verify_attn.argtypes = [P] * 8 + [i32] * 9 + [f32, i32, P, sz, i32, P, P]
        L.ltd_tree_verify_attn.restype = i32
        L.ltd_tree_accept_workspace_size.argtypes = [i32] * 3
        L.ltd_tree_accept_workspace_size.restype = sz
        L.ltd_tree_accept.argtypes = [P] * 4 + [i32] * 3 + [P] * 5 + [sz, i32, P, P]
        L.ltd_tree_accept.restype = i32
        L.ltd_tree_accept_noalloc_max_bytes.argtypes = []
        L.ltd_tree_accept_noalloc_max_bytes.restype = sz
        L.ltd_tree_accept_noalloc.argtypes = [P] * 4 + [i32] * 3 + [P] * 4 + [i32, P, P]
        L.ltd_tree_accept_noalloc.restype = i32
        L.ltd_kv_compact.argtypes = [P] * 7 + [i32] * 8 + [i64, i32, i32, P, P]
        L.ltd_kv_compact.restype = i32
        L.ltd_tree_verify_attn_grid.argtypes = [i32] * 9
        L.ltd_tree_verify_attn_grid.restype = i32
        L.ltd_select_candidates.argtypes = [P] * 5 + [i32] * 3 + [P] * 5 + [i32, P, P]
        L.ltd_select_candidates.restype = i32
        L.ltd_policy_workspace_size.argtypes = [i32] * 3
        L.ltd_policy_workspace_size.restype = sz
        L.ltd_policy_forward.argtypes = ([i32, P, P, i32, P, P, f32, i32, i32, P, P, i32, P, P, i32,
                                          P, P, i32, i32, i32, P, P, P, sz, P])
        L.ltd_policy_forward.restype = i32
        L.ltd_draft_expand_workspace_size.argtypes = [i32] * 4
        L.ltd_draft_expand_workspace_size.restype = sz
        L.ltd_draft_expand.argtypes = [P, P] + [i32] * 5 + [P] * 4 + [i32, P, P, sz, i32, P, P]
        L.ltd_draft_expand.restype = i32
        L.ltd_tree_accept_sampling_workspace_size.argtypes = [i32] * 3
        L.ltd_tree_accept_sampling_workspace_size.restype = sz
        L.ltd_tree_accept_sampling.argtypes = [P] * 6 + [i32] * 3 + [f32] + [P] * 4 + [sz, i32, P,
                                                                                     P]
        L.ltd_tree_accept_sampling.restype = i32
        L.ltd_kv_append_q8.argtypes = [P, P, i64] + [P] * 7 + [i32] * 10 + [P, P]
        L.ltd_kv_append_q8.restype = i32
        L.ltd_tree_verify_attn_q8_workspace_size.argtypes = [i32] * 7
        L.ltd_tree_verify_attn_q8_workspace_size.restype = sz
        L.ltd_tree_verify_attn_q8.argtypes = [P] * 10 + [i32] * 10 + [f32, i32, P, sz, i32, P, P]
        L.ltd_tree_verify_attn_q8.restype = i32
        L.ltd_kv_compact_q8.argtypes = [P] * 9 + [i32] * 9 + [i64, i64, i32, P, P]
        L.ltd_kv_compact_q8.restype = i32
        L.ltd_token_counts.argtypes = [P, P] + [i32] * 5 + [P, P]
        L.ltd_token_counts.restype = i32
        L.ltd_tree_process_logits.argtypes = [P] * 10 + [i32] * 4 + [P, i32, P, P]
        L.ltd_tree_process_logits.restype = i32
        L.ltd_tree_accept_processed.argtypes = [P] * 10 + [i32] * 4 + [P] * 5 + [sz, i32, P, P]
        L.ltd_tree_accept_processed.restype = i32
        L.ltd_version.argtypes = []
        L.ltd_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _p(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream
    # The current stream's handle without a torch.cuda.Stream object around it:
    # building one took 2.9 of a call's 12.1 us of host time (a drafting phase
    # of 12 calls and 25 launches is bound by the host: 148.7 us with it, 123.2
    # without).
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dtype_code(t) -> int:
    import torch
    dtype = t.dtype
    if dtype == torch.bfloat16:
        return DTYPE_BF16
    if dtype == torch.float32:
        return DTYPE_F32
    raise TypeError(f"unsupported dtype {dtype}")


def _check(fn, rc):
    if rc != LTD_OK:
        raise LtdError(fn, rc)


def version() -> str:
    return lib().ltd_version().decode()


def attn_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype) -> int:
    return int(lib().ltd_tree_verify_attn_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype))


def attn_grid(B, Nmax, Hq, Hkv, d, max_prefix, dtype, kv_rows, paged=False) -> int:
    """Workgroups of the attention launch; see ``ltd_tree_verify_attn_grid``."""
    return int(lib().ltd_tree_verify_attn_grid(B, Nmax, Hq, Hkv, d, max_prefix, dtype, kv_rows,
                                               int(bool(paged))))


def accept_workspace_size(B, Nmax, Voc) -> int:
    return int(lib().ltd_tree_accept_workspace_size(B, Nmax, Voc))


def _alloc_workspace(nbytes, device):
    import torch
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def tree_verify_attn(q, k_cache, v_cache, prefix_len, parents, n_nodes, out, *, max_prefix: int,
                     block_table=None, num_blocks: int = 0, scale: Optional[float] = None,
                     workspace=None, validate: bool = False, status=None, stream=None):
    """Tree attention; see ``ltd_tree_verify_attn`` in include/ltd_verify.h.

    Tensors are CUDA (HIP) tensors: q/out ``[B][Nmax][Hq][d]``, caches
    contiguous ``[B][Hkv][cap][d]`` or paged ``[num_blocks][Hkv][block][d]``.
    """
    B, Nmax, Hq, d = q.shape
    Hkv = k_cache.shape[1]
    kv_rows = k_cache.shape[2]
    max_blocks = 0 if block_table is None else block_table.shape[1]
    dtype = _dtype_code(q)
    if scale is None:
        scale = d ** -0.5
    if workspace is None:
        workspace = _alloc_workspace(attn_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype),
                                     q.device)
    rc = lib().ltd_tree_verify_attn(
        _p(q), _p(k_cache), _p(v_cache), _p(block_table), _p(prefix_len), _p(parents), _p(n_nodes),
        _p(out), B, Nmax, Hq, Hkv, d, int(max_prefix), kv_rows, max_blocks, int(num_blocks),
        float(scale), dtype, _p(workspace), workspace.numel() * workspace.element_size(),
        int(validate), _p(status), _stream(stream))
    _check("ltd_tree_verify_attn", rc)
    return out


def tree_accept(logits, draft_tokens, parents, n_nodes, pred, accepted_nodes, out_tokens,
                n_accepted, *, workspace=None, validate: bool = False, status=None, stream=None):
    """Per-node argmax and greedy acceptance; see ``ltd_tree_accept``."""
    B, Nmax, Voc = logits.shape
    if workspace is None:
        workspace = _alloc_workspace(accept_workspace_size(B, Nmax, Voc), logits.device)
    rc = lib().ltd_tree_accept(
        _p(logits), _p(draft_tokens), _p(parents), _p(n_nodes), B, Nmax, Voc, _p(pred),
        _p(accepted_nodes), _p(out_tokens), _p(n_accepted), _p(workspace),
        workspace.numel() * workspace.element_size(), int(validate), _p(status), _stream(stream))
    _check("ltd_tree_accept", rc)


def accept_noalloc_max_bytes() -> int:
    return int(lib().ltd_tree_accept_noalloc_max_bytes())


def tree_accept_noalloc(logits, draft_tokens, parents, n_nodes, pred, accepted_nodes, out_tokens,
                        n_accepted, *, validate: bool = False, status=None, stream=None):
    """Greedy acceptance without a workspace; see ``ltd_tree_accept_noalloc``."""
    B, Nmax, Voc = logits.shape
    rc = lib().ltd_tree_accept_noalloc(
        _p(logits), _p(draft_tokens), _p(parents), _p(n_nodes), B, Nmax, Voc, _p(pred),
        _p(accepted_nodes), _p(out_tokens), _p(n_accepted), int(validate), _p(status),
        _stream(stream))
    _check("ltd_tree_accept_noalloc", rc)


def kv_compact(k_cache, v_cache, prefix_len, new_prefix_len, accepted_nodes, n_accepted, *,
               block_table=None, num_blocks: int = 0, num_layers: int = 1,
               layer_stride_elems: int = 0, validate: bool = False, status=None, stream=None):
    """In-place KV compaction; see ``ltd_kv_compact``.

    With ``num_layers > 1`` the caches hold the layers ``layer_stride_elems``
    elements apart and the last three dims are ``[Hkv][rows][d]``.
    """
    B, Nmax = accepted_nodes.shape
    Hkv, kv_rows, d = k_cache.shape[-3], k_cache.shape[-2], k_cache.shape[-1]
    max_blocks = 0 if block_table is None else block_table.shape[1]
    rc = lib().ltd_kv_compact(
        _p(k_cache), _p(v_cache), _p(block_table), _p(prefix_len), _p(new_prefix_len),
        _p(accepted_nodes), _p(n_accepted), B, Nmax, Hkv, d, kv_rows, max_blocks, int(num_blocks),
        int(num_layers), int(layer_stride_elems), _dtype_code(k_cache), int(validate), _p(status),
        _stream(stream))
    _check("ltd_kv_compact", rc)


def select_candidates(scores, pool_parents, pool_tokens, pool_size, n_select, parents, tokens,
                      n_nodes, *, selected=None, depth=None, validate: bool = False, status=None,
                      stream=None):
    """Candidate token selection; see ``ltd_select_candidates``.  Pools are
    ``[B][Vpool]``, outputs ``[B][Nmax]`` int32 CUDA (HIP) tensors."""
    B, Vpool = scores.shape
    Nmax = parents.shape[1]
    rc = lib().ltd_select_candidates(
        _p(scores), _p(pool_parents), _p(pool_tokens), _p(pool_size), _p(n_select), B, Vpool, Nmax,
        _p(selected), _p(parents), _p(tokens), _p(depth), _p(n_nodes), int(validate), _p(status),
        _stream(stream))
    _check("ltd_select_candidates", rc)


def policy_workspace_size(B, h1, h2) -> int:
    return int(lib().ltd_policy_workspace_size(B, h1, h2))


def policy_forward(layout, scores, pool_size, depth, ctx_len, layers, logits, action, *,
                   pad: float = -100.0, action_offset: int = 0, action_scale: int = 1,
                   workspace=None, stream=None):
    """Draft-policy inference; see ``ltd_policy_forward``.  ``layers`` is a
    list of (W [out][in], b [out]) float32 CUDA tensors: two or three layers
    (one or two hidden ReLU layers, then the output layer)."""
    if len(layers) not in (2, 3):
        raise ValueError("a policy has one or two hidden layers")
    B, Vpool = scores.shape
    (w1, b1), *mid, (wo, bo) = layers
    w2, b2 = mid[0] if mid else (None, None)
    h1 = w1.shape[0]
    h2 = 0 if w2 is None else w2.shape[0]
    if workspace is None:
        workspace = _alloc_workspace(policy_workspace_size(B, h1, h2), scores.device)
    rc = lib().ltd_policy_forward(
        int(layout), _p(scores), _p(pool_size), Vpool, _p(depth), _p(ctx_len), float(pad), B,
        w1.shape[1], _p(w1), _p(b1), h1, _p(w2), _p(b2), h2, _p(wo), _p(bo), wo.shape[0],
        int(action_offset), int(action_scale), _p(logits), _p(action), _p(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream))
    _check("ltd_policy_forward", rc)


def draft_expand_workspace_size(B, F, Voc, W) -> int:
    return int(lib().ltd_draft_expand_workspace_size(B, F, Voc, W))


def draft_expand(logits, frontier, scores, pool_parents, pool_tokens, pool_size, new_frontier, *,
                 W: int, workspace=None, validate: bool = False, status=None, stream=None):
    """One round of draft tree expansion; see ``ltd_draft_expand``.  logits
    ``[B][F][Voc]`` float32, pool arrays ``[B][Vpool]`` (updated in place),
    new_frontier ``[B][W_next]``."""
    B, F, Voc = logits.shape
    Vpool = scores.shape[1]
    if workspace is None:
        workspace = _alloc_workspace(draft_expand_workspace_size(B, F, Voc, W), logits.device)
    rc = lib().ltd_draft_expand(
        _p(logits), _p(frontier), B, F, Voc, int(W), new_frontier.shape[1], _p(scores),
        _p(pool_parents), _p(pool_tokens), _p(pool_size), Vpool, _p(new_frontier), _p(workspace),
        workspace.numel() * workspace.element_size(), int(validate), _p(status), _stream(stream))
    _check("ltd_draft_expand", rc)


def accept_sampling_workspace_size(B, Nmax, Voc) -> int:
    return int(lib().ltd_tree_accept_sampling_workspace_size(B, Nmax, Voc))


def tree_accept_sampling(logits, draft_probs, draft_tokens, parents, n_nodes, uniforms,
                         accepted_nodes, out_tokens, n_accepted, *, temperature: float = 1.0,
                         workspace=None, validate: bool = False, status=None, stream=None):
    """Acceptance by recursive rejection sampling at temperature T > 0; see
    ``ltd_tree_accept_sampling``."""
    B, Nmax, Voc = logits.shape
    if workspace is None:
        workspace = _alloc_workspace(accept_sampling_workspace_size(B, Nmax, Voc), logits.device)
    rc = lib().ltd_tree_accept_sampling(
        _p(logits), _p(draft_probs), _p(draft_tokens), _p(parents), _p(n_nodes), _p(uniforms), B,
        Nmax, Voc, float(temperature), _p(accepted_nodes), _p(out_tokens), _p(n_accepted),
        _p(workspace), workspace.numel() * workspace.element_size(), int(validate), _p(status),
        _stream(stream))
    _check("ltd_tree_accept_sampling", rc)


# ---- the 8-bit KV cache and the sampling rules.  These calls check their
# tensors (types, shapes, layouts, one device) before they pass pointers on, and
# run on the tensors' GPU whichever is current.

def _want(name, t, dtypes, shape):
    """t has one of the types and the shape and is contiguous."""
    if t.dtype in dtypes and t.shape == shape and t.is_contiguous():
        return  # (the usual case, in as little host time as can be)
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has type {t.dtype}, not {' or '.join(map(str, dtypes))}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")


def _dims(name, t, n):
    """t's shape, of n dimensions."""
    if t.dim() != n:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {n} dimensions")
    return t.shape


def _int32(shape, **tensors):
    import torch
    kind = (torch.int32,)
    for name, t in tensors.items():
        if t is not None:
            _want(name, t, kind, shape)


def _workspace_for(stream, nbytes, device):
    """A workspace from the memory of the stream that will use it: of another
    stream's, it could be handed out again while the call still runs."""
    if stream is None:
        return _alloc_workspace(nbytes, device)
    import torch
    with torch.cuda.stream(stream):
        return _alloc_workspace(nbytes, device)


def _space(workspace):
    """A workspace's pointer and bytes."""
    if not workspace.is_contiguous():
        raise ValueError("workspace is not contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _run(fn, args, tensors, stream):
    """Calls fn(*args, stream) on the GPU that holds the tensors, the last of
    which is the call's status."""
    import torch
    status = tensors[-1]
    if status is not None and (status.dtype != torch.int32 or status.numel() < 1):
        raise TypeError(f"status is {status.numel()} of {status.dtype}, not an int32")
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{fn}: tensors on {tensors[0].device} and on {t.device}")
    if dev < 0:
        raise ValueError(f"{fn} needs tensors on a GPU, not on {tensors[0].device}")
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"{fn}: tensors on {tensors[0].device}, a stream of {stream.device}")
    handle = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    call = getattr(lib(), fn)
    if torch.cuda.current_device() == dev:
        rc = call(*args, handle)
    else:
        with torch.cuda.device(dev):
            rc = call(*args, handle)
    if rc != LTD_OK:
        raise LtdError(fn, rc)


def _q8_cache(k_cache, v_cache, k_scale, v_scale, block_table, num_blocks, scale_rows, lead):
    """The geometry of an 8-bit cache of `lead` leading dimensions (layers):
    kv heads, rows of a page, head size, blocks a sequence."""
    import torch
    if scale_rows not in (16, 32, 64, 128):
        raise ValueError(f"scale_rows is {scale_rows}, not 16, 32, 64 or 128")
    if k_cache.dim() != lead + 4:
        raise ValueError(f"k_cache has {k_cache.dim()} dimensions, not {lead + 4}")
    pages, Hkv, kv_rows, d = k_cache.shape[lead:]
    codes = (torch.float8_e4m3fn, torch.uint8)
    scales = (torch.uint8, torch.float8_e8m0fnu)
    shape = tuple(k_cache.shape)
    _want("k_cache", k_cache, codes, shape)
    _want("v_cache", v_cache, codes, shape)
    sshape = shape[:lead + 2] + (-(-kv_rows // scale_rows),)
    _want("k_scale", k_scale, scales, sshape)
    _want("v_scale", v_scale, scales, sshape)
    max_blocks = 0
    if block_table is not None:
        _int32(_dims("block_table", block_table, 2), block_table=block_table)
        max_blocks = block_table.shape[1]
        if num_blocks > pages:
            raise ValueError(f"num_blocks is {num_blocks}, the cache holds {pages}")
    return pages, Hkv, kv_rows, d, max_blocks


def _batch_pages(B, pages, block_table):
    """A contiguous cache holds a page per sequence, a block table a row."""
    if block_table is None and pages < B:
        raise ValueError(f"the cache holds {pages} sequences, the batch {B}")
    if block_table is not None and block_table.shape[0] != B:
        raise ValueError(f"block_table has {block_table.shape[0]} rows for {B} sequences")


def _row_stride(name, t):
    """Elements from one [Hkv][d] row of t [B][Nmax][Hkv][d] to the next."""
    B, N, Hkv, d = t.shape
    if d > 1 and t.stride(3) != 1 or Hkv > 1 and t.stride(2) != d:
        raise ValueError(f"{name}: a row's heads and dims are not contiguous")
    stride = t.stride(1) if N > 1 else t.stride(0) if B > 1 else Hkv * d
    if B > 1 and t.stride(0) != N * stride:
        raise ValueError(f"{name}: rows are not evenly spaced over the batch")
    return stride


def kv_append_q8(k_new, v_new, k_cache, v_cache, k_scale, v_scale, prefix_len, n_rows, *,
                 scale_rows: int, block_table=None, num_blocks: int = 0, validate: bool = False,
                 status=None, stream=None):
    """Rows of a prompt or a draft tree into an 8-bit KV cache; see
    ``ltd_kv_append_q8``.  k_new, v_new ``[B][Nmax][Hkv][d]`` (bfloat16 or
    float32, views with evenly spaced rows welcome), caches ``[pages][Hkv][rows][d]``
    float8_e4m3fn or uint8, scales ``[pages][Hkv][ceil(rows / scale_rows)]`` uint8."""
    pages, Hkv, kv_rows, d, max_blocks = _q8_cache(k_cache, v_cache, k_scale, v_scale, block_table,
                                                   num_blocks, scale_rows, 0)
    dtype = _dtype_code(k_new)
    if v_new.dtype != k_new.dtype:
        raise TypeError(f"k_new has type {k_new.dtype}, v_new {v_new.dtype}")
    if k_new.dim() != 4 or k_new.shape != v_new.shape or tuple(k_new.shape[2:]) != (Hkv, d):
        raise ValueError(f"k_new {tuple(k_new.shape)} and v_new {tuple(v_new.shape)} are not both "
                         f"(*, *, {Hkv}, {d})")
    B, Nmax = k_new.shape[:2]
    _batch_pages(B, pages, block_table)
    _int32((B,), prefix_len=prefix_len, n_rows=n_rows)
    if B == 0 or Nmax == 0:
        return
    stride = _row_stride("k_new", k_new)
    if v_new.stride() != k_new.stride() and _row_stride("v_new", v_new) != stride:
        raise ValueError("k_new and v_new have rows of different strides")
    _run("ltd_kv_append_q8",
         (_p(k_new), _p(v_new), stride, _p(k_cache), _p(v_cache), _p(k_scale), _p(v_scale),
          _p(block_table), _p(prefix_len), _p(n_rows), B, Nmax, Hkv, d, kv_rows, max_blocks,
          int(num_blocks), int(scale_rows), dtype, int(validate), _p(status)),
         (k_new, v_new, k_cache, v_cache, k_scale, v_scale, block_table, prefix_len, n_rows, status),
         stream)


def attn_q8_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype) -> int:
    return int(lib().ltd_tree_verify_attn_q8_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype))


def tree_verify_attn_q8(q, k_cache, v_cache, k_scale, v_scale, prefix_len, parents, n_nodes, out, *,
                        max_prefix: int, scale_rows: int, block_table=None, num_blocks: int = 0,
                        scale: Optional[float] = None, workspace=None, validate: bool = False,
                        status=None, stream=None):
    """Tree attention over an 8-bit KV cache; see ``ltd_tree_verify_attn_q8``.
    q/out ``[B][Nmax][Hq][d]`` bfloat16 or float32, the cache as for
    ``kv_append_q8``.  A single token a sequence is a tree of one node."""
    pages, Hkv, kv_rows, d, max_blocks = _q8_cache(k_cache, v_cache, k_scale, v_scale, block_table,
                                                   num_blocks, scale_rows, 0)
    dtype = _dtype_code(q)
    B, Nmax, Hq, _ = _dims("q", q, 4)
    _want("q", q, (q.dtype,), (B, Nmax, Hq, d))
    _want("out", out, (q.dtype,), q.shape)
    _batch_pages(B, pages, block_table)
    _int32((B,), prefix_len=prefix_len, n_nodes=n_nodes)
    _int32((B, Nmax), parents=parents)
    if scale is None:
        scale = d ** -0.5
    if workspace is None:
        workspace = _workspace_for(
            stream, attn_q8_workspace_size(B, Nmax, Hq, Hkv, d, max_prefix, dtype), q.device)
    _run("ltd_tree_verify_attn_q8",
         (_p(q), _p(k_cache), _p(v_cache), _p(k_scale), _p(v_scale), _p(block_table),
          _p(prefix_len), _p(parents), _p(n_nodes), _p(out), B, Nmax, Hq, Hkv, d, int(max_prefix),
          kv_rows, max_blocks, int(num_blocks), int(scale_rows), float(scale), dtype,
          *_space(workspace), int(validate), _p(status)),
         (q, k_cache, v_cache, k_scale, v_scale, block_table, prefix_len, parents, n_nodes, out,
          workspace, status), stream)
    return out


def kv_compact_q8(k_cache, v_cache, k_scale, v_scale, prefix_len, new_prefix_len, accepted_nodes,
                  n_accepted, *, scale_rows: int, block_table=None, num_blocks: int = 0,
                  num_layers: Optional[int] = None, layer_stride_elems: int = 0, scale_stride_elems: int = 0,
                  validate: bool = False, status=None, stream=None):
    """In-place compaction of an 8-bit KV cache; see ``ltd_kv_compact_q8``.
    With a leading dimension of layers, caches ``[layers][pages][Hkv][rows][d]``
    and scales alike, the strides default to the tensors' own and num_layers to
    all of them; without one the tensors are the first layer's views of buffers
    that hold num_layers at the strides."""
    lead = k_cache.dim() - 4
    if lead not in (0, 1):
        raise ValueError(f"k_cache has {k_cache.dim()} dimensions, not 4 or 5")
    pages, Hkv, kv_rows, d, max_blocks = _q8_cache(k_cache, v_cache, k_scale, v_scale, block_table,
                                                   num_blocks, scale_rows, lead)
    if num_layers is None:
        num_layers = k_cache.shape[0] if lead else 1
    if lead:
        if num_layers > k_cache.shape[0]:
            raise ValueError(f"num_layers is {num_layers}, the cache holds {k_cache.shape[0]}")
        layer_stride_elems = layer_stride_elems or k_cache.stride(0)
        scale_stride_elems = scale_stride_elems or k_scale.stride(0)
        last = max(k_cache.shape[0] - 1, 0)
        if ((num_layers - 1) * layer_stride_elems > last * k_cache.stride(0)
                or (num_layers - 1) * scale_stride_elems > last * k_scale.stride(0)):
            raise ValueError(f"{num_layers} layers at these strides pass the tensors' end")
    elif num_layers > 1:  # one layer's view of a larger buffer: the others lie in the same one
        for t, stride in ((k_cache, layer_stride_elems), (v_cache, layer_stride_elems),
                          (k_scale, scale_stride_elems), (v_scale, scale_stride_elems)):
            end = t.storage_offset() + (num_layers - 1) * stride + t.numel()  # (elements of a byte)
            if end > t.untyped_storage().nbytes():
                raise ValueError(f"{num_layers} layers at these strides pass the tensors' end")
    B, Nmax = _dims("accepted_nodes", accepted_nodes, 2)
    _batch_pages(B, pages, block_table)
    _int32((B, Nmax), accepted_nodes=accepted_nodes)
    _int32((B,), prefix_len=prefix_len, new_prefix_len=new_prefix_len, n_accepted=n_accepted)
    _run("ltd_kv_compact_q8",
         (_p(k_cache), _p(v_cache), _p(k_scale), _p(v_scale), _p(block_table), _p(prefix_len),
          _p(new_prefix_len), _p(accepted_nodes), _p(n_accepted), B, Nmax, Hkv, d, kv_rows,
          max_blocks, int(num_blocks), int(scale_rows), int(num_layers), int(layer_stride_elems),
          int(scale_stride_elems), int(validate), _p(status)),
         (k_cache, v_cache, k_scale, v_scale, block_table, prefix_len, new_prefix_len,
          accepted_nodes, n_accepted, status), stream)


def token_counts(tokens, n_tokens, counts, *, prompt: bool = False, reset: bool = False,
                 stream=None):
    """Adds tokens ``[B][T]`` (the first n_tokens[b] of each row) to the table of
    occurrences counts ``[B][Voc]`` int32; see ``ltd_token_counts``."""
    B, T = _dims("tokens", tokens, 2)
    _int32((B, T), tokens=tokens)
    _int32((B,), n_tokens=n_tokens)
    _int32((B, _dims("counts", counts, 2)[1]), counts=counts)
    _run("ltd_token_counts",
         (_p(tokens), _p(n_tokens), B, T, counts.shape[1], int(bool(prompt)), int(bool(reset)),
          _p(counts)), (counts, tokens, n_tokens, None), stream)


def _rules(logits, draft_tokens, parents, n_nodes, counts, penalties, bias_tokens, bias_values,
           n_bias, mask):
    """The checked arguments of a call with sampling rules, and its tensors."""
    import torch
    B, Nmax, Voc = _dims("logits", logits, 3)
    _want("logits", logits, (torch.float32,), (B, Nmax, Voc))
    _int32((B, Nmax), draft_tokens=draft_tokens, parents=parents)
    _int32((B,), n_nodes=n_nodes, n_bias=n_bias)
    _int32((B, Voc), counts=counts)
    _int32((B, Nmax, -(-Voc // 32)), mask=mask)
    if penalties is not None:
        _want("penalties", penalties, (torch.float32,), (B, 3))
    max_bias = 0
    if bias_tokens is not None:
        if bias_values is None or n_bias is None:
            raise ValueError("bias_tokens needs bias_values and n_bias")
        max_bias = _dims("bias_tokens", bias_tokens, 2)[1]
        _int32((B, max_bias), bias_tokens=bias_tokens)
        _want("bias_values", bias_values, (torch.float32,), (B, max_bias))
    elif bias_values is not None or n_bias is not None:
        raise ValueError("bias_values and n_bias need bias_tokens")
    tensors = (logits, draft_tokens, parents, n_nodes, counts, penalties, bias_tokens, bias_values,
               n_bias, mask)
    return (*map(_p, tensors), B, Nmax, Voc, max_bias), tensors


def tree_process_logits(logits, draft_tokens, parents, n_nodes, out, *, counts=None, penalties=None,
                        bias_tokens=None, bias_values=None, n_bias=None, mask=None,
                        validate: bool = False, status=None, stream=None):
    """Penalties, biases and masks on the logits ``[B][Nmax][Voc]`` of every tree
    node, written to out (which may be logits itself); see
    ``ltd_tree_process_logits``.  mask ``[B][Nmax][ceil(Voc / 32)]`` int32."""
    import torch
    args, tensors = _rules(logits, draft_tokens, parents, n_nodes, counts, penalties, bias_tokens,
                           bias_values, n_bias, mask)
    _want("out", out, (torch.float32,), logits.shape)
    _run("ltd_tree_process_logits", args + (_p(out), int(validate), _p(status)),
         tensors + (out, status), stream)
    return out


def tree_accept_processed(logits, draft_tokens, parents, n_nodes, pred, accepted_nodes, out_tokens,
                          n_accepted, *, counts=None, penalties=None, bias_tokens=None,
                          bias_values=None, n_bias=None, mask=None, workspace=None,
                          validate: bool = False, status=None, stream=None):
    """Greedy acceptance on processed logits, which are not written; see
    ``ltd_tree_accept_processed``."""
    args, tensors = _rules(logits, draft_tokens, parents, n_nodes, counts, penalties, bias_tokens,
                           bias_values, n_bias, mask)
    B, Nmax, Voc = logits.shape
    _int32((B, Nmax), pred=pred, accepted_nodes=accepted_nodes, out_tokens=out_tokens)
    _int32((B,), n_accepted=n_accepted)
    if workspace is None:
        workspace = _workspace_for(stream, accept_workspace_size(B, Nmax, Voc), logits.device)
    _run("ltd_tree_accept_processed",
         args + (_p(pred), _p(accepted_nodes), _p(out_tokens), _p(n_accepted), *_space(workspace), int(validate), _p(status)),
         tensors + (pred, accepted_nodes, out_tokens, n_accepted, workspace, status), stream)
