"""ctypes binding of libsparse_attn.so (include/sparse_attn.h).

The functions named like the C entry points only marshal arguments: every
step of the computation runs in the library's HIP kernels.  PyTorch supplies
device memory and the current stream.  The convenience layer below them
(``build_layout``, ``forward``, ``backward``, ``SparseAttention``) allocates
outputs with torch and calls those same entry points.

Loading fails loudly when the library has not been built; there is no
fallback implementation.
"""
import contextlib
import ctypes
import math
import os
from dataclasses import dataclass

import torch
from torch.autograd.graph import increment_version

# SPARSE_ATTN_LIB names another build of the same sources to load instead (the
# sanitizer test loads one whose host code is built with ASan and UBSan).
LIB_PATH = os.environ.get("SPARSE_ATTN_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                              "libsparse_attn.so")

SA_OK, SA_ERR_INVALID, SA_ERR_UNSUPPORTED, SA_ERR_BUFFER_TOO_SMALL, SA_ERR_HIP = 0, -1, -2, -3, -4
SA_STRIDED, SA_FIXED, SA_FIXED_PER_HEAD = 0, 1, 2
SA_MODE_A1, SA_MODE_A2, SA_MODE_MERGED, SA_MODE_INTERLEAVED = 0, 1, 2, 3
SA_F32, SA_BF16 = 0, 1
SA_TILE_FULL, SA_TILE_MASKED = 0, 1
SA_ROTARY_ADJACENT, SA_ROTARY_HALVES = 0, 1
SA_BWD_ROW_STATS, SA_BWD_DQ, SA_BWD_DKDV, SA_BWD_ALL_STAGES = 1, 2, 4, 7

EXPORTED = (
    "sparse_attn_layout_count",
    "sparse_attn_layout_size",
    "sparse_attn_layout",
    "sparse_attn_fwd",
    "sparse_attn_bwd_workspace_size",
    "sparse_attn_bwd",
    "sparse_attn_decode_workspace_size",
    "sparse_attn_decode",
    "sparse_attn_rotary",
    "sparse_attn_cache8_store",
    "sparse_attn_decode8_workspace_size",
    "sparse_attn_decode8",
    "sparse_attn_transposed_workspace_size",
    "sparse_attn_fwd_transposed",
    "sparse_attn_bwd_transposed",
    "sparse_attn_bwd_stage",
    "sparse_attn_bwd_noalloc_max_workspace",
    "sparse_attn_bwd_noalloc",
    "sparse_attn_status_string",
)

_lib = None
_i32, _i64, _f32, _vp, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
_PAT = [_i64, _i32, _i32, _i32, _i32, _i32]  # n, block, stride_l, summary_c, pattern, head_mode


class SparseAttnError(RuntimeError):
    def __init__(self, func, status):
        self.status = status
        super().__init__(f"{func} failed: {status_string(status)} ({status})")


def lib():
    """Load the built library (raises if it is missing)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
        L = ctypes.CDLL(LIB_PATH)
        L.sparse_attn_layout_count.argtypes = [_i32, _i32, _i32, _i32, _vp]
        L.sparse_attn_layout_size.argtypes = _PAT + [_vp, _vp]
        L.sparse_attn_layout.argtypes = _PAT + [_vp] * 6 + [_i64, _vp]
        L.sparse_attn_fwd.argtypes = _PAT + [_vp] * 3 + [_i32] * 4 + [_vp] * 4 + [_f32, _vp, _vp, _vp]
        L.sparse_attn_bwd_workspace_size.argtypes = _PAT + [_i32] * 4 + [_vp]
        L.sparse_attn_bwd.argtypes = (_PAT + [_vp] * 6 + [_i32] * 4 + [_vp] * 7 + [_f32]
                                      + [_vp] * 4 + [_sz, _vp])
        _DEC = [_i64, _i32, _i32, _i32, _i32]  # pos, stride_l, summary_c, pattern, head_mode
        L.sparse_attn_decode_workspace_size.argtypes = _DEC + [_i32] * 4 + [_vp]
        L.sparse_attn_decode.argtypes = _DEC + [_i32] * 4 + [_vp] * 5 + [_f32] + [_vp] * 3 + [_sz, _vp]
        L.sparse_attn_rotary.argtypes = ([_i32, _i64] + [_i32] * 4 + [_vp] * 10 + [_i32, _vp, ctypes.c_double, _i32, _i32,
                                                                                   _vp])
        L.sparse_attn_cache8_store.argtypes = ([_i32, _i32, _i64, _i32, _i32] + [_vp] * 5 + [_i64, _i32] + [_vp] * 6)
        L.sparse_attn_decode8_workspace_size.argtypes = _DEC + [_i32] * 5 + [_vp]
        L.sparse_attn_decode8.argtypes = ([_vp] + _DEC + [_i32] * 5 + [_vp] * 7 + [_i64, _i32, _f32] + [_vp] * 4
                                          + [_sz, _vp])
        _TR = [_i64, _i32, _i32, _i32]  # n, block, stride_l, class_block
        L.sparse_attn_transposed_workspace_size.argtypes = _TR + [_i32] * 4 + [_vp]
        L.sparse_attn_fwd_transposed.argtypes = _TR + [_vp] * 3 + [_i32] * 4 + [_vp] * 3 + [_f32] + [_vp] * 3 + [_sz, _vp]
        L.sparse_attn_bwd_transposed.argtypes = (_TR + [_vp] * 6 + [_i32] * 4 + [_vp] * 6 + [_f32] + [_vp] * 4
                                                 + [_sz, _vp])
        L.sparse_attn_bwd_stage.argtypes = (_PAT + [_vp] * 6 + [_i32] * 4 + [_vp] * 7 + [_f32]
                                            + [_vp] * 4 + [_sz, _i32, _vp])
        L.sparse_attn_bwd_noalloc_max_workspace.argtypes = [_vp]
        L.sparse_attn_bwd_noalloc.argtypes = (_PAT + [_vp] * 6 + [_i32] * 4 + [_vp] * 7 + [_f32] + [_vp] * 4)
        L.sparse_attn_status_string.argtypes = [ctypes.c_int]
        L.sparse_attn_status_string.restype = ctypes.c_char_p
        for name in EXPORTED[:-1]:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().sparse_attn_status_string(int(status)).decode()


def _check(func, status):
    if status != SA_OK:
        raise SparseAttnError(func, status)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream, device):
    if stream is None:
        # the handle alone, without a torch.cuda.Stream around it, where torch offers it (no public name)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None and device.type == "cuda" and device.index is not None:
            return raw(device.index)
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _strides(*tensors):
    """Element strides of [batch, heads, n, d] tensors that agree with the
    first in shape, element type, device and strides (d contiguous); raises
    ValueError otherwise, before anything reaches the library."""
    ref = tensors[0]
    shape, st, dtype, device = ref.shape, ref.stride(), ref.dtype, ref.device
    if len(shape) != 4:
        raise ValueError("tensors must be [batch, heads, n, d]")
    # each attribute of a tensor is a call into torch: the first tensor's are read
    # once and the others' once each, and what differs is looked for only then
    if device.type == "cuda" and st[3] == 1:
        for t in tensors[1:]:
            if t.shape != shape or t.stride() != st or t.dtype != dtype or t.device != device:
                break
        else:
            return (ctypes.c_int64 * 3)(st[0], st[1], st[2])
    for t in tensors:
        if t.dim() != 4 or t.shape != ref.shape:
            raise ValueError(f"tensor of shape {tuple(t.shape)} where {tuple(ref.shape)} is expected")
        if t.dtype != ref.dtype:
            raise ValueError(f"tensor of type {t.dtype} where {ref.dtype} is expected")
        if t.device != ref.device or t.device.type != "cuda":
            raise ValueError("every tensor must be on the same GPU")
        if t.stride() != st or t.stride(3) != 1:
            raise ValueError("tensors must have d contiguous and identical strides")
    return (ctypes.c_int64 * 3)(st[0], st[1], st[2])


def _check_lse(lse, q):
    b, h, n, _ = q.shape
    if lse.dtype != torch.float32 or tuple(lse.shape) != (b, h, n) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [batch, heads, n] tensor")
    if lse.device != q.device:
        raise ValueError("lse must be on q's device")


def _check_layout(layout, q):
    if q.shape[2] != layout.n:
        raise ValueError("sequence length differs from the layout's")
    if layout.row_ptr.device != q.device:
        raise ValueError("the layout must be on q's device")


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return SA_BF16
    if t.dtype == torch.float32:
        return SA_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


# ---------------------------------------------------------------------------
# Entry points, same names and argument order as the C ABI
# ---------------------------------------------------------------------------
def sparse_attn_layout_count(stride_l, summary_c, pattern, head_mode):
    ng = ctypes.c_int32(0)
    st = lib().sparse_attn_layout_count(stride_l, summary_c, pattern, head_mode, ctypes.byref(ng))
    _check("sparse_attn_layout_count", st)
    return ng.value


def sparse_attn_layout_size(n, block, stride_l, summary_c, pattern, head_mode):
    entries = max(2, sparse_attn_layout_count(stride_l, summary_c, pattern, head_mode))
    ng = ctypes.c_int32(0)
    nnz = (ctypes.c_int64 * entries)()
    st = lib().sparse_attn_layout_size(n, block, stride_l, summary_c, pattern, head_mode,
                                       ctypes.byref(ng), nnz)
    _check("sparse_attn_layout_size", st)
    return ng.value, list(nnz)[: ng.value]


def sparse_attn_layout(n, block, stride_l, summary_c, pattern, head_mode, row_ptr, col_idx, kind,
                       col_ptr, row_idx, kind_t, capacity, stream=None):
    st = lib().sparse_attn_layout(n, block, stride_l, summary_c, pattern, head_mode, _ptr(row_ptr),
                                  _ptr(col_idx), _ptr(kind), _ptr(col_ptr), _ptr(row_idx), _ptr(kind_t),
                                  capacity, _stream(stream, row_ptr.device))
    _check("sparse_attn_layout", st)


def sparse_attn_fwd(n, block, stride_l, summary_c, pattern, head_mode, row_ptr, col_idx, kind,
                    batch, heads, d_head, dtype, q, k, v, strides, softmax_scale, o, lse, stream=None):
    st = lib().sparse_attn_fwd(n, block, stride_l, summary_c, pattern, head_mode, _ptr(row_ptr),
                               _ptr(col_idx), _ptr(kind), batch, heads, d_head, dtype, _ptr(q), _ptr(k),
                               _ptr(v), strides, softmax_scale, _ptr(o), _ptr(lse),
                               _stream(stream, q.device))
    _check("sparse_attn_fwd", st)


def sparse_attn_bwd_workspace_size(n, block, stride_l, summary_c, pattern, head_mode, batch, heads,
                                   d_head, dtype):
    out = ctypes.c_size_t(0)
    st = lib().sparse_attn_bwd_workspace_size(n, block, stride_l, summary_c, pattern, head_mode, batch,
                                              heads, d_head, dtype, ctypes.byref(out))
    _check("sparse_attn_bwd_workspace_size", st)
    return out.value


def sparse_attn_bwd(n, block, stride_l, summary_c, pattern, head_mode, row_ptr, col_idx, kind,
                    col_ptr, row_idx, kind_t, batch, heads, d_head, dtype, q, k, v, o, dout, lse,
                    strides, softmax_scale, dq, dk, dv, workspace, workspace_bytes, stream=None):
    st = lib().sparse_attn_bwd(n, block, stride_l, summary_c, pattern, head_mode, _ptr(row_ptr),
                               _ptr(col_idx), _ptr(kind), _ptr(col_ptr), _ptr(row_idx), _ptr(kind_t),
                               batch, heads, d_head, dtype, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                               _ptr(dout), _ptr(lse), strides, softmax_scale, _ptr(dq), _ptr(dk),
                               _ptr(dv), _ptr(workspace), workspace_bytes, _stream(stream, q.device))
    _check("sparse_attn_bwd", st)


def sparse_attn_bwd_stage(n, block, stride_l, summary_c, pattern, head_mode, row_ptr, col_idx, kind,
                          col_ptr, row_idx, kind_t, batch, heads, d_head, dtype, q, k, v, o, dout, lse,
                          strides, softmax_scale, dq, dk, dv, workspace, workspace_bytes, stages, stream=None):
    st = lib().sparse_attn_bwd_stage(n, block, stride_l, summary_c, pattern, head_mode, _ptr(row_ptr),
                                     _ptr(col_idx), _ptr(kind), _ptr(col_ptr), _ptr(row_idx), _ptr(kind_t),
                                     batch, heads, d_head, dtype, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                     _ptr(dout), _ptr(lse), strides, softmax_scale, _ptr(dq), _ptr(dk),
                                     _ptr(dv), _ptr(workspace), workspace_bytes, stages, _stream(stream, q.device))
    _check("sparse_attn_bwd_stage", st)


def sparse_attn_bwd_noalloc_max_workspace():
    out = ctypes.c_size_t(0)
    _check("sparse_attn_bwd_noalloc_max_workspace", lib().sparse_attn_bwd_noalloc_max_workspace(ctypes.byref(out)))
    return out.value


def sparse_attn_bwd_noalloc(n, block, stride_l, summary_c, pattern, head_mode, row_ptr, col_idx, kind,
                            col_ptr, row_idx, kind_t, batch, heads, d_head, dtype, q, k, v, o, dout, lse,
                            strides, softmax_scale, dq, dk, dv, stream=None):
    st = lib().sparse_attn_bwd_noalloc(n, block, stride_l, summary_c, pattern, head_mode, _ptr(row_ptr),
                                       _ptr(col_idx), _ptr(kind), _ptr(col_ptr), _ptr(row_idx), _ptr(kind_t),
                                       batch, heads, d_head, dtype, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                       _ptr(dout), _ptr(lse), strides, softmax_scale, _ptr(dq), _ptr(dk),
                                       _ptr(dv), _stream(stream, q.device))
    _check("sparse_attn_bwd_noalloc", st)


def sparse_attn_decode_workspace_size(pos, stride_l, summary_c, pattern, head_mode, batch, heads, d_head, dtype):
    out = ctypes.c_size_t(0)
    st = lib().sparse_attn_decode_workspace_size(pos, stride_l, summary_c, pattern, head_mode, batch, heads,
                                                 d_head, dtype, ctypes.byref(out))
    _check("sparse_attn_decode_workspace_size", st)
    return out.value


def sparse_attn_decode(pos, stride_l, summary_c, pattern, head_mode, batch, heads, d_head, dtype, q, q_strides,
                       k_cache, v_cache, kv_strides, softmax_scale, o, lse, workspace, workspace_bytes,
                       stream=None):
    st = lib().sparse_attn_decode(pos, stride_l, summary_c, pattern, head_mode, batch, heads, d_head, dtype,
                                  _ptr(q), q_strides, _ptr(k_cache), _ptr(v_cache), kv_strides, softmax_scale,
                                  _ptr(o), _ptr(lse), _ptr(workspace), workspace_bytes, _stream(stream, q.device))
    _check("sparse_attn_decode", st)


def sparse_attn_rotary(batch, n, q_heads, k_heads, d_head, dtype, q, q_strides, q_out, q_out_strides, k, k_strides,
                       k_out, k_out_strides, positions, position_strides, n_axes, axis_dims, base, pairing, inverse,
                       stream=None):
    st = lib().sparse_attn_rotary(batch, n, q_heads, k_heads, d_head, dtype, _ptr(q), q_strides, _ptr(q_out),
                                  q_out_strides, _ptr(k), k_strides, _ptr(k_out), k_out_strides, _ptr(positions),
                                  position_strides, n_axes, axis_dims, base, pairing, inverse,
                                  _stream(stream, positions.device))
    _check("sparse_attn_rotary", st)


def sparse_attn_cache8_store(batch, kv_heads, n_new, d_head, dtype, k, v, kv_strides, start, counts, capacity,
                             scale_block, k_cache, v_cache, cache_strides, k_scale, v_scale, stream=None):
    st = lib().sparse_attn_cache8_store(batch, kv_heads, n_new, d_head, dtype, _ptr(k), _ptr(v), kv_strides, _ptr(start),
                                        _ptr(counts), capacity, scale_block, _ptr(k_cache), _ptr(v_cache),
                                        cache_strides, _ptr(k_scale), _ptr(v_scale), _stream(stream, k.device))
    _check("sparse_attn_cache8_store", st)


def sparse_attn_decode8_workspace_size(max_pos, stride_l, summary_c, pattern, head_mode, batch, heads, kv_heads, d_head,
                                       dtype):
    out = ctypes.c_size_t(0)
    st = lib().sparse_attn_decode8_workspace_size(max_pos, stride_l, summary_c, pattern, head_mode, batch, heads,
                                                  kv_heads, d_head, dtype, ctypes.byref(out))
    _check("sparse_attn_decode8_workspace_size", st)
    return out.value


def sparse_attn_decode8(positions, max_pos, stride_l, summary_c, pattern, head_mode, batch, heads, kv_heads, d_head,
                        dtype, q, q_strides, k_cache, v_cache, cache_strides, k_scale, v_scale, capacity, scale_block,
                        softmax_scale, o, o_strides, lse, workspace, workspace_bytes, stream=None):
    st = lib().sparse_attn_decode8(_ptr(positions), max_pos, stride_l, summary_c, pattern, head_mode, batch, heads,
                                   kv_heads, d_head, dtype, _ptr(q), q_strides, _ptr(k_cache), _ptr(v_cache),
                                   cache_strides, _ptr(k_scale), _ptr(v_scale), capacity, scale_block, softmax_scale,
                                   _ptr(o), o_strides, _ptr(lse), _ptr(workspace), workspace_bytes,
                                   _stream(stream, q.device))
    _check("sparse_attn_decode8", st)


# ---------------------------------------------------------------------------
# Convenience layer: torch allocates, the entry points above compute
# ---------------------------------------------------------------------------
@dataclass
class Layout:
    n: int
    block: int
    stride_l: int
    summary_c: int
    pattern: int
    head_mode: int
    n_layouts: int
    nnz: list
    row_ptr: torch.Tensor
    col_idx: torch.Tensor
    kind: torch.Tensor
    col_ptr: torch.Tensor
    row_idx: torch.Tensor
    kind_t: torch.Tensor

    @property
    def pattern_args(self):
        return (self.n, self.block, self.stride_l, self.summary_c, self.pattern, self.head_mode)

    @property
    def row_args(self):
        return (self.row_ptr, self.col_idx, self.kind)

    @property
    def col_args(self):
        return (self.col_ptr, self.row_idx, self.kind_t)


def build_layout(n, block, stride_l, summary_c, pattern, head_mode, device="cuda", stream=None):
    ng, nnz = sparse_attn_layout_size(n, block, stride_l, summary_c, pattern, head_mode)
    nq = n // block
    total = max(1, sum(nnz))
    dev = torch.device(device)
    lay = Layout(n, block, stride_l, summary_c, pattern, head_mode, ng, nnz,
                 row_ptr=torch.empty(ng * (nq + 1), dtype=torch.int32, device=dev),
                 col_idx=torch.empty(total, dtype=torch.int32, device=dev),
                 kind=torch.empty(total, dtype=torch.uint8, device=dev),
                 col_ptr=torch.empty(ng * (nq + 1), dtype=torch.int32, device=dev),
                 row_idx=torch.empty(total, dtype=torch.int32, device=dev),
                 kind_t=torch.empty(total, dtype=torch.uint8, device=dev))
    sparse_attn_layout(*lay.pattern_args, lay.row_ptr, lay.col_idx, lay.kind, lay.col_ptr, lay.row_idx,
                       lay.kind_t, total, stream)
    return lay


def _scale(softmax_scale, d):
    return float(1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale)


def forward(q, k, v, layout: Layout, softmax_scale=None, out=None, lse=None, stream=None):
    """O and LSE of sparse attention over ``layout``; q, k, v are [b, h, n, d] on the GPU."""
    b, h, n, d = q.shape
    strides = _strides(q, k, v)
    _check_layout(layout, q)
    o = torch.empty_like(q) if out is None else out
    _strides(q, o)
    lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if lse is None else lse
    _check_lse(lse, q)
    sparse_attn_fwd(*layout.pattern_args, *layout.row_args, b, h, d, _dtype_code(q), q, k, v, strides,
                    _scale(softmax_scale, d), o, lse, stream)
    return o, lse


def backward(q, k, v, o, dout, lse, layout: Layout, softmax_scale=None, grads=None, workspace=None,
             stream=None, stages=None):
    """dq, dk, dv of sparse attention given the forward's o and lse (``stages``:
    a subset of the SA_BWD_* stages, through sparse_attn_bwd_stage)."""
    b, h, n, d = q.shape
    strides = _strides(q, k, v, o, dout)
    _check_layout(layout, q)
    _check_lse(lse, q)
    dq, dk, dv = grads if grads is not None else (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    _strides(q, dq, dk, dv)
    dtype = _dtype_code(q)
    need = sparse_attn_bwd_workspace_size(*layout.pattern_args, b, h, d, dtype)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    elif workspace.device != q.device:
        raise ValueError("workspace must be on q's device")
    if stages is not None:
        sparse_attn_bwd_stage(*layout.pattern_args, *layout.row_args, *layout.col_args, b, h, d, dtype, q, k, v, o,
                              dout, lse, strides, _scale(softmax_scale, d), dq, dk, dv, workspace,
                              workspace.numel() * workspace.element_size(), stages, stream)
        return dq, dk, dv
    sparse_attn_bwd(*layout.pattern_args, *layout.row_args, *layout.col_args, b, h, d, dtype, q, k, v, o,
                    dout, lse, strides, _scale(softmax_scale, d), dq, dk, dv, workspace,
                    workspace.numel() * workspace.element_size(), stream)
    return dq, dk, dv


def decode(q, k_cache, v_cache, pos, stride_l, summary_c, pattern, head_mode, softmax_scale=None, out=None,
           lse=None, workspace=None, stream=None):
    """Output of query position ``pos`` (q: [b, h, d]) over the cache ([b, h, >= pos + 1, d]) and S_pos."""
    b, h, d = q.shape
    if k_cache.dim() != 4 or k_cache.shape[:2] != (b, h) or k_cache.shape[3] != d or k_cache.shape[2] <= pos:
        raise ValueError("cache must be [batch, heads, >= pos + 1, d] matching q")
    if v_cache.shape != k_cache.shape or v_cache.stride() != k_cache.stride() or k_cache.stride(3) != 1:
        raise ValueError("k_cache and v_cache must share shape and strides, d contiguous")
    if q.stride(2) != 1:
        raise ValueError("q must have d contiguous")
    o = torch.empty_like(q) if out is None else out
    if o.shape != q.shape or o.stride() != q.stride():
        raise ValueError("out must match q in shape and strides")
    lse = torch.empty((b, h), dtype=torch.float32, device=q.device) if lse is None else lse
    dtype = _dtype_code(q)
    if workspace is None:
        need = sparse_attn_decode_workspace_size(pos, stride_l, summary_c, pattern, head_mode, b, h, d, dtype)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    qs = (ctypes.c_int64 * 2)(q.stride(0), q.stride(1))
    ks = (ctypes.c_int64 * 3)(k_cache.stride(0), k_cache.stride(1), k_cache.stride(2))
    try:
        sparse_attn_decode(pos, stride_l, summary_c, pattern, head_mode, b, h, d, dtype, q, qs, k_cache, v_cache, ks,
                           _scale(softmax_scale, d), o, lse, workspace, workspace.numel() * workspace.element_size(),
                           stream)
    except SparseAttnError:
        # a pattern or shape that the size query refuses is reported by it, with or without a workspace
        sparse_attn_decode_workspace_size(pos, stride_l, summary_c, pattern, head_mode, b, h, d, dtype)
        raise
    return o, lse


# ---------------------------------------------------------------------------
# Rotary positions of several axes, and the 8-bit cache with its decoding step
# ---------------------------------------------------------------------------
_SAME = contextlib.nullcontext()
_I64x2, _I64x3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3
_CODE_TYPES = (torch.float8_e4m3fn, torch.uint8)
_DTYPE_CODES = {torch.bfloat16: SA_BF16, torch.float32: SA_F32}


def _here(device, stream):
    """Context in which a call's buffers are allocated and its kernels launched: the
    tensors' device current and, where the caller names a stream, that stream too
    (memory from another stream's pool could still be in use there)."""
    if stream is None:
        return _SAME if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream, device=device)
    return torch.cuda.stream(stream)


def _row_strides(shape, st):
    """Strides of [batch, heads, n, d] (or [batch, heads, d], one token) as the entry points take them.  A dimension of
    one element is never stepped over, so torch's value for it is replaced by one that any layout has."""
    return _I64x3(st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0,
                  st[2] if len(shape) == 4 and shape[2] > 1 else shape[-1])


def _one_layout(shape, st, other):
    """Whether the entry points would step over both alike."""
    return st == other or st[-1] == other[-1] and tuple(_row_strides(shape, st)) == tuple(_row_strides(shape, other))


def _check_ints(name, t, count, device):
    """A contiguous int32 tensor of `count` elements on the device."""
    if t.dtype != torch.int32 or t.shape != (count,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape ({count},)")
    if t.device != device:
        raise ValueError(f"{name} must be on the device of the other tensors")


def grid_positions(shape, device="cuda"):
    """Places of the tokens of a grid in raster order, [tokens, axes] int32, for ``rotary``: (frames, rows, columns) of
    a video, (rows, columns, channels) of an image, (n,) of a sequence."""
    axes = torch.meshgrid(*(torch.arange(s, dtype=torch.int32, device=device) for s in shape), indexing="ij")
    return torch.stack([a.reshape(-1) for a in axes], dim=1)


def _rotary_args(q, k, axis_dims, base, pairing):
    """What a call on tensors of these shapes passes in front of the tensors, and what behind the positions, checked."""
    shape, device, dtype = q.shape, q.device, q.dtype
    k_shape = shape if k is None else k.shape
    # (every attribute of a tensor is a call into torch: each is read once)
    if len(shape) not in (3, 4) or len(k_shape) != len(shape) or k_shape[0] != shape[0] or k_shape[2:] != shape[2:]:
        raise ValueError("q and k must be [batch, heads, n, d] (or [batch, heads, d]) of one batch, n and d")
    if (device.type != "cuda" or dtype not in _DTYPE_CODES
            or k is not None and (k.device != device or k.dtype != dtype)):
        raise ValueError("q and k must share type and GPU, in bfloat16 or float32")
    n, axes = 1 if len(shape) == 3 else shape[2], len(axis_dims)
    return ((shape[0], n, shape[1], 0 if k is None else k_shape[1], shape[-1], _DTYPE_CODES[dtype]),
            (axes, (ctypes.c_int32 * axes)(*axis_dims), base, pairing))


def _rotary_places(positions, shape, axes, device):
    """Address and strides of the positions of tokens [batch, heads, n, d] or [batch, heads, d], checked."""
    single, b = len(shape) == 3, shape[0]
    n = 1 if single else shape[2]
    places, st = positions.shape, positions.stride()
    shared = not single and places in ((n, axes), (1, n, axes))
    if not shared and places != ((b, axes) if single else (b, n, axes)):
        raise ValueError("positions must be [n, axes] or [batch, n, axes] (one token: [batch, axes])")
    if positions.dtype != torch.int32 or positions.device != device or axes > 1 and st[-1] != 1:
        raise ValueError("positions must be int32 with the axes contiguous, on the device of q and k")
    return positions.data_ptr(), _I64x2(0, st[-2]) if shared else _I64x2(st[0], 0 if single else st[1])


def _rotary_run(args, q, k, positions, inverse, out, stream):
    front, behind = args
    shape, device, q_st = q.shape, q.device, q.stride()
    k_shape, k_st = (shape, q_st) if k is None else (k.shape, k.stride())
    if q_st[-1] != 1 or k_st[-1] != 1:
        raise ValueError("q and k must have d contiguous")
    # (of the tensor that is read now: an address is never kept from one call for the next)
    places = _rotary_places(positions, shape, behind[0], device)
    with _here(device, stream):
        if out is None:
            q_out, k_out = torch.empty_like(q), None if k is None else torch.empty_like(k)
        else:
            q_out, k_out = out[0], None if k is None else out[1]
            for t, y in ((q, q_out), (k, k_out)):
                if t is not None and (y.shape != t.shape or y.dtype != t.dtype or y.device != device
                                      or y.stride(-1) != 1):
                    raise ValueError("out must match q and k in shape, type and device, d contiguous")
            if k is not None and (q_out.data_ptr() in (k.data_ptr(), k_out.data_ptr()) or k_out.data_ptr() == q.data_ptr()):
                raise ValueError("out must be the inputs, each its own, or memory apart from them and from each other")
        # (the library itself, as in store8 and decode8: the entry points above would look at every argument again)
        q_rows, k_rows = _row_strides(shape, q_st), _row_strides(k_shape, k_st)
        qo_st, ko_st = q_out.stride(), k_st if k is None else k_out.stride()
        st = lib().sparse_attn_rotary(
            *front, q.data_ptr(), q_rows, q_out.data_ptr(), q_rows if qo_st == q_st else _row_strides(shape, qo_st),
            None if k is None else k.data_ptr(), k_rows, None if k is None else k_out.data_ptr(),
            k_rows if ko_st == k_st else _row_strides(k_shape, ko_st), *places, *behind, 1 if inverse else 0,
            _stream(stream, device))
    _check("sparse_attn_rotary", st)
    if out is not None:  # written behind torch's back: a graph that saved these has to know
        increment_version((q_out,) if k is None else (q_out, k_out))
    return q_out, k_out


def rotary(q, k, positions, axis_dims, base=10000.0, pairing=SA_ROTARY_ADJACENT, inverse=False, out=None, stream=None):
    """q and k turned by their tokens' places on each axis: (q_out, k_out).

    q [b, h, n, d] and k [b, kv_h, n, d] (k may be None), or [b, h, d] and [b, kv_h, d]
    for one token a sequence.  ``positions``: int32 [n, axes] or [b, n, axes] (one
    token: [b, axes]); ``axis_dims``: the elements of d that each axis owns.
    ``inverse`` turns back, which is also the gradient.  ``out``: (q_out, k_out), each its
    own input or memory apart from both inputs.  The result is not differentiable: ``Rotary``'s is."""
    return _rotary_run(_rotary_args(q, k, axis_dims, base, pairing), q, k, positions, inverse, out, stream)


class Rotary(torch.autograd.Function):
    """Autograd wrapper of ``rotary`` for [b, h, n, d] tensors.  The gradient is the inverse rotation, and its own
    gradient the rotation again."""

    @staticmethod
    def forward(ctx, q, k, positions, axis_dims, base=10000.0, pairing=SA_ROTARY_ADJACENT, inverse=False):
        args = _rotary_args(q, k, axis_dims, base, pairing)
        ctx.save_for_backward(positions)
        ctx.args, ctx.axis_dims, ctx.inverse = args, tuple(axis_dims), inverse
        ctx.set_materialize_grads(False)
        return _rotary_run(args, q, k, positions, inverse, None, None)

    @staticmethod
    def backward(ctx, dq, dk):
        (positions,) = ctx.saved_tensors  # what a saved-tensor hook made of them, at another address perhaps
        args, inverse = ctx.args, not ctx.inverse
        if (dq is not None and dk is not None and dq.is_contiguous() and dk.is_contiguous()
                and (dq.data_ptr() | dk.data_ptr()) % 16 == 0 and not torch.is_grad_enabled()):
            # the gradients have the outputs' shapes and type: what the forward's call said of those holds for them
            dq, dk = _rotary_run(args, dq, dk, positions, inverse, None, None)
            return dq, dk, None, None, None, None, None
        # gradients can be absent, or come expanded, permuted or at an odd address: rows have to be contiguous, in whole
        # 16-byte pieces
        grads = [g if g is None or _rows_ok(g) else g.clone(memory_format=torch.contiguous_format) for g in (dq, dk)]
        if grads[0] is None:
            grads.reverse()  # rotary's k is the one that may be absent
        if grads[0] is not None:
            base, pairing = args[1][-2:]
            turn = Rotary.apply if torch.is_grad_enabled() else rotary
            grads = list(turn(grads[0], grads[1], positions, ctx.axis_dims, base, pairing, inverse))
        if dq is None:
            grads.reverse()
        return grads[0], grads[1], None, None, None, None, None


def _rows_ok(t):
    if t.data_ptr() % 16 != 0:
        return False
    unit = 16 // t.element_size()
    return t.is_contiguous() or (t.stride(-1) == 1 and t.stride(-2) >= t.shape[-1]
                                 and all(s % unit == 0 for s in t.stride()[:-1]))


@dataclass
class Cache8:
    """Keys and values in 8 bits (e4m3): k, v [b, kv_heads, capacity, d] (float8_e4m3fn or uint8) with one set of
    strides, k_scale, v_scale [b, kv_heads, ceil(capacity / block)] float32."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    block: int

    def _args(self, d, device):
        """Batch, heads, capacity and strides, checked."""
        k, v, k_scale, v_scale = self.k, self.v, self.k_scale, self.v_scale
        shape, st = k.shape, k.stride()
        # (other types of eight bits have other values for the codes)
        if k.dtype not in _CODE_TYPES or v.dtype not in _CODE_TYPES:
            raise ValueError("the cache's k and v must be float8_e4m3fn or uint8 tensors")
        if len(shape) != 4 or v.shape != shape or not _one_layout(shape, st, v.stride()):
            raise ValueError("the cache's k and v must be [batch, kv_heads, capacity, d] tensors of one layout")
        if shape[3] != d or st[3] != 1:
            raise ValueError("the cache must have the d of the tensors, contiguous")
        b, h, capacity, _ = shape
        scales = (b, h, -(-capacity // self.block))
        for t in (k_scale, v_scale):
            if t.dtype != torch.float32 or t.shape != scales or not t.is_contiguous():
                raise ValueError(f"the scales must be contiguous float32 tensors of shape {scales}")
        if k.device != device or v.device != device or k_scale.device != device or v_scale.device != device:
            raise ValueError("the cache must be on the device of the other tensors")
        return b, h, capacity, _row_strides(shape, st)


def build_cache8(batch, kv_heads, capacity, d, block=64, device="cuda"):
    """An empty 8-bit cache.  A token's key and value lie side by side: the patterns that gather single tokens read
    them in one piece."""
    kv = torch.empty((batch, kv_heads, capacity, 2, d), dtype=torch.float8_e4m3fn, device=device)
    # scales of 0: nothing is held yet
    scales = torch.zeros((2, batch, kv_heads, -(-capacity // block)), dtype=torch.float32, device=device)
    return Cache8(kv[..., 0, :], kv[..., 1, :], scales[0], scales[1], block)


def store8(cache: Cache8, k, v, start=None, counts=None, stream=None):
    """Write new keys and values [b, kv_heads, n_new, d] (or [b, kv_heads, d]: one token) into the cache, the first
    counts[b] of sequence b at positions start[b], ... (int32 [b] on the device; None: 0, and all of them).  The library
    takes one set of strides for k and v; where theirs differ, what is not contiguous is copied first."""
    shape, st, device, dtype = k.shape, k.stride(), k.device, k.dtype
    v_st = v.stride()
    if len(shape) not in (3, 4) or v.shape != shape or v.dtype != dtype or v.device != device:
        raise ValueError("k and v must be [batch, kv_heads, n_new, d] (or [batch, kv_heads, d]) of one type and GPU")
    if device.type != "cuda" or dtype not in _DTYPE_CODES or st[-1] != 1 or v_st[-1] != 1:
        raise ValueError("k and v must be bfloat16 or float32 on the GPU, d contiguous")
    b, h, d = shape[0], shape[1], shape[-1]
    cb, ch, capacity, cache_strides = cache._args(d, device)
    if cb != b or ch != h:
        raise ValueError("k and v must have the cache's batch and heads")
    if start is not None:
        _check_ints("start", start, b, device)
    if counts is not None:
        _check_ints("counts", counts, b, device)
    with _here(device, stream):
        if not _one_layout(shape, st, v_st):
            k, v = k.contiguous(), v.contiguous()
            st = k.stride()
        st = lib().sparse_attn_cache8_store(
            b, h, shape[2] if len(shape) == 4 else 1, d, _DTYPE_CODES[dtype], k.data_ptr(), v.data_ptr(),
            _row_strides(shape, st), None if start is None else start.data_ptr(),
            None if counts is None else counts.data_ptr(), capacity, cache.block, cache.k.data_ptr(), cache.v.data_ptr(),
            cache_strides, cache.k_scale.data_ptr(), cache.v_scale.data_ptr(), _stream(stream, device))
    _check("sparse_attn_cache8_store", st)
    # written behind torch's back: a graph that saved these has to know
    increment_version((cache.k, cache.v, cache.k_scale, cache.v_scale))


def decode8(q, cache: Cache8, positions, stride_l, summary_c, pattern, head_mode, max_pos=None, softmax_scale=None,
            out=None, lse=None, workspace=None, stream=None):
    """Output of one query a sequence (q: [b, h, d], at positions[b], int32 on the device) over the 8-bit cache, and its
    log-sum-exp.  A negative position is a sequence without a query (o = 0, lse = -inf).  ``max_pos``: an upper bound of
    the positions (default: the cache's last); above it o and lse are NaN."""
    shape, st, device, dtype = q.shape, q.stride(), q.device, q.dtype
    if len(shape) != 3 or st[2] != 1 or device.type != "cuda" or dtype not in _DTYPE_CODES:
        raise ValueError("q must be [batch, heads, d] in bfloat16 or float32 on the GPU, d contiguous")
    b, h, d = shape
    cb, kv_heads, capacity, cache_strides = cache._args(d, device)
    if cb != b or h % kv_heads != 0:
        raise ValueError("q must have the cache's batch and a multiple of its heads")
    _check_ints("positions", positions, b, device)
    max_pos = capacity - 1 if max_pos is None else max_pos
    given = [t for t in (out, lse) if t is not None]  # written behind torch's back
    code = _DTYPE_CODES[dtype]
    with _here(device, stream):
        if out is None:
            o = torch.empty_like(q)
            o_st = o.stride()
        else:
            o, o_st = out, out.stride()
            if o.shape != shape or o.dtype != dtype or o.device != device or o_st[2] != 1:
                raise ValueError("out must match q in shape, type and device, d contiguous")
        if lse is None:
            lse = q.new_empty((b, h), dtype=torch.float32)
        elif lse.shape != (b, h) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != device:
            raise ValueError("lse must be a contiguous float32 [batch, heads] tensor on q's device")
        if workspace is None:
            size = ctypes.c_size_t()
            _check("sparse_attn_decode8_workspace_size", lib().sparse_attn_decode8_workspace_size(
                max_pos, stride_l, summary_c, pattern, head_mode, b, h, kv_heads, d, code, ctypes.byref(size)))
            need = size.value
            workspace = q.new_empty(need, dtype=torch.uint8)
        else:
            need = workspace.numel() * workspace.element_size()
            if workspace.device != device or not workspace.is_contiguous():
                raise ValueError("workspace must be contiguous, on q's device")
        status = lib().sparse_attn_decode8(
            positions.data_ptr(), max_pos, stride_l, summary_c, pattern, head_mode, b, h, kv_heads, d, code, q.data_ptr(),
            _I64x2(st[0] if b > 1 else 0, st[1] if h > 1 else 0), cache.k.data_ptr(), cache.v.data_ptr(), cache_strides,
            cache.k_scale.data_ptr(), cache.v_scale.data_ptr(), capacity, cache.block,
            1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale, o.data_ptr(),
            _I64x2(o_st[0] if b > 1 else 0, o_st[1] if h > 1 else 0), lse.data_ptr(), workspace.data_ptr(), need,
            _stream(stream, device))
    _check("sparse_attn_decode8", status)
    if given:
        increment_version(given)
    return o, lse


# ---------------------------------------------------------------------------
# Strided A2 by transposition (Sec. 5.5).  With l dividing n, write positions
# as i = m l + r (class r = i mod l, index m = i div l): j is in A2 of i iff
# j has the same class and m_j <= m_i.  In class order A2 is therefore dense
# causal attention inside each of the l classes of n / l positions.  A class is
# a strided view of a [b, h, n, d] tensor (first row r, a step of l rows), so
# the entry points above compute it unchanged: "batch" = the b * h heads (the
# stride of one head), "heads" = the l classes (a stride of d elements),
# sequence stride l rows, and the dense causal layout of n / l positions (the
# strided pattern with a stride of n / l).  O and the gradients land in place
# in the original layout; LSE comes out in class order, [b * h, l, n / l].
# ---------------------------------------------------------------------------
def transposed_a2_layout(n, stride_l, block, device="cuda", stream=None):
    """Dense causal layout of one class: n / l positions in blocks of ``block``."""
    if n % stride_l != 0 or (n // stride_l) % block != 0:
        raise ValueError("needs l | n and block | n / l")
    m = n // stride_l
    return build_layout(m, block, m, 0, SA_STRIDED, SA_MODE_A1, device=device, stream=stream)


def _class_view_strides(t, stride_l):
    b, h, n, d = t.shape
    if not t.is_contiguous():
        raise ValueError("the transposed path takes contiguous [b, h, n, d] tensors")
    return (ctypes.c_int64 * 3)(n * d, d, stride_l * d)  # a head, a class, a step within a class


def forward_a2_transposed(q, k, v, stride_l, class_layout: Layout, softmax_scale=None, out=None, lse=None,
                          stream=None):
    """O (original layout) and LSE (class order) of strided A2 attention, computed per class."""
    b, h, n, d = q.shape
    strides = _class_view_strides(q, stride_l)
    for t in (k, v):
        if t.shape != q.shape:
            raise ValueError("q, k, v must have one shape")
        _class_view_strides(t, stride_l)
    m = n // stride_l
    if class_layout.n != m:
        raise ValueError("class layout is for another n / l")
    o = torch.empty_like(q) if out is None else out
    _class_view_strides(o, stride_l)
    lse = torch.empty((b * h, stride_l, m), dtype=torch.float32, device=q.device) if lse is None else lse
    sparse_attn_fwd(*class_layout.pattern_args, *class_layout.row_args, b * h, stride_l, d, _dtype_code(q), q, k,
                    v, strides, _scale(softmax_scale, d), o, lse, stream)
    return o, lse


def backward_a2_transposed(q, k, v, o, dout, lse, stride_l, class_layout: Layout, softmax_scale=None, grads=None,
                           workspace=None, stream=None):
    """dq, dk, dv (original layout) of strided A2 attention, given the class-order LSE."""
    b, h, n, d = q.shape
    strides = _class_view_strides(q, stride_l)
    for t in (k, v, o, dout):
        _class_view_strides(t, stride_l)
    dq, dk, dv = grads if grads is not None else (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    dtype = _dtype_code(q)
    need = sparse_attn_bwd_workspace_size(*class_layout.pattern_args, b * h, stride_l, d, dtype)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    sparse_attn_bwd(*class_layout.pattern_args, *class_layout.row_args, *class_layout.col_args, b * h, stride_l,
                    d, dtype, q, k, v, o, dout, lse, strides, _scale(softmax_scale, d), dq, dk, dv, workspace,
                    workspace.numel() * workspace.element_size(), stream)
    return dq, dk, dv


def sparse_attn_transposed_workspace_size(n, block, stride_l, class_block, batch, heads, d_head, dtype):
    out = ctypes.c_size_t(0)
    st = lib().sparse_attn_transposed_workspace_size(n, block, stride_l, class_block, batch, heads, d_head, dtype,
                                                     ctypes.byref(out))
    _check("sparse_attn_transposed_workspace_size", st)
    return out.value


def sparse_attn_fwd_transposed(n, block, stride_l, class_block, row_ptr, col_idx, kind, batch, heads, d_head, dtype,
                               q, k, v, softmax_scale, o, lse, workspace, workspace_bytes, stream=None):
    st = lib().sparse_attn_fwd_transposed(n, block, stride_l, class_block, _ptr(row_ptr), _ptr(col_idx), _ptr(kind),
                                          batch, heads, d_head, dtype, _ptr(q), _ptr(k), _ptr(v), softmax_scale,
                                          _ptr(o), _ptr(lse), _ptr(workspace), workspace_bytes,
                                          _stream(stream, q.device))
    _check("sparse_attn_fwd_transposed", st)


def sparse_attn_bwd_transposed(n, block, stride_l, class_block, row_ptr, col_idx, kind, col_ptr, row_idx, kind_t,
                               batch, heads, d_head, dtype, q, k, v, o, dout, lse, softmax_scale, dq, dk, dv,
                               workspace, workspace_bytes, stream=None):
    st = lib().sparse_attn_bwd_transposed(n, block, stride_l, class_block, _ptr(row_ptr), _ptr(col_idx), _ptr(kind),
                                          _ptr(col_ptr), _ptr(row_idx), _ptr(kind_t), batch, heads, d_head, dtype,
                                          _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse), softmax_scale,
                                          _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), workspace_bytes,
                                          _stream(stream, q.device))
    _check("sparse_attn_bwd_transposed", st)


def band_layout(n, block, stride_l, device="cuda", stream=None):
    """The strided A1 layout the merged transposed path takes for its band."""
    return build_layout(n, block, stride_l, 0, SA_STRIDED, SA_MODE_A1, device=device, stream=stream)


def _check_contiguous(*tensors):
    """The transposed entry points take no strides: [b, h, n, d] contiguous, one shape."""
    shape = tensors[0].shape
    for t in tensors:
        if t.dim() != 4 or t.shape != shape or not t.is_contiguous():
            raise ValueError("the transposed path takes contiguous [batch, heads, n, d] tensors of one shape")


def _transposed_workspace(q, band: Layout, class_block, workspace):
    b, h, n, d = q.shape
    need = sparse_attn_transposed_workspace_size(n, band.block, band.stride_l, class_block, b, h, d, _dtype_code(q))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    return workspace, workspace.numel() * workspace.element_size()


def forward_merged_transposed(q, k, v, band: Layout, class_block, softmax_scale=None, out=None, lse=None,
                              workspace=None, stream=None):
    """O and LSE of strided merged attention, A2 by transposition; contiguous [b, h, n, d] tensors."""
    b, h, n, d = q.shape
    if band.pattern != SA_STRIDED or band.head_mode != SA_MODE_A1 or band.n != n:
        raise ValueError("band must be the strided A1 layout of this n")
    o = torch.empty_like(q) if out is None else out
    _check_contiguous(q, k, v, o)
    lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if lse is None else lse
    if not lse.is_contiguous() or lse.shape != (b, h, n):
        raise ValueError("lse must be a contiguous [batch, heads, n] tensor")
    ws, nbytes = _transposed_workspace(q, band, class_block, workspace)
    sparse_attn_fwd_transposed(n, band.block, band.stride_l, class_block, *band.row_args, b, h, d, _dtype_code(q),
                               q, k, v, _scale(softmax_scale, d), o, lse, ws, nbytes, stream)
    return o, lse


def backward_merged_transposed(q, k, v, o, dout, lse, band: Layout, class_block, softmax_scale=None, grads=None,
                               workspace=None, stream=None):
    """dq, dk, dv of strided merged attention, A2 by transposition."""
    b, h, n, d = q.shape
    if band.pattern != SA_STRIDED or band.head_mode != SA_MODE_A1 or band.n != n:
        raise ValueError("band must be the strided A1 layout of this n")
    dq, dk, dv = grads if grads is not None else (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    _check_contiguous(q, k, v, o, dout, dq, dk, dv)
    if not lse.is_contiguous() or lse.shape != (b, h, n):
        raise ValueError("lse must be a contiguous [batch, heads, n] tensor")
    ws, nbytes = _transposed_workspace(q, band, class_block, workspace)
    sparse_attn_bwd_transposed(n, band.block, band.stride_l, class_block, *band.row_args, *band.col_args, b, h, d,
                               _dtype_code(q), q, k, v, o, dout, lse, _scale(softmax_scale, d), dq, dk, dv, ws,
                               nbytes, stream)
    return dq, dk, dv


class SparseAttention(torch.autograd.Function):
    """Autograd wrapper: saves O and LSE, recomputes attention weights in backward."""

    @staticmethod
    def forward(ctx, q, k, v, layout, softmax_scale=None):
        o, lse = forward(q, k, v, layout, softmax_scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.layout = layout
        ctx.softmax_scale = softmax_scale
        return o

    @staticmethod
    def backward(ctx, dout):
        q, k, v, o, lse = ctx.saved_tensors
        # the entry point takes one set of strides for all tensors: q's
        if dout.stride() != q.stride():
            dout = torch.empty_like(q).copy_(dout)
        dq, dk, dv = backward(q, k, v, o, dout, lse, ctx.layout, ctx.softmax_scale)
        return dq, dk, dv, None, None


class SparseAttentionTransposed(torch.autograd.Function):
    """Autograd wrapper of strided merged attention with A2 by transposition
    (band = the strided A1 layout, class_block = the block of the per-class
    dense causal attention); saves O and LSE, recomputes the weights."""

    @staticmethod
    def forward(ctx, q, k, v, band, class_block, softmax_scale=None):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        o, lse = forward_merged_transposed(q, k, v, band, class_block, softmax_scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.band = band
        ctx.class_block = class_block
        ctx.softmax_scale = softmax_scale
        return o

    @staticmethod
    def backward(ctx, dout):
        q, k, v, o, lse = ctx.saved_tensors
        dq, dk, dv = backward_merged_transposed(q, k, v, o, dout.contiguous(), lse, ctx.band, ctx.class_block,
                                                ctx.softmax_scale)
        return dq, dk, dv, None, None, None
