"""ctypes binding of libstructkv.so: same names as the C entry points, marshalling only.

Tensors are torch tensors (device memory + streams are PyTorch's job); every step of the path
runs inside the library's HIP kernels.  cu_seqlens / k_per_seq / rows_per_seq are host sequences.
"""
from __future__ import annotations

import array
import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstructkv.so")

STRUCTKV_OK = 0
STRUCTKV_ERR_INVALID_ARG = 1
STRUCTKV_ERR_UNSUPPORTED = 2
STRUCTKV_ERR_WORKSPACE = 3
STRUCTKV_ERR_HIP = 4
STRUCTKV_DTYPE_F32 = 0
STRUCTKV_DTYPE_BF16 = 1
STRUCTKV_MAX_BATCH = 64
STRUCTKV_STATIC_TOPK_MAX_TOKENS = 1048576
STRUCTKV_MAX_DRAFTS = 64

EXPORTS = (
    "structkv_last_error", "structkv_version", "structkv_workspace_bytes", "structkv_score_layer",
    "structkv_accumulate_centrality", "structkv_score_layer_accumulate", "structkv_score_layer_groups",
    "structkv_select_topk", "structkv_select_topk_static",
    "structkv_gather_kv", "structkv_layer_step", "structkv_layer_step_workspace_bytes", "structkv_layer_begin",
    "structkv_layer_finish",
    "structkv_truncate_hidden", "structkv_block_scores",
    "structkv_pivot_workspace_bytes", "structkv_pivot_metrics", "structkv_score_layer_pivot", "structkv_transition_scores",
    "structkv_cache_workspace_bytes", "structkv_cache_append", "structkv_cache_attend", "structkv_cache_accept",
    "structkv_cache_evict",
    "structkv_debug_probs", "structkv_debug_score_steps",
)


class structkv_shape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("window", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class structkv_cache(ctypes.Structure):
    """A layer's cache in use; make_cache fills it in from tensors (and keeps those alive)."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("stride_head", ctypes.c_int64), ("stride_slot", ctypes.c_int64),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("planes", ctypes.c_int32),
                ("mass", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("cu_slots", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("missed", ctypes.c_void_p)]


class StructKVError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("structkv status %d: %s" % (status, message))
        self.status = status


if not os.path.exists(LIB_PATH):
    raise ImportError("libstructkv.so is not built: run `python -m paper_2604_06746_amd.build` "
                      "(hipcc, --offload-arch=gfx950).  There is no fallback path.")
_lib = ctypes.CDLL(LIB_PATH)

_vp, _i32, _i64, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_sp = ctypes.POINTER(structkv_shape)
_lib.structkv_last_error.restype = ctypes.c_char_p
_lib.structkv_last_error.argtypes = []
_lib.structkv_version.restype = _i32
_lib.structkv_workspace_bytes.restype = _sz
_lib.structkv_workspace_bytes.argtypes = [_sp, _i32, _i64]
_lib.structkv_score_layer.restype = _i32
_lib.structkv_score_layer.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.structkv_debug_score_steps.restype = _i32
_lib.structkv_debug_score_steps.argtypes = _lib.structkv_score_layer.argtypes + [_i32, _i32]
_lib.structkv_accumulate_centrality.restype = _i32
_lib.structkv_accumulate_centrality.argtypes = [_vp, _vp, _i64, _f32, _f32, _vp]
_lib.structkv_score_layer_accumulate.restype = _i32
_lib.structkv_score_layer_accumulate.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp, _f32, _f32, _vp,
                                                 _vp, _vp, _sz, _vp]
_lib.structkv_score_layer_groups.restype = _i32
_lib.structkv_score_layer_groups.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.structkv_select_topk.restype = _i32
_lib.structkv_select_topk.argtypes = [_vp, _i32, _vp, _vp, _i32, _vp, _vp, _sz, _vp]
_lib.structkv_select_topk_static.restype = _i32
_lib.structkv_select_topk_static.argtypes = [_vp, _i32, _vp, _vp, _i32, _vp, _vp]
_lib.structkv_gather_kv.restype = _i32
_lib.structkv_gather_kv.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _vp,
                                    _vp, _vp, _vp]
_lib.structkv_layer_step_workspace_bytes.restype = _sz
_lib.structkv_layer_step_workspace_bytes.argtypes = [_sp, _i32, _i64]
_lib.structkv_layer_step.restype = _i32
_lib.structkv_layer_step.argtypes = [_sp, _vp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _i32, _vp, _vp, _f32, _f32, _vp,
                                     _vp, _vp, _vp, _vp, _i64, _i64, _vp, _sz, _vp]
_lib.structkv_layer_begin.restype = _i32
_lib.structkv_layer_begin.argtypes = _lib.structkv_layer_step.argtypes
_lib.structkv_layer_finish.restype = _i32
_lib.structkv_layer_finish.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _i64, _i64,
                                       _vp, _sz, _vp]
_lib.structkv_truncate_hidden.restype = _i32
_lib.structkv_truncate_hidden.argtypes = [_vp, _i64, _vp, _i64, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp]
_lib.structkv_block_scores.restype = _i32
_lib.structkv_block_scores.argtypes = [_vp, _i32, _vp, _i32, _vp, _vp]
_lib.structkv_pivot_workspace_bytes.restype = _sz
_lib.structkv_pivot_workspace_bytes.argtypes = [_sp, _i64]
_lib.structkv_score_layer_pivot.restype = _i32
_lib.structkv_score_layer_pivot.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, ctypes.c_double, _vp, _vp, _vp, _vp,
                                            _vp, _vp, _sz, _vp]
_lib.structkv_pivot_metrics.restype = _i32
_lib.structkv_pivot_metrics.argtypes = [_sp, _vp, _vp, _i64, _i64, _i32, _vp, ctypes.c_double, _vp, _vp, _vp, _sz,
                                        _vp]
_lib.structkv_transition_scores.restype = _i32
_lib.structkv_transition_scores.argtypes = [_vp, _vp, _vp, _i32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                            _vp, _vp]
_lib.structkv_debug_probs.restype = _i32
_lib.structkv_debug_probs.argtypes = [_sp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _sz, _vp, _i32]
_cp = ctypes.POINTER(structkv_cache)
_lib.structkv_cache_workspace_bytes.restype = _sz
_lib.structkv_cache_workspace_bytes.argtypes = [_cp, _i32, _i64]
_lib.structkv_cache_append.restype = _i32
_lib.structkv_cache_append.argtypes = [_cp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _vp]
_lib.structkv_cache_attend.restype = _i32
_lib.structkv_cache_attend.argtypes = [_cp, _i32, _f32, _f32, _vp, _vp, _i64, _i64, _vp, _vp, _f32, _vp, _vp, _vp, _sz, _vp]
_lib.structkv_cache_accept.restype = _i32
_lib.structkv_cache_accept.argtypes = [_cp, _i32, _f32, _f32, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp]
_lib.structkv_cache_evict.restype = _i32
_lib.structkv_cache_evict.argtypes = [_cp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]


def make_shape(n_q_heads: int, n_kv_heads: int, head_dim: int, window: int, dtype: int,
               causal: bool = False, scale: float = 0.0) -> structkv_shape:
    return structkv_shape(n_q_heads, n_kv_heads, head_dim, window, dtype, int(bool(causal)), float(scale))


# What a call costs on the host is part of its time: a layer step of a few hundred tokens takes the GPU 11 us.  Pointers and streams
# go to ctypes as plain integers (its argument types convert them), arrays of budgets and offsets straight from the sequence, and the
# current stream's handle comes without a Stream object around it (through a function of torch's own that a build may lack; then with
# one): 18.0 -> 12.0 us a step with its two launches.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _host_i64(values: Sequence[int]):
    try:
        if len(values) > 8:   # (65 offsets: 2.0 us against 4.0)
            return (_i64 * len(values)).from_buffer(array.array("q", values))
        return (_i64 * len(values))(*values)
    except TypeError:   # (numbers of other kinds)
        return (_i64 * len(values))(*[int(v) for v in values])


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int) -> None:
    if status != STRUCTKV_OK:
        raise StructKVError(status, _lib.structkv_last_error().decode())


def structkv_last_error() -> str:
    return _lib.structkv_last_error().decode()


def structkv_version() -> int:
    return int(_lib.structkv_version())


def structkv_workspace_bytes(shape: Optional[structkv_shape], batch: int, total_tokens: int) -> int:
    return int(_lib.structkv_workspace_bytes(ctypes.byref(shape) if shape is not None else None, batch,
                                             total_tokens))


def structkv_score_layer(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor,
                         cu_seqlens: Sequence[int], indeg_out: torch.Tensor, entropy_out: torch.Tensor,
                         entropy_per_head_out: Optional[torch.Tensor], workspace: torch.Tensor,
                         stream=None) -> None:
    """k: [G, total, d] view with d contiguous (head/token strides are passed through)."""
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous()
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_score_layer(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                     len(cu_seqlens) - 1, cu, _ptr(indeg_out), _ptr(entropy_out),
                                     _ptr(entropy_per_head_out), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream)))


def structkv_debug_score_steps(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor,
                               cu_seqlens: Sequence[int], indeg_out: torch.Tensor, entropy_out: torch.Tensor,
                               entropy_per_head_out: Optional[torch.Tensor], workspace: torch.Tensor,
                               step_mask: int, stream=None, force_simt: bool = False) -> None:
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_debug_score_steps(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                           len(cu_seqlens) - 1, cu, _ptr(indeg_out), _ptr(entropy_out),
                                           _ptr(entropy_per_head_out), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _stream(stream),
                                           step_mask, int(bool(force_simt))))


def structkv_accumulate_centrality(centrality: torch.Tensor, indeg: torch.Tensor, lam: float, inv_w: float,
                                   stream=None) -> None:
    assert centrality.numel() == indeg.numel()
    _check(_lib.structkv_accumulate_centrality(_ptr(centrality), _ptr(indeg), centrality.numel(), lam, inv_w,
                                               _stream(stream)))


def structkv_score_layer_accumulate(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor,
                                    cu_seqlens: Sequence[int], indeg_out: torch.Tensor, centrality: torch.Tensor,
                                    lam: float, inv_w: float, entropy_out: torch.Tensor,
                                    entropy_per_head_out: Optional[torch.Tensor], workspace: torch.Tensor,
                                    stream=None) -> None:
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous()
    assert centrality.numel() == indeg_out.numel()
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_score_layer_accumulate(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                                len(cu_seqlens) - 1, cu, _ptr(indeg_out), _ptr(centrality), lam,
                                                inv_w, _ptr(entropy_out), _ptr(entropy_per_head_out),
                                                _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                _stream(stream)))


def structkv_score_layer_groups(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor,
                                cu_seqlens: Sequence[int], indeg_out: torch.Tensor, indeg_groups_out: torch.Tensor,
                                entropy_out: torch.Tensor, entropy_per_head_out: Optional[torch.Tensor],
                                workspace: torch.Tensor, stream=None) -> None:
    """indeg_groups_out: [G, total] fp32, contiguous."""
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous() and indeg_groups_out.is_contiguous()
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_score_layer_groups(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                            len(cu_seqlens) - 1, cu, _ptr(indeg_out), _ptr(indeg_groups_out),
                                            _ptr(entropy_out), _ptr(entropy_per_head_out), _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)))


def structkv_select_topk(scores: torch.Tensor, cu_seqlens: Sequence[int], k_per_seq: Sequence[int],
                         keep_tail: int, idx_out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    cu, ks = _host_i64(cu_seqlens), _host_i64(k_per_seq)
    _check(_lib.structkv_select_topk(_ptr(scores), len(k_per_seq), cu, ks, keep_tail, _ptr(idx_out),
                                     _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)))


def structkv_select_topk_static(scores: torch.Tensor, cu_seqlens: Sequence[int], k_per_seq: Sequence[int],
                                keep_tail: int, idx_out: torch.Tensor, stream=None) -> None:
    cu, ks = _host_i64(cu_seqlens), _host_i64(k_per_seq)
    _check(_lib.structkv_select_topk_static(_ptr(scores), len(k_per_seq), cu, ks, keep_tail, _ptr(idx_out),
                                            _stream(stream)))


def structkv_gather_kv(k_src: Optional[torch.Tensor], v_src: Optional[torch.Tensor],
                       k_dst: Optional[torch.Tensor], v_dst: Optional[torch.Tensor],
                       cu_seqlens: Sequence[int], rows_per_seq: Sequence[int], idx: torch.Tensor,
                       stream=None) -> None:
    """src/dst: [G, tokens, d] views with d contiguous; K and V must share strides."""
    src = k_src if k_src is not None else v_src
    dst = k_dst if k_dst is not None else v_dst
    if v_src is not None and k_src is not None:
        assert v_src.stride() == k_src.stride() and v_dst.stride() == k_dst.stride()
    cu, rows = _host_i64(cu_seqlens), _host_i64(rows_per_seq)
    _check(_lib.structkv_gather_kv(_ptr(k_src), _ptr(v_src), src.stride(0), src.stride(1), _ptr(k_dst),
                                   _ptr(v_dst), dst.stride(0), dst.stride(1), src.shape[0], src.shape[2],
                                   src.element_size(), len(rows_per_seq), cu, rows, _ptr(idx),
                                   _stream(stream)))


def structkv_layer_step_workspace_bytes(shape: structkv_shape, batch: int, total_tokens: int) -> int:
    return int(_lib.structkv_layer_step_workspace_bytes(ctypes.byref(shape), batch, total_tokens))


def structkv_layer_step(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor],
                        cu_seqlens: Sequence[int], k_per_seq: Sequence[int], keep_tail: int,
                        indeg_out: torch.Tensor, centrality: Optional[torch.Tensor], lam: float, inv_w: float,
                        entropy_out: torch.Tensor, entropy_per_head_out: Optional[torch.Tensor],
                        idx_out: torch.Tensor, k_dst: Optional[torch.Tensor], v_dst: Optional[torch.Tensor],
                        workspace: torch.Tensor, stream=None, _entry=None) -> None:
    """k, v: [G, total, d] views sharing strides; k_dst, v_dst: [G, rows, d] views sharing strides (or None)."""
    fn = _entry or _lib.structkv_layer_step
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous()
    if v is not None:
        assert v.stride() == k.stride() and v.dtype == k.dtype
    dst = k_dst if k_dst is not None else v_dst
    if k_dst is not None and v_dst is not None:
        assert k_dst.stride() == v_dst.stride()
    cu, ks = _host_i64(cu_seqlens), _host_i64(k_per_seq)
    _check(fn(ctypes.byref(shape), _ptr(q_win), _ptr(k), _ptr(v), k.stride(0), k.stride(1),
              len(k_per_seq), cu, ks, keep_tail, _ptr(indeg_out), _ptr(centrality), lam, inv_w,
              _ptr(entropy_out), _ptr(entropy_per_head_out), _ptr(idx_out), _ptr(k_dst),
              _ptr(v_dst), dst.stride(0) if dst is not None else 0,
              dst.stride(1) if dst is not None else 0, _ptr(workspace),
              workspace.numel() * workspace.element_size(), _stream(stream)))


def structkv_layer_begin(*args, **kwargs) -> None:
    """Same arguments as structkv_layer_step; enqueues its first half."""
    structkv_layer_step(*args, _entry=_lib.structkv_layer_begin, **kwargs)


def structkv_layer_finish(shape: structkv_shape, k: torch.Tensor, v: Optional[torch.Tensor],
                          cu_seqlens: Sequence[int], k_per_seq: Sequence[int], keep_tail: int, indeg: torch.Tensor,
                          idx_out: torch.Tensor, k_dst: Optional[torch.Tensor], v_dst: Optional[torch.Tensor],
                          workspace: torch.Tensor, stream=None) -> None:
    dst = k_dst if k_dst is not None else v_dst
    cu, ks = _host_i64(cu_seqlens), _host_i64(k_per_seq)
    _check(_lib.structkv_layer_finish(ctypes.byref(shape), _ptr(k), _ptr(v), k.stride(0), k.stride(1), len(k_per_seq),
                                      cu, ks, keep_tail, _ptr(indeg), _ptr(idx_out), _ptr(k_dst), _ptr(v_dst),
                                      dst.stride(0) if dst is not None else 0,
                                      dst.stride(1) if dst is not None else 0, _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)))


def structkv_truncate_hidden(h_src: Optional[torch.Tensor], h_dst: Optional[torch.Tensor],
                             pos_src: Optional[torch.Tensor], pos_dst: Optional[torch.Tensor],
                             cu_seqlens: Sequence[int], rows_per_seq: Sequence[int], idx: torch.Tensor,
                             stream=None) -> None:
    """h_src [total, hidden], h_dst [rows, hidden] (last dim contiguous); pos_* int64 vectors or None."""
    hidden = elem = ss = ds = 0
    if h_src is not None:
        assert h_src.dim() == 2 and h_src.stride(1) == 1 and h_dst.stride(1) == 1 and h_dst.dtype == h_src.dtype
        hidden, elem, ss, ds = h_src.shape[1], h_src.element_size(), h_src.stride(0), h_dst.stride(0)
    for p in (pos_src, pos_dst):
        assert p is None or (p.dtype == torch.int64 and p.is_contiguous())
    cu, rows = _host_i64(cu_seqlens), _host_i64(rows_per_seq)
    _check(_lib.structkv_truncate_hidden(_ptr(h_src), ss, _ptr(h_dst), ds, hidden, elem, _ptr(pos_src),
                                         _ptr(pos_dst), len(rows_per_seq), cu, rows, _ptr(idx), _stream(stream)))


def structkv_block_scores(scores: torch.Tensor, cu_seqlens: Sequence[int], block_size: int,
                          block_scores_out: torch.Tensor, stream=None) -> None:
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_block_scores(_ptr(scores), len(cu_seqlens) - 1, cu, block_size, _ptr(block_scores_out),
                                      _stream(stream)))


def structkv_pivot_workspace_bytes(shape: structkv_shape, max_seq_len: int) -> int:
    return int(_lib.structkv_pivot_workspace_bytes(ctypes.byref(shape), int(max_seq_len)))


def structkv_pivot_metrics(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor, cu_seqlens: Sequence[int],
                           top_frac: float, sparsity_out: torch.Tensor, variance_out: torch.Tensor,
                           workspace: torch.Tensor, stream=None) -> None:
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous()
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_pivot_metrics(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                       len(cu_seqlens) - 1, cu, top_frac, _ptr(sparsity_out), _ptr(variance_out),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream)))


def structkv_score_layer_pivot(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor,
                               cu_seqlens: Sequence[int], top_frac: float, indeg_out: torch.Tensor,
                               entropy_out: torch.Tensor, entropy_per_head_out: Optional[torch.Tensor],
                               sparsity_out: torch.Tensor, variance_out: torch.Tensor, workspace: torch.Tensor,
                               stream=None) -> None:
    assert k.dim() == 3 and k.stride(2) == 1 and q_win.is_contiguous()
    cu = _host_i64(cu_seqlens)
    _check(_lib.structkv_score_layer_pivot(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1),
                                           len(cu_seqlens) - 1, cu, top_frac, _ptr(indeg_out), _ptr(entropy_out),
                                           _ptr(entropy_per_head_out), _ptr(sparsity_out), _ptr(variance_out),
                                           _ptr(workspace), workspace.numel() * workspace.element_size(),
                                           _stream(stream)))


def structkv_transition_scores(entropy: Sequence[float], sparsity: Sequence[float], variance: Sequence[float],
                               weights: Sequence[float] = (0.2, 0.3, 0.5)):
    """Host arithmetic (Eq. 7-9): returns (list of T_l, pivot layer L*)."""
    n = len(entropy)
    assert len(sparsity) == n and len(variance) == n
    arr = ctypes.c_double * max(n, 1)
    H, R, V, T = arr(*entropy), arr(*sparsity), arr(*variance), arr()
    ls = ctypes.c_int32(0)
    _check(_lib.structkv_transition_scores(H, R, V, n, weights[0], weights[1], weights[2], T, ctypes.byref(ls)))
    return list(T)[:n], int(ls.value)


def structkv_debug_probs(shape: structkv_shape, q_win: torch.Tensor, k: torch.Tensor, n: int,
                         probs_out: torch.Tensor, workspace: torch.Tensor, stream=None,
                         force_simt: bool = False) -> None:
    _check(_lib.structkv_debug_probs(ctypes.byref(shape), _ptr(q_win), _ptr(k), k.stride(0), k.stride(1), n,
                                     _ptr(probs_out), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream),
                                     int(bool(force_simt))))


# ---- a layer's cache in use ----------------------------------------------------------------------------------------------------

def _require(ok: bool, message: str) -> None:
    if not ok:
        raise StructKVError(STRUCTKV_ERR_INVALID_ARG, message)


def _vector(t: Optional[torch.Tensor], dtype: torch.dtype, numel: int, index: int, name: str) -> None:
    if t is not None and (t.dtype is not dtype or t.numel() != numel or t.get_device() != index or not t.is_contiguous()):
        raise StructKVError(STRUCTKV_ERR_INVALID_ARG, "%s must be a contiguous %s tensor of %d elements on the cache's GPU" % (name, dtype, numel))


def make_cache(k: torch.Tensor, v: torch.Tensor, cu_slots: Sequence[int], lens: torch.Tensor, mass: Optional[torch.Tensor] = None,
               pos: Optional[torch.Tensor] = None, missed: Optional[torch.Tensor] = None) -> structkv_cache:
    """k, v: [G, slots, d] views sharing strides, d contiguous; lens: int32 [batch]; mass fp32, pos int32: [planes, slots] (or [slots]),
    planes = 1 or G; missed: int32 [batch], zeros, where an append leaves a mark for a sequence without room.  The tensors are kept
    alive by the result; `lens` is read by the calls, whose lens_out is another tensor."""
    _require(k.dim() == 3 and v.dim() == 3 and v.shape == k.shape and v.stride() == k.stride() and v.dtype == k.dtype,
             "k and v must be [G, slots, d] views of one dtype that share shape and strides")
    _require(k.dtype in (torch.float32, torch.bfloat16), "k and v must be float32 or bfloat16")
    G, slots, d = k.shape
    _require(G >= 1 and d >= 1 and (k.stride(2) == 1 or d == 1), "k and v need a KV head, and contiguous components")
    batch = len(cu_slots) - 1
    _require(batch >= 0 and cu_slots[batch] <= slots, "cu_slots needs batch + 1 entries, at most %d" % slots)
    total = cu_slots[batch]
    planes = 1
    for t, name in ((mass, "mass"), (pos, "pos")):
        if t is not None:
            _require(t.dim() in (1, 2), "%s must be [planes, slots] or [slots]" % name)
            planes = t.shape[0] if t.dim() == 2 else 1
            _require(planes in (1, G), "%s must have one plane, or one per KV head" % name)
    index = k.get_device()
    _vector(mass, torch.float32, planes * total, index, "mass")
    _vector(pos, torch.int32, planes * total, index, "pos")
    _vector(lens, torch.int32, batch, index, "lens")
    _vector(missed, torch.int32, batch, index, "missed")
    _require(v.device == k.device and index >= 0, "the cache must be on one GPU")
    host = _host_i64(cu_slots)
    code = STRUCTKV_DTYPE_BF16 if k.dtype == torch.bfloat16 else STRUCTKV_DTYPE_F32
    c = structkv_cache(_ptr(k), _ptr(v), k.stride(0), k.stride(1), G, d, code, planes, _ptr(mass), _ptr(pos), _ptr(lens),
                       ctypes.addressof(host), batch, _ptr(missed))
    c.tensors = (k, v, lens, mass, pos, missed, host)
    c.tensor_dtype, c.device, c.index, c.slots = k.dtype, k.device, index, total
    return c


# (torch's own functions check more on every call: 1.2 us a call)
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _cache_call(fn, cache: structkv_cache, stream, *args) -> None:
    """The call on the cache's GPU: on `stream`, or on the current one of that GPU."""
    index = cache.index
    if stream is None:
        raw = _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream
    else:
        _require(getattr(stream, "device", cache.device) == cache.device, "the stream belongs to another device than the cache")
        raw = _stream(stream)
    if index == _get_device():
        status = fn(ctypes.byref(cache), *args, raw)
    else:
        with torch.cuda.device(index):
            status = fn(ctypes.byref(cache), *args, raw)
    if status:
        _check(status)


def _query_strides(cache: structkv_cache, n_q_heads: int, q: torch.Tensor, new: int):
    if q.shape != (new, n_q_heads, cache.head_dim) or q.dtype is not cache.tensor_dtype or q.get_device() != cache.index:
        raise StructKVError(STRUCTKV_ERR_INVALID_ARG, "q must be [new tokens, n_q_heads, head_dim], of the cache's dtype and GPU")
    st, sh, sc = q.stride()
    _require(sc == 1 or cache.head_dim == 1, "q must have contiguous components")
    return st, sh


def _workspace(cache: structkv_cache, workspace: torch.Tensor) -> int:
    _require(workspace.get_device() == cache.index and workspace.is_contiguous(), "workspace must be contiguous and on the cache's GPU")
    return workspace.numel() * workspace.element_size()


def structkv_cache_workspace_bytes(cache: structkv_cache, n_q_heads: int, new_tokens: int) -> int:
    return int(_lib.structkv_cache_workspace_bytes(ctypes.byref(cache), n_q_heads, new_tokens))


def structkv_cache_append(cache: structkv_cache, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: Sequence[int],
                          lens_out: torch.Tensor, pos_new: Optional[torch.Tensor] = None, mass_new: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """k_new, v_new: [G, new, d] views sharing strides; pos_new int32, mass_new fp32: [new] for all planes, or [planes, new]."""
    _require(len(cu_new) == cache.batch + 1, "cu_new needs batch + 1 entries")
    new = cu_new[cache.batch]
    shape, strides = k_new.shape, k_new.stride()
    _require(len(shape) == 3 and shape[0] == cache.n_kv_heads and shape[1] >= new and shape[2] == cache.head_dim and v_new.shape == shape and
             v_new.stride() == strides and (strides[2] == 1 or shape[2] == 1) and k_new.dtype is cache.tensor_dtype and
             v_new.dtype is cache.tensor_dtype and k_new.get_device() == cache.index and v_new.get_device() == cache.index,
             "k_new and v_new must be [G, new tokens, head_dim] views sharing strides, of the cache's dtype and GPU, with contiguous components")
    plane = 0
    for t, dtype, name in ((pos_new, torch.int32, "pos_new"), (mass_new, torch.float32, "mass_new")):
        if t is not None:
            rows = t.dim()
            _vector(t, dtype, new if rows == 1 else new * cache.planes, cache.index, name)
            _require(rows == 1 or t.shape == (cache.planes, new), "pos_new and mass_new must be [new tokens] or [planes, new tokens]")
            plane = new if rows == 2 else 0
    _require(pos_new is None or mass_new is None or pos_new.dim() == mass_new.dim(), "pos_new and mass_new must have the same shape")
    _vector(lens_out, torch.int32, cache.batch, cache.index, "lens_out")
    _cache_call(_lib.structkv_cache_append, cache, stream, k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1], _host_i64(cu_new),
                _ptr(pos_new), _ptr(mass_new), plane, lens_out.data_ptr())


def structkv_cache_attend(cache: structkv_cache, n_q_heads: int, q: torch.Tensor, cu_new: Sequence[int], out: torch.Tensor,
                          lse_out: torch.Tensor, workspace: torch.Tensor, tree_mask: Optional[torch.Tensor] = None, scale: float = 0.0,
                          softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, lam: float = 0.0, stream=None) -> None:
    """q: [new, H_q, d] view with d contiguous; out [new, H_q, d] and lse_out fp32 [new, H_q] contiguous; tree_mask: int64 [new], whose
    64 bits are the fresh tokens that a token sees; slopes: fp32 [H_q]."""
    _require(len(cu_new) == cache.batch + 1, "cu_new needs batch + 1 entries")
    new = cu_new[cache.batch]
    st, sh = _query_strides(cache, n_q_heads, q, new)
    _vector(out, cache.tensor_dtype, new * n_q_heads * cache.head_dim, cache.index, "out")
    _vector(lse_out, torch.float32, new * n_q_heads, cache.index, "lse_out")
    _vector(tree_mask, torch.int64, new, cache.index, "tree_mask")
    _vector(slopes, torch.float32, n_q_heads, cache.index, "slopes")
    _cache_call(_lib.structkv_cache_attend, cache, stream, n_q_heads, scale, softcap, _ptr(slopes), q.data_ptr(), st, sh, _host_i64(cu_new),
                _ptr(tree_mask), lam, out.data_ptr(), lse_out.data_ptr(), workspace.data_ptr(), _workspace(cache, workspace))


def structkv_cache_accept(cache: structkv_cache, n_q_heads: int, q: Optional[torch.Tensor], lse: Optional[torch.Tensor],
                          cu_new: Sequence[int], lens_out: torch.Tensor, path: Optional[torch.Tensor] = None,
                          n_accept: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None, scale: float = 0.0,
                          softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, lam: float = 0.0, stream=None) -> None:
    """q, lse, tree_mask, scale, softcap, slopes as in the attend call (q and lse may be None with lam = 0); path: int32 [new], the accepted
    tokens first in each sequence's part; n_accept: int32 [batch]."""
    _require(len(cu_new) == cache.batch + 1, "cu_new needs batch + 1 entries")
    new = cu_new[cache.batch]
    st, sh = _query_strides(cache, n_q_heads, q, new) if q is not None else (0, 0)
    _vector(lse, torch.float32, new * n_q_heads, cache.index, "lse")
    _vector(tree_mask, torch.int64, new, cache.index, "tree_mask")
    _vector(slopes, torch.float32, n_q_heads, cache.index, "slopes")
    _vector(path, torch.int32, new, cache.index, "path")
    _vector(n_accept, torch.int32, cache.batch, cache.index, "n_accept")
    _vector(lens_out, torch.int32, cache.batch, cache.index, "lens_out")
    _cache_call(_lib.structkv_cache_accept, cache, stream, n_q_heads, scale, softcap, _ptr(slopes), _ptr(q), st, sh, _ptr(lse),
                _host_i64(cu_new), _ptr(tree_mask), _ptr(path), _ptr(n_accept), lam, lens_out.data_ptr())


def structkv_cache_evict(cache: structkv_cache, scores: Optional[torch.Tensor], budget: Sequence[int], keep_tail: int,
                         lens_out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """scores: fp32 [planes, slots], or None for the cache's mass."""
    _require(len(budget) == cache.batch, "budget needs batch entries")
    _vector(scores, torch.float32, cache.planes * cache.slots, cache.index, "scores")
    _vector(lens_out, torch.int32, cache.batch, cache.index, "lens_out")
    _cache_call(_lib.structkv_cache_evict, cache, stream, _ptr(scores), _host_i64(budget), keep_tail, lens_out.data_ptr(), workspace.data_ptr(),
                _workspace(cache, workspace))
