"""ctypes binding of libfocus_hip.so: argument marshalling only.

Every function has the name of the C entry point it wraps (include/focus.h) minus the `focus_` prefix of
the status code: it takes torch CUDA tensors, passes their device pointers, sizes and strides through, and
raises FocusError on a non-zero status.  No step of the method runs in Python, and there is no fallback:
if the HIP library is not built, importing this module's `lib()` fails.
"""
from __future__ import annotations

import ctypes as C
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfocus_hip.so")

FOCUS_OK, FOCUS_EINVAL, FOCUS_EUNSUPPORTED, FOCUS_EWORKSPACE, FOCUS_ELAUNCH = 0, -1, -2, -3, -4
FN_BLOCK_SCORES, FN_FIND_SINKS, FN_SPARSE_ATTN, FN_SPARSE_LAYER, FN_PROBE_LAYER, FN_QUANT_ATTN, FN_QUANT_LAYER = 1, 2, 3, 4, 5, 6, 7

EXPORTS = ("focus_select_queries", "focus_expand_groups", "focus_block_means", "focus_block_scores", "focus_find_sinks", "focus_select_and_find_sinks",
           "focus_sparse_attn",
           "focus_sparse_layer", "focus_sparse_layer_static", "focus_block_partials", "focus_top_blocks", "focus_probe_layer", "focus_refresh_attn", "focus_cache_refresh", "focus_block_entry",
           "focus_token_confidence", "focus_token_confidence_workspace", "focus_cache_update", "focus_update_sparse_layer",
           "focus_quant_update", "focus_quant_refresh", "focus_quant_read", "focus_quant_attn", "focus_quant_layer",
           "focus_sample_tokens", "focus_sample_tokens_workspace",
           "focus_rotary", "focus_helper_rotary", "focus_paged_append", "focus_paged_attn", "focus_paged_attn_workspace",
           "focus_token_logprobs", "focus_token_logprobs_workspace",
           "focus_workspace_bytes", "focus_helper_k", "focus_helper_n_keep", "focus_helper_n_sink", "focus_last_error",
           "focus_version")


class FocusError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"focus status {status}: {message}")
        self.status = status


class Shape(C.Structure):
    """Mirror of `focus_shape`."""
    _fields_ = [("n_heads", C.c_int32), ("head_dim", C.c_int32), ("n_ctx", C.c_int32), ("n_resp", C.c_int32),
                ("block", C.c_int32), ("n_gen", C.c_int32),
                ("q_stride_h", C.c_int64), ("q_stride_n", C.c_int64), ("k_stride_h", C.c_int64), ("k_stride_n", C.c_int64),
                ("v_stride_h", C.c_int64), ("v_stride_n", C.c_int64), ("o_stride_h", C.c_int64), ("o_stride_n", C.c_int64)]


class QuantCache(C.Structure):
    """Mirror of `focus_quant_cache`."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("exp_stride_h", C.c_int64), ("exp_stride_n", C.c_int64)]


class Rotation(C.Structure):
    """Mirror of `focus_rotation`."""
    device = None  # set by make_rotation; one that a caller filled in by hand is taken as it is, and so the next two
    _fields_ = [("freq", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_double)]


class PagedCache(C.Structure):
    """Mirror of `focus_paged_cache`."""
    device = None
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("k_stride_p", C.c_int64), ("k_stride_h", C.c_int64), ("k_stride_n", C.c_int64),
                ("v_stride_p", C.c_int64), ("v_stride_h", C.c_int64), ("v_stride_n", C.c_int64),
                ("exp_stride_p", C.c_int64), ("exp_stride_h", C.c_int64), ("exp_stride_n", C.c_int64),
                ("n_pages", C.c_int32), ("page", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32)]


class PagedBatch(C.Structure):
    """Mirror of `focus_paged_batch`."""
    device = None
    _fields_ = [("seq_len", C.c_void_p), ("page_table", C.c_void_p), ("row_start", C.c_void_p), ("positions", C.c_void_p),
                ("table_stride", C.c_int64), ("table_width", C.c_int32), ("n_req", C.c_int32), ("max_rows", C.c_int32), ("n_rows", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (python -m paper_2602_02159_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is not built: run `python -m paper_2602_02159_amd.build`")
        L = C.CDLL(LIB_PATH)
        p, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        sp = C.POINTER(Shape)
        L.focus_select_queries.argtypes = [p, p, i32, i32, i32, i32, i32, p, p, i32, p, p]
        L.focus_expand_groups.argtypes = [p, i32, p, i32, p, i32, i32, p, p, p, p]
        L.focus_block_means.argtypes = [p, sp, p, p]
        L.focus_block_scores.argtypes = [p, p, p, i32, p, p, sp, i32, p, p, p, sz, p]
        L.focus_find_sinks.argtypes = [p, p, p, i32, p, sp, i32, p, p, p, sz, p]
        L.focus_select_and_find_sinks.argtypes = [p, p, i32, i32, i32, i32, p, p, i32, p, p, p, sp, i32, p, p, p, sz, p]
        L.focus_sparse_attn.argtypes = [p, p, p, i32, p, p, sp, p, i32, p, i32, p, p, p, sz, p]
        L.focus_sparse_layer.argtypes = [p, p, p, p, i32, i32, p, p, p, sp, i32, p, i32, p, p, p, p, p, sz, p]
        L.focus_sparse_layer_static.argtypes = [p, p, p, p, i32, i32, p, p, p, sp, i32, p, i32, p, p, p, p, p]
        L.focus_probe_layer.argtypes = [p, p, p, i32, p, p, sp, i32, p, p, p, p, p, sz, p]
        L.focus_refresh_attn.argtypes = [p, p, p, sp, p, p, p]
        L.focus_cache_refresh.argtypes = [p, p, sp, p, p, C.c_int64, C.c_int64, p, p]
        L.focus_block_entry.argtypes = [p, p, sp, p, p, p, C.c_int64, C.c_int64, p, p, p, p]
        L.focus_token_confidence.argtypes = [p, C.c_int64, p, i32, i32, p, p, p, sz, p]
        L.focus_token_confidence_workspace.argtypes = [i32, i32]
        L.focus_token_confidence_workspace.restype = sz
        L.focus_cache_update.argtypes = [p, p, sp, p, p, C.c_int64, C.c_int64, p, p, i32, i32, p]
        L.focus_update_sparse_layer.argtypes = [p, p, p, p, C.c_int64, C.c_int64, i32, p, p, p, p, i32, i32, p, sp, i32, p, i32, p, p, p, p, p, sz, p]
        L.focus_block_partials.argtypes = [p, p, p, i32, p, p, sp, p, p]
        L.focus_top_blocks.argtypes = [p, i32, p, i32, i32, i32, p, p, p]
        qp = C.POINTER(QuantCache)
        L.focus_quant_update.argtypes = [qp, sp, p, p, C.c_int64, C.c_int64, p, p, i32, i32, p]
        L.focus_quant_refresh.argtypes = [qp, sp, p, p, C.c_int64, C.c_int64, p, p]
        L.focus_quant_read.argtypes = [qp, sp, i32, i32, p, p, C.c_int64, C.c_int64, p]
        L.focus_quant_attn.argtypes = [p, p, p, i32, qp, sp, p, i32, p, i32, p, p, p, sz, p]
        L.focus_quant_layer.argtypes = [p, p, p, p, i32, i32, qp, p, sp, i32, p, i32, p, p, p, p, p, sz, p]
        L.focus_sample_tokens.argtypes = [p, i32, C.c_int64, p, p, p, p, p, p, i32, i32, p, p, p, p, sz, p]
        L.focus_sample_tokens_workspace.argtypes = [i32, i32]
        L.focus_sample_tokens_workspace.restype = sz
        i64, rp, cp, bp = C.c_int64, C.POINTER(Rotation), C.POINTER(PagedCache), C.POINTER(PagedBatch)
        L.focus_rotary.argtypes = [p, i64, i64, p, i64, i64, i32, i32, i32, p, i32, rp, p]
        L.focus_helper_rotary.argtypes = [C.c_double, i32, C.c_double, i32, C.c_double, C.c_double, C.POINTER(C.c_double)]
        L.focus_paged_append.argtypes = [cp, bp, p, p, i64, i64, rp, p, i64, i64, p, i64, i64, i32, p]
        L.focus_paged_attn.argtypes = [p, i64, i64, i32, cp, bp, i32, p, i64, i64, p, p, sz, p]
        L.focus_paged_attn_workspace.argtypes = [cp, bp, i32]
        L.focus_paged_attn_workspace.restype = sz
        L.focus_token_logprobs.argtypes = [p, i32, i64, p, p, i32, i32, i32, p, p, p, p, p, sz, p]
        L.focus_token_logprobs_workspace.argtypes = [i32, i32, i32]
        L.focus_token_logprobs_workspace.restype = sz
        for name in ("focus_rotary", "focus_helper_rotary", "focus_paged_append", "focus_paged_attn", "focus_token_logprobs",
                     "focus_sample_tokens", "focus_quant_update", "focus_quant_refresh", "focus_quant_read", "focus_quant_attn", "focus_quant_layer",
                     "focus_select_queries", "focus_expand_groups", "focus_block_means", "focus_block_scores", "focus_find_sinks",
                     "focus_select_and_find_sinks", "focus_sparse_attn", "focus_sparse_layer", "focus_sparse_layer_static", "focus_block_partials", "focus_top_blocks",
                     "focus_probe_layer", "focus_refresh_attn", "focus_token_confidence", "focus_cache_update", "focus_update_sparse_layer", "focus_cache_refresh", "focus_block_entry"):
            getattr(L, name).restype = C.c_int
        L.focus_workspace_bytes.argtypes = [i32, sp, i32, i32, i32]
        L.focus_workspace_bytes.restype = sz
        L.focus_helper_k.argtypes = [C.c_double, i32]
        L.focus_helper_k.restype = i32
        L.focus_helper_n_keep.argtypes = [C.c_double, i32]
        L.focus_helper_n_keep.restype = i32
        L.focus_helper_n_sink.argtypes = [C.c_double, i32]
        L.focus_helper_n_sink.restype = i32
        L.focus_last_error.restype = C.c_char_p
        L.focus_version.restype = C.c_char_p
        _lib = L
    return _lib


def last_error() -> str:
    return lib().focus_last_error().decode()


def _check(status: int) -> None:
    if status != FOCUS_OK:
        raise FocusError(status, last_error())


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _raw_stream(device: int) -> int:
    # the handle of torch.cuda.current_stream() without the object around it: 0.1 us instead of 2.7, a quarter of a short call's host time
    try:
        return torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:  # (not part of torch's interface)
        return torch.cuda.current_stream(device).cuda_stream


def _stream() -> int:
    return _raw_stream(torch.cuda.current_device())


def _device_of(t: torch.Tensor, name: str = "tensors") -> int:
    """The current device: kernels run there, so `t` has to be there."""
    device = torch.cuda.current_device()
    if t.get_device() != device:
        raise ValueError(f"{name} on {t.device}, but the current device is cuda:{device}")
    return device


def _need(t: torch.Tensor, dtype, name: str) -> None:
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name}: expected a CUDA tensor of {dtype}, got {t.dtype} on {t.device}")


def make_shape(q: torch.Tensor, k: torch.Tensor | None, v: torch.Tensor | None, n_ctx: int, block: int,
               out: torch.Tensor | None = None) -> Shape:
    """focus_shape from [H, rows, d] tensors (any strides with a unit innermost stride)."""
    H, n_gen, d = q.shape
    s = Shape()
    s.n_heads, s.head_dim, s.n_gen, s.block, s.n_ctx = H, d, n_gen, block, n_ctx
    ref = k if k is not None else v
    s.n_resp = (ref.shape[1] - n_ctx) if ref is not None else 0
    for name, t in (("q", q), ("k", k), ("v", v), ("o", out)):
        if t is None:
            continue
        if t.stride(2) != 1:
            raise ValueError(f"{name}: innermost stride must be 1")
        setattr(s, f"{name}_stride_h", t.stride(0))
        setattr(s, f"{name}_stride_n", t.stride(1))
    return s


def workspace_bytes(fn: int, shape: Shape, max_active: int = 1, n_keep: int = 0, n_sink: int = 0) -> int:
    return int(lib().focus_workspace_bytes(fn, C.byref(shape), max_active, n_keep, n_sink))


def helper_k(rho: float, n_unmask: int) -> int:
    return int(lib().focus_helper_k(rho, n_unmask))


def helper_n_keep(alpha: float, n_blocks: int) -> int:
    return int(lib().focus_helper_n_keep(alpha, n_blocks))


def helper_n_sink(frac: float, n_ctx: int) -> int:
    return int(lib().focus_helper_n_sink(frac, n_ctx))


def select_queries(conf, masked, k: int, window: int, lo: int, hi: int, focus_idx, active_idx, counts) -> None:
    _need(conf, torch.float32, "conf")
    _check(lib().focus_select_queries(_ptr(conf), _ptr(masked), conf.numel(), k, window, lo, hi, _ptr(focus_idx),
                                      _ptr(active_idx), active_idx.numel(), _ptr(counts), _stream()))


def expand_groups(focus_idx, active_idx, counts, n_gen: int, group: int, focus_out, active_out, counts_out) -> None:
    """Index lists of select_queries -> lists of rows g * n_gen + i of the [H_kv, group * n_gen, d] view of Q."""
    _check(lib().focus_expand_groups(_ptr(focus_idx), focus_idx.numel(), _ptr(active_idx), active_idx.numel(), _ptr(counts),
                                     n_gen, group, _ptr(focus_out), _ptr(active_out), _ptr(counts_out), _stream()))


def block_means(k, shape: Shape, kbar) -> None:
    _need(k, torch.bfloat16, "K")
    _check(lib().focus_block_means(_ptr(k), C.byref(shape), _ptr(kbar), _stream()))


def block_scores(q, focus_idx, counts, k, kbar, shape: Shape, n_keep: int, scores, kept_blocks, workspace) -> None:
    _need(q, torch.bfloat16, "Q")
    _check(lib().focus_block_scores(_ptr(q), _ptr(focus_idx), _ptr(counts), focus_idx.numel(), _ptr(k), _ptr(kbar),
                                    C.byref(shape), n_keep, _ptr(scores), _ptr(kept_blocks), _ptr(workspace),
                                    0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def block_partials(q, focus_idx, counts, k, kbar, shape: Shape, partials) -> None:
    _need(q, torch.bfloat16, "Q")
    _need(partials, torch.float32, "partials")
    _check(lib().focus_block_partials(_ptr(q), _ptr(focus_idx), _ptr(counts), focus_idx.numel(), _ptr(k), _ptr(kbar),
                                      C.byref(shape), _ptr(partials), _stream()))


def top_blocks(partials, counts, n_focus_max: int, n_keep: int, scores, kept_blocks) -> None:
    _need(partials, torch.float32, "partials")
    n_parts, n_blocks = partials.shape
    _check(lib().focus_top_blocks(_ptr(partials), n_parts, _ptr(counts), n_focus_max, n_blocks, n_keep, _ptr(scores),
                                  _ptr(kept_blocks), _stream()))


def find_sinks(q, active_idx, counts, k, shape: Shape, n_sink: int, col_mass, sink_idx, workspace) -> None:
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _check(lib().focus_find_sinks(_ptr(q), _ptr(active_idx), _ptr(counts), active_idx.numel(), _ptr(k), C.byref(shape),
                                  n_sink, _ptr(col_mass), _ptr(sink_idx), _ptr(workspace),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def select_and_find_sinks(conf, masked, k_focus: int, window: int, lo: int, hi: int, focus_idx, active_idx, counts, q, k, shape: Shape,
                          n_sink: int, col_mass, sink_idx, workspace) -> None:
    """select_queries followed by find_sinks with its lists."""
    _need(conf, torch.float32, "conf")
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _check(lib().focus_select_and_find_sinks(_ptr(conf), _ptr(masked), k_focus, window, lo, hi, _ptr(focus_idx), _ptr(active_idx),
                                             active_idx.numel(), _ptr(counts), _ptr(q), _ptr(k), C.byref(shape), n_sink, _ptr(col_mass),
                                             _ptr(sink_idx), _ptr(workspace),
                                             0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def sparse_attn(q, active_idx, counts, k, v, shape: Shape, kept_blocks, n_keep: int, sink_idx, n_sink: int, out, lse,
                workspace) -> None:
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _need(v, torch.bfloat16, "V")
    _need(out, torch.bfloat16, "out")
    _check(lib().focus_sparse_attn(_ptr(q), _ptr(active_idx), _ptr(counts), active_idx.numel(), _ptr(k), _ptr(v),
                                   C.byref(shape), _ptr(kept_blocks), n_keep, _ptr(sink_idx), n_sink, _ptr(out), _ptr(lse),
                                   _ptr(workspace),
                                   0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def probe_layer(q, active_idx, counts, k, v, shape: Shape, n_sink: int, out, lse, col_mass, sink_idx, workspace) -> None:
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _need(v, torch.bfloat16, "V")
    _need(out, torch.bfloat16, "out")
    _check(lib().focus_probe_layer(_ptr(q), _ptr(active_idx), _ptr(counts), active_idx.numel(), _ptr(k), _ptr(v),
                                   C.byref(shape), n_sink, _ptr(out), _ptr(lse), _ptr(col_mass), _ptr(sink_idx),
                                   _ptr(workspace),
                                   0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def refresh_attn(q, k, v, shape: Shape, out, lse) -> None:
    """Dense attention of every row of q over every row of k / v (block-entry refresh)."""
    for t, name in ((q, "Q"), (k, "K"), (v, "V"), (out, "out")):
        _need(t, torch.bfloat16, name)
    _check(lib().focus_refresh_attn(_ptr(q), _ptr(k), _ptr(v), C.byref(shape), _ptr(out), _ptr(lse), _stream()))


def token_confidence_workspace(n_rows: int, vocab: int) -> int:
    return int(lib().focus_token_confidence_workspace(n_rows, vocab))


def token_confidence(logits, masked, tokens, conf, workspace) -> None:
    """logits bf16 [n_rows, vocab] (row stride a multiple of 8); workspace of token_confidence_workspace() bytes."""
    _need(logits, torch.bfloat16, "logits")
    _need(conf, torch.float32, "conf")
    if logits.stride(1) != 1:
        raise ValueError("logits: innermost stride must be 1")
    _check(lib().focus_token_confidence(_ptr(logits), logits.stride(0), _ptr(masked), logits.shape[0], logits.shape[1],
                                        _ptr(tokens), _ptr(conf), _ptr(workspace),
                                        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def sample_tokens_workspace(n_rows: int, vocab: int) -> int:
    return int(lib().focus_sample_tokens_workspace(n_rows, vocab))


def sample_tokens(logits, masked, uniform, temperature, top_k, top_p, min_p, tokens, conf, prob, workspace) -> None:
    """logits bf16 or fp32 [n_rows, vocab] (rows 16-byte aligned); uniform, temperature, top_p, min_p fp32 and top_k int32 [n_rows] (all
    but uniform may be None, as may masked, conf and prob); workspace of sample_tokens_workspace() bytes."""
    if not logits.is_cuda or logits.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"logits: expected a CUDA tensor of bfloat16 or float32, got {logits.dtype} on {logits.device}")
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits: expected [n_rows, vocab], innermost stride 1")
    device = _device_of(logits)
    rows, vocab = logits.shape[:1], logits.shape[1]
    stride = logits.stride(0) if rows[0] > 1 else (vocab + 7) // 8 * 8  # (of one row any will do)
    for t, dtype, name in ((uniform, torch.float32, "uniform"), (temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"),
                           (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p"), (tokens, torch.int32, "tokens"), (conf, torch.float32, "conf"),
                           (prob, torch.float32, "prob")):
        if t is not None and not (t.dtype == dtype and t.get_device() == device and t.shape == rows and t.is_contiguous()):
            _need(t, dtype, name)
            _device_of(t, name)
            if t.shape != rows or not t.is_contiguous():
                raise ValueError(f"{name}: expected {rows[0]} values next to each other, got shape {tuple(t.shape)}, strides {t.stride()}")
    if masked is not None and (masked.get_device() != device or masked.element_size() != 1 or masked.shape != rows or not masked.is_contiguous()):
        raise ValueError(f"masked: expected {rows[0]} bytes on cuda:{device}, got {masked.dtype}, shape {tuple(masked.shape)} on {masked.device}")
    _check(lib().focus_sample_tokens(_ptr(logits), int(logits.dtype == torch.float32), stride, _ptr(masked), _ptr(uniform), _ptr(temperature),
                                     _ptr(top_k), _ptr(top_p), _ptr(min_p), rows[0], vocab, _ptr(tokens), _ptr(conf), _ptr(prob),
                                     _ptr(workspace), _space(workspace, device), _raw_stream(device)))


def cache_update(k_cache, v_cache, shape: Shape, k_new, v_new, active_idx, counts, row_base: int) -> None:
    """k_cache, v_cache bf16 [H, M+N, d] (strides from `shape`), k_new, v_new bf16 [H, max_active, d]."""
    for t, name in ((k_cache, "K_cache"), (v_cache, "V_cache"), (k_new, "K_new"), (v_new, "V_new")):
        _need(t, torch.bfloat16, name)
    if k_new.stride() != v_new.stride() or k_new.stride(2) != 1:
        raise ValueError("K_new and V_new must share their strides, innermost 1")
    _check(lib().focus_cache_update(_ptr(k_cache), _ptr(v_cache), C.byref(shape), _ptr(k_new), _ptr(v_new), k_new.stride(0),
                                    k_new.stride(1), _ptr(active_idx), _ptr(counts), active_idx.numel(), row_base, _stream()))


def cache_refresh(k_cache, v_cache, shape: Shape, k_new, v_new, kbar) -> None:
    """All rows of k_cache / v_cache bf16 [H, M+N, d] take k_new / v_new; kbar fp32 [H, n_b, d] (or None) gets the block means."""
    for t, name in ((k_cache, "K_cache"), (v_cache, "V_cache"), (k_new, "K_new"), (v_new, "V_new")):
        _need(t, torch.bfloat16, name)
    if kbar is not None:
        _need(kbar, torch.float32, "kbar")
    if k_new.stride() != v_new.stride() or k_new.stride(2) != 1:
        raise ValueError("K_new and V_new must share their strides, innermost 1")
    _check(lib().focus_cache_refresh(_ptr(k_cache), _ptr(v_cache), C.byref(shape), _ptr(k_new), _ptr(v_new), k_new.stride(0),
                                     k_new.stride(1), _ptr(kbar), _stream()))


def block_entry(k_cache, v_cache, shape: Shape, q, k_new, v_new, kbar, out, lse) -> None:
    """cache_refresh and refresh_attn of one layer in one call; k_new and v_new share their strides."""
    assert k_new.stride() == v_new.stride() and k_new.stride(2) == 1
    for t, name in ((q, "Q"), (k_new, "K"), (v_new, "V")):
        _need(t, torch.bfloat16, name)
    _check(lib().focus_block_entry(_ptr(k_cache), _ptr(v_cache), C.byref(shape), _ptr(q), _ptr(k_new), _ptr(v_new), k_new.stride(0),
                                   k_new.stride(1), _ptr(kbar), _ptr(out), _ptr(lse), _stream()))


def sparse_layer(q, focus_idx, active_idx, counts, k, v, kbar, shape: Shape, n_keep: int, sink_idx, n_sink: int, scores,
                 kept_blocks, out, lse, workspace) -> None:
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _need(v, torch.bfloat16, "V")
    _need(out, torch.bfloat16, "out")
    _check(lib().focus_sparse_layer(_ptr(q), _ptr(focus_idx), _ptr(active_idx), _ptr(counts), focus_idx.numel(),
                                    active_idx.numel(), _ptr(k), _ptr(v), _ptr(kbar), C.byref(shape), n_keep, _ptr(sink_idx),
                                    n_sink, _ptr(scores), _ptr(kept_blocks), _ptr(out), _ptr(lse), _ptr(workspace),
                                    0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def update_sparse_layer(k_cache, v_cache, k_new, v_new, row_base: int, q, focus_idx, active_idx, counts, kbar, shape: Shape, n_keep: int,
                        sink_idx, n_sink: int, scores, kept_blocks, out, lse, workspace) -> None:
    """cache_update and sparse_layer of one layer in one call; k_new and v_new share their strides."""
    for t, name in ((k_cache, "K_cache"), (v_cache, "V_cache"), (k_new, "K_new"), (v_new, "V_new"), (q, "Q"), (out, "out")):
        _need(t, torch.bfloat16, name)
    if k_new.stride() != v_new.stride() or k_new.stride(2) != 1:
        raise ValueError("K_new and V_new must share their strides, innermost 1")
    _check(lib().focus_update_sparse_layer(_ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new), k_new.stride(0), k_new.stride(1), row_base,
                                           _ptr(q), _ptr(focus_idx), _ptr(active_idx), _ptr(counts), focus_idx.numel(), active_idx.numel(),
                                           _ptr(kbar), C.byref(shape), n_keep, _ptr(sink_idx), n_sink, _ptr(scores), _ptr(kept_blocks),
                                           _ptr(out), _ptr(lse), _ptr(workspace),
                                           0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def sparse_layer_static(q, focus_idx, active_idx, counts, k, v, kbar, shape: Shape, n_keep: int, sink_idx, n_sink: int, scores,
                        kept_blocks, out, lse) -> None:
    """focus_sparse_layer without a workspace argument: the library's built-in scratch array is used; nothing is allocated."""
    _need(q, torch.bfloat16, "Q")
    _need(k, torch.bfloat16, "K")
    _need(v, torch.bfloat16, "V")
    _need(out, torch.bfloat16, "out")
    _check(lib().focus_sparse_layer_static(_ptr(q), _ptr(focus_idx), _ptr(active_idx), _ptr(counts), focus_idx.numel(),
                                           active_idx.numel(), _ptr(k), _ptr(v), _ptr(kbar), C.byref(shape), n_keep,
                                           _ptr(sink_idx), n_sink, _ptr(scores), _ptr(kept_blocks), _ptr(out), _ptr(lse),
                                           _stream()))


def make_quant_cache(k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor) -> QuantCache:
    """focus_quant_cache from the codes uint8 [H, M+N, d] (their strides go into the shape: make_shape takes them for k and v) and
    the exponent bytes uint8 [H, M+N], which share their strides.  The tensors have to outlive the description."""
    for t, name in ((k, "k"), (v, "v"), (k_exp, "k_exp"), (v_exp, "v_exp")):
        _need(t, torch.uint8, name)
    if k.dim() != 3 or k.shape != v.shape or k_exp.shape != k.shape[:2] or v_exp.shape != k.shape[:2]:
        raise ValueError("codes [H, rows, d] and exponents [H, rows] must agree")
    if k.stride(2) != 1 or v.stride(2) != 1:
        raise ValueError("codes: innermost stride must be 1")
    if k_exp.stride() != v_exp.stride():
        raise ValueError("k_exp and v_exp must share their strides")
    if not k.get_device() == v.get_device() == k_exp.get_device() == v_exp.get_device():
        raise ValueError("codes and exponents must be on one device")
    cache = QuantCache(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), k_exp.stride(0), k_exp.stride(1))
    cache.sizes, cache.strides, cache.device, cache.fits = tuple(k.shape), (k.stride()[:2], v.stride()[:2]), k.get_device(), None
    return cache


# What the calls over such a cache check: that no kernel leaves a tensor.  A comparison each where everything is as it should be, since a step's calls
# are a few microseconds long; what exactly is wrong, or only larger than it needs to be, is told in functions of their own.
def _strides_fit(sizes, strides, stride_h: int, stride_n: int) -> bool:
    """Whether these are the strides of [heads, rows, ...] (that of one head or one row means nothing)."""
    return (strides[0] == stride_h or sizes[0] == 1) and (strides[1] == stride_n or sizes[1] == 1)


def _check_shape(cache: QuantCache, s: Shape, device: int) -> None:
    """Cache and shape belong together (a cache that a caller filled in by hand is taken as it is)."""
    sizes = getattr(cache, "sizes", None)
    if sizes is None:
        return
    k, v = cache.strides
    if (sizes != (s.n_heads, s.n_ctx + s.n_resp, s.head_dim) or not _strides_fit(sizes, k, s.k_stride_h, s.k_stride_n)
            or not _strides_fit(sizes, v, s.v_stride_h, s.v_stride_n)):
        raise ValueError(f"shape and cache do not agree: the codes are {list(sizes)}, strides {k} and {v}")
    if cache.device != device:
        raise ValueError(f"cache on cuda:{cache.device}, but the current device is cuda:{device}")
    cache.fits = (bytes(s), device)


def _quant_device(cache: QuantCache, s: Shape, t: torch.Tensor) -> int:
    """The current device, which a call's first tensor and its cache have to be on."""
    device = _device_of(t)
    if getattr(cache, "fits", None) != (bytes(s), device):
        _check_shape(cache, s, device)
    return device


def _check_rows(device: int, *expected) -> None:
    """bf16 tensors of at least these sizes, innermost stride 1."""
    for t, name, sizes in expected:
        if t.dtype != torch.bfloat16 or t.get_device() != device:
            raise TypeError(f"{name}: expected a tensor of torch.bfloat16 on cuda:{device}, got {t.dtype} on {t.device}")
        if t.dim() != 3 or any(n < least for n, least in zip(t.shape, sizes)) or t.stride(2) != 1:
            raise ValueError(f"{name}: expected {list(sizes)}, innermost stride 1, got {list(t.shape)}, strides {t.stride()}")


def _check_pair(device: int, a: torch.Tensor, b: torch.Tensor, names: str, sizes) -> None:
    """Two such tensors with common strides."""
    strides = a.stride()
    if not (a.shape == sizes == b.shape and strides == b.stride() and strides[-1] == 1 and a.dtype == b.dtype == torch.bfloat16 and b.get_device() == device):
        _check_rows(device, (a, "K_" + names, sizes), (b, "V_" + names, sizes))
        if strides != b.stride():
            raise ValueError(f"K_{names} and V_{names} must share their strides")


def _check_values(device: int, *expected) -> None:
    """At least so many values next to each other (None where none are needed)."""
    for t, name, dtype, least in expected:
        if t is None:
            if least > 0:
                raise ValueError(f"{name}: expected {least} values, got None")
        elif not (t.dtype == dtype and t.get_device() == device and t.numel() >= least and t.is_contiguous()):
            if t.dtype != dtype or t.get_device() != device:
                raise TypeError(f"{name}: expected a tensor of {dtype} on cuda:{device}, got {t.dtype} on {t.device}")
            raise ValueError(f"{name}: expected {least} values next to each other, got shape {list(t.shape)}, strides {t.stride()}")


def _space(workspace: torch.Tensor | None, device: int) -> int:
    """Bytes of a workspace."""
    if workspace is None:
        return 0
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected memory without gaps on cuda:{device}, got strides {workspace.stride()} on {workspace.device}")
    return workspace.numel() * workspace.element_size()


def quant_update(cache: QuantCache, shape: Shape, k_new, v_new, active_idx, counts, row_base: int) -> None:
    """cache_update into a quantised cache: k_new, v_new bf16 [H, max_active, d]."""
    device, slots = _quant_device(cache, shape, k_new), active_idx.numel()
    _check_pair(device, k_new, v_new, "new", (shape.n_heads, slots, shape.head_dim))
    _check_values(device, (active_idx, "active_idx", torch.int32, 0), (counts, "counts", torch.int32, 0 if counts is None else 2))
    _check(lib().focus_quant_update(C.byref(cache), C.byref(shape), _ptr(k_new), _ptr(v_new), k_new.stride(0), k_new.stride(1), _ptr(active_idx),
                                    _ptr(counts), slots, row_base, _raw_stream(device)))


def quant_refresh(cache: QuantCache, shape: Shape, k_new, v_new, kbar) -> None:
    """cache_refresh into a quantised cache; kbar fp32 [H, n_b, d] (or None): block means of the values it reads back as."""
    device, H, d = _quant_device(cache, shape, k_new), shape.n_heads, shape.head_dim
    _check_pair(device, k_new, v_new, "new", (H, shape.n_ctx + shape.n_resp, d))
    _check_values(device, (kbar, "kbar", torch.float32, 0 if kbar is None else H * _n_blocks(shape) * d))
    _check(lib().focus_quant_refresh(C.byref(cache), C.byref(shape), _ptr(k_new), _ptr(v_new), k_new.stride(0), k_new.stride(1), _ptr(kbar),
                                     _raw_stream(device)))


def quant_read(cache: QuantCache, shape: Shape, first_row: int, k_out, v_out) -> None:
    """Rows first_row, ... of a quantised cache into k_out, v_out bf16 [H, rows, d]."""
    device, rows = _quant_device(cache, shape, k_out), k_out.shape[1]
    _check_pair(device, k_out, v_out, "out", (shape.n_heads, rows, shape.head_dim))
    _check(lib().focus_quant_read(C.byref(cache), C.byref(shape), first_row, rows, _ptr(k_out), _ptr(v_out), k_out.stride(0), k_out.stride(1),
                                  _raw_stream(device)))


def _n_blocks(shape: Shape) -> int:
    return -(-shape.n_ctx // max(shape.block, 1))


def _check_attention(device: int, s: Shape, q, active_idx, slots: int, counts, kept_blocks, n_keep: int, sink_idx, n_sink: int, out, lse) -> None:
    """The tensors of an attention are what its shape and its counts say."""
    H, d = s.n_heads, s.head_dim
    if not (q.shape == (H, s.n_gen, d) and out.shape == (H, slots, d) and q.stride() == (s.q_stride_h, s.q_stride_n, 1)
            and out.stride() == (s.o_stride_h, s.o_stride_n, 1) and q.dtype == out.dtype == torch.bfloat16 and out.get_device() == device):
        _check_rows(device, (q, "Q", (H, s.n_gen, d)), (out, "out", (H, slots, d)))
        if not _strides_fit(q.shape, q.stride(), s.q_stride_h, s.q_stride_n) or not _strides_fit(out.shape, out.stride(), s.o_stride_h, s.o_stride_n):
            raise ValueError("Q and out must have the strides that the shape has for them")
    i32 = torch.int32
    _check_values(device, (active_idx, "active_idx", i32, 0), (kept_blocks, "kept_blocks", i32, n_keep), (sink_idx, "sink_idx", i32, n_sink),
                  (counts, "counts", i32, 0 if counts is None else 2), (lse, "lse", torch.float32, 0 if lse is None else H * slots))


def quant_attn(q, active_idx, counts, cache: QuantCache, shape: Shape, kept_blocks, n_keep: int, sink_idx, n_sink: int, out, lse, workspace) -> None:
    """sparse_attn over a quantised cache."""
    device, slots = _quant_device(cache, shape, q), active_idx.numel()
    _check_attention(device, shape, q, active_idx, slots, counts, kept_blocks, n_keep, sink_idx, n_sink, out, lse)
    _check(lib().focus_quant_attn(_ptr(q), _ptr(active_idx), _ptr(counts), slots, C.byref(cache), C.byref(shape), _ptr(kept_blocks), n_keep,
                                  _ptr(sink_idx), n_sink, _ptr(out), _ptr(lse), _ptr(workspace), _space(workspace, device), _raw_stream(device)))


def quant_layer(q, focus_idx, active_idx, counts, cache: QuantCache, kbar, shape: Shape, n_keep: int, sink_idx, n_sink: int, scores, kept_blocks, out,
                lse, workspace) -> None:
    """sparse_layer over a quantised cache, from the block means that the block entry left behind."""
    device, slots = _quant_device(cache, shape, q), active_idx.numel()
    _check_attention(device, shape, q, active_idx, slots, counts, kept_blocks, n_keep, sink_idx, n_sink, out, lse)
    n_b = _n_blocks(shape)
    _check_values(device, (focus_idx, "focus_idx", torch.int32, 1), (kbar, "kbar", torch.float32, shape.n_heads * n_b * shape.head_dim),
                  (scores, "scores", torch.float32, 0 if scores is None else n_b))
    _check(lib().focus_quant_layer(_ptr(q), _ptr(focus_idx), _ptr(active_idx), _ptr(counts), focus_idx.numel(), slots, C.byref(cache),
                                   _ptr(kbar), C.byref(shape), n_keep, _ptr(sink_idx), n_sink, _ptr(scores), _ptr(kept_blocks), _ptr(out), _ptr(lse),
                                   _ptr(workspace), _space(workspace, device), _raw_stream(device)))


# ---- requests over a paged cache
def rotary_freqs(base: float, rot_dim: int, factor: float = 1.0, orig_len: int = 1, turns_low: float = math.inf, turns_high: float = math.inf) -> torch.Tensor:
    """Frequencies for make_rotation, float64 on the host: see focus_helper_rotary.  Without turns_low and turns_high all are divided by `factor`."""
    values = (C.c_double * max(rot_dim // 2, 1))()
    _check(lib().focus_helper_rotary(base, rot_dim, factor, orig_len, turns_low, turns_high, values))
    return torch.tensor(list(values)[:rot_dim // 2], dtype=torch.float64)


def make_rotation(freq: torch.Tensor, interleaved: bool = False, scale: float = 1.0) -> Rotation:
    """focus_rotation from its frequencies, float64 [rot_dim / 2] on the device (kept by the description)."""
    _need(freq, torch.float64, "freq")
    if freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError(f"freq: expected values next to each other, got shape {tuple(freq.shape)}, strides {freq.stride()}")
    rotation = Rotation(_ptr(freq), 2 * freq.numel(), int(interleaved), scale)
    rotation.tensors, rotation.device = (freq,), freq.get_device()
    return rotation


def _page_strides(t: torch.Tensor):
    """Of a page, a head and a row (those of a single one mean nothing)."""
    return [0 if n == 1 else s for n, s in zip(t.shape[:3], t.stride()[:3])]


def make_paged_cache(k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor | None = None, v_exp: torch.Tensor | None = None) -> PagedCache:
    """focus_paged_cache from [n_pages, H, page, d] tensors (of any strides but the innermost, 1): bf16, or uint8 codes with the exponent bytes
    uint8 [n_pages, H, page].  The description keeps the tensors."""
    dtype = torch.bfloat16 if k_exp is None else torch.uint8
    if (k_exp is None) != (v_exp is None):
        raise ValueError("k_exp and v_exp go together")
    for t, name in ((k, "k"), (v, "v")):
        _need(t, dtype, name)
        if t.dim() != 4 or t.shape != k.shape or t.stride(3) != 1:
            raise ValueError(f"{name}: expected [n_pages, H, page, d], innermost stride 1, got {list(t.shape)}, strides {t.stride()}")
        if t.get_device() != k.get_device():
            raise ValueError("k, v and their exponents must be on one device")
    cache = PagedCache()
    cache.k, cache.v = _ptr(k), _ptr(v)
    cache.n_pages, cache.n_heads, cache.page, cache.head_dim = k.shape
    for t, name in ((k, "k"), (v, "v")):
        p, h, n = _page_strides(t)
        for axis, stride in (("p", p), ("h", h), ("n", n if t.shape[2] > 1 else max(t.shape[3], 16))):
            setattr(cache, f"{name}_stride_{axis}", stride)
    if k_exp is not None:
        for t, name in ((k_exp, "k_exp"), (v_exp, "v_exp")):
            _need(t, torch.uint8, name)
            if t.shape != k.shape[:3] or _page_strides(t) != _page_strides(k_exp) or t.get_device() != k.get_device():
                raise ValueError(f"{name}: expected {list(k.shape[:3])} with common strides on {k.device}, got {list(t.shape)}, strides {t.stride()}")
        cache.k_exp, cache.v_exp = _ptr(k_exp), _ptr(v_exp)
        cache.exp_stride_p, cache.exp_stride_h, n = _page_strides(k_exp)
        cache.exp_stride_n = n if k_exp.shape[2] > 1 else 1
    cache.tensors, cache.device = (k, v, k_exp, v_exp), k.get_device()
    return cache


def make_paged_batch(seq_len: torch.Tensor, page_table: torch.Tensor, row_start: torch.Tensor | None = None, max_rows: int = 1,
                     n_rows: int | None = None, positions: torch.Tensor | None = None) -> PagedBatch:
    """focus_paged_batch: seq_len int32 [n_req], page_table int32 [n_req, width], row_start int32 [n_req + 1] and positions int32 [n_rows] or None.
    n_rows: rows of the tensors that the calls take (None: n_req).  The description keeps the tensors, whose values may change between calls."""
    n_req = seq_len.numel()
    n_rows = n_req if n_rows is None else n_rows
    if page_table.dim() != 2 or page_table.shape[0] != n_req or page_table.shape[1] < 1 or (page_table.stride(1) != 1 and page_table.shape[1] > 1):
        raise ValueError(f"page_table: expected [{n_req}, width], innermost stride 1, got {list(page_table.shape)}, strides {page_table.stride()}")
    _need(page_table, torch.int32, "page_table")
    device = page_table.get_device()
    _check_values(device, (seq_len, "seq_len", torch.int32, 1), (row_start, "row_start", torch.int32, 0 if row_start is None else n_req + 1),
                  (positions, "positions", torch.int32, 0 if positions is None else n_rows))
    batch = PagedBatch(_ptr(seq_len), _ptr(page_table), _ptr(row_start), _ptr(positions),
                       max(page_table.stride(0), page_table.shape[1]) if n_req > 1 else page_table.shape[1], page_table.shape[1], n_req, max_rows, n_rows)
    if n_req > 1 and page_table.stride(0) < page_table.shape[1]:
        raise ValueError(f"page_table: rows lie on one another, strides {page_table.stride()}")
    batch.tensors, batch.device = (seq_len, page_table, row_start, positions), device
    return batch


# The checks of these calls: one condition where everything is as it should be (they are a few microseconds long), and functions that tell what is not.
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _current_device() -> int:
    # the number without the initialisation that torch.cuda.current_device looks for: a CUDA tensor is there already
    try:
        return torch._C._cuda_getDevice()
    except AttributeError:  # (not part of torch's interface)
        return torch.cuda.current_device()


def _explain_devices(device: int, *things) -> None:
    for t, name in things:
        there = device if t is None else t.get_device() if isinstance(t, torch.Tensor) else t.device
        if there is not None and there != device:
            raise ValueError(f"{name} on device {there}, but the current device is cuda:{device}")


def _explain_heads(device: int, rows: int, head_dim: int, *expected) -> None:
    """bf16 [rows, heads, head_dim], innermost stride 1."""
    for t, name, heads in expected:
        if t.dtype != _BF16 or t.get_device() != device:
            raise TypeError(f"{name}: expected a tensor of torch.bfloat16 on cuda:{device}, got {t.dtype} on {t.device}")
        if t.shape != (rows, heads, head_dim) or t.stride(2) != 1:
            raise ValueError(f"{name}: expected {[rows, heads, head_dim]}, innermost stride 1, got {list(t.shape)}, strides {t.stride()}")


def _strides(shape, strides):
    """Strides of a head and of a row of [rows, heads, d] (those of a single one mean nothing)."""
    return (strides[1] if shape[1] > 1 else 0), (strides[0] if shape[0] > 1 else 0)


def _fits(t, dtype, device: int, shape) -> bool:
    return t is None or (t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous())


def rotary(x, out, positions, pos_base: int, rotation: Rotation) -> None:
    """x, out bf16 [rows, heads, d] of any strides (a transposed view of head-major rows is one; out may be x); positions int32 [rows] or None."""
    device, shape, xs, outs = _current_device(), x.shape, x.stride(), out.stride()
    if not (x.dtype is out.dtype is _BF16 and x.get_device() == out.get_device() == device and out.shape == shape and len(shape) == 3 and xs[2] == 1 == outs[2]
            and rotation.device in (device, None) and _fits(positions, _I32, device, shape[:1])):
        _explain_devices(device, (x, "x"), (rotation, "rotation"))
        if len(shape) != 3:
            raise ValueError(f"x: expected [rows, heads, d], got {list(shape)}")
        _explain_heads(device, shape[0], shape[2], (x, "x", shape[1]), (out, "out", shape[1]))
        _check_values(device, (positions, "positions", _I32, 0 if positions is None else shape[0]))
    if not -0x80000000 <= pos_base <= 0x7fffffff:  # (ctypes would take the lower 32 bits)
        raise ValueError(f"pos_base: {pos_base} is not a number of 32 bits")
    n, heads, d = shape
    status = lib().focus_rotary(x.data_ptr(), *_strides(shape, xs), out.data_ptr(), *_strides(shape, outs), n, heads, d, _ptr(positions), pos_base,
                                C.byref(rotation), _raw_stream(device))
    if status:
        _check(status)


def paged_append(cache: PagedCache, batch: PagedBatch, k_new, v_new, rotation: Rotation | None = None, q=None, q_out=None) -> None:
    """k_new, v_new bf16 [n_rows, H, d] (common strides) into the requests' pages; with q, q_out bf16 [n_rows, heads, d] those turned as well."""
    device, shape, strides = _current_device(), k_new.shape, k_new.stride()
    n, d = batch.n_rows, cache.head_dim
    if not (shape == (n, cache.n_heads, d) == v_new.shape and strides == v_new.stride() and strides[2] == 1 and k_new.dtype is v_new.dtype is _BF16
            and k_new.get_device() == v_new.get_device() == device and cache.device in (device, None) and batch.device in (device, None)
            and (rotation is None or rotation.device in (device, None))):
        _explain_devices(device, (k_new, "k_new"), (cache, "cache"), (batch, "batch"), (rotation, "rotation"))
        _explain_heads(device, n, d, (k_new, "k_new", cache.n_heads), (v_new, "v_new", cache.n_heads))
        if _strides(shape, strides) != _strides(shape, v_new.stride()):
            raise ValueError("k_new and v_new must share their strides")
    heads, q_strides, out_strides = 0, (0, 0), (0, 0)
    if q is not None and q_out is not None:
        q_shape, qs, outs = q.shape, q.stride(), q_out.stride()
        heads = q_shape[1] if len(q_shape) == 3 else -1
        if not (q_shape == (n, heads, d) == q_out.shape and qs[2] == 1 == outs[2] and q.dtype is q_out.dtype is _BF16 and q.get_device() == q_out.get_device() == device):
            _explain_heads(device, n, d, (q, "q", heads), (q_out, "q_out", heads))
        q_strides, out_strides = _strides(q_shape, qs), _strides(q_shape, outs)
    elif q is not None or q_out is not None:
        raise ValueError("q and q_out go together")
    status = lib().focus_paged_append(C.byref(cache), C.byref(batch), k_new.data_ptr(), v_new.data_ptr(), *_strides(shape, strides),
                                      None if rotation is None else C.byref(rotation), _ptr(q), *q_strides, _ptr(q_out), *out_strides, heads, _raw_stream(device))
    if status:
        _check(status)


def paged_attn_workspace(cache: PagedCache, batch: PagedBatch, n_q_heads: int) -> int:
    return int(lib().focus_paged_attn_workspace(C.byref(cache), C.byref(batch), n_q_heads))


def paged_attn(q, cache: PagedCache, batch: PagedBatch, causal: bool, out, lse, workspace) -> None:
    """q, out bf16 [n_rows, n_q_heads, d], lse fp32 [n_rows, n_q_heads] or None; workspace of paged_attn_workspace() bytes."""
    device, shape, qs, outs = _current_device(), q.shape, q.stride(), out.stride()
    heads = shape[1] if len(shape) == 3 else -1
    if not (shape == (batch.n_rows, heads, cache.head_dim) == out.shape and qs[2] == 1 == outs[2] and q.dtype is out.dtype is _BF16
            and q.get_device() == out.get_device() == device and cache.device in (device, None) and batch.device in (device, None)
            and _fits(lse, _F32, device, shape[:2])):
        _explain_devices(device, (q, "q"), (cache, "cache"), (batch, "batch"))
        _explain_heads(device, batch.n_rows, cache.head_dim, (q, "q", heads), (out, "out", heads))
        _check_values(device, (lse, "lse", _F32, 0 if lse is None else shape[0] * heads))
    status = lib().focus_paged_attn(q.data_ptr(), *_strides(shape, qs), heads, C.byref(cache), C.byref(batch), causal, out.data_ptr(), *_strides(shape, outs),
                                    _ptr(lse), _ptr(workspace), _space(workspace, device), _raw_stream(device))
    if status:
        _check(status)


def token_logprobs_workspace(n_rows: int, vocab: int, top_n: int) -> int:
    return int(lib().focus_token_logprobs_workspace(n_rows, vocab, top_n))


def token_logprobs(logits, targets, masked, logprob, entropy, top_ids, top_logprobs, workspace) -> None:
    """logits bf16 or fp32 [n_rows, vocab] (rows 16-byte aligned); targets int32 and logprob fp32 [n_rows] (both or neither), entropy fp32 [n_rows] or
    None, top_ids int32 and top_logprobs fp32 [n_rows, top_n] (both or neither); workspace of token_logprobs_workspace() bytes."""
    dtype = logits.dtype
    if not logits.is_cuda or (dtype is not _BF16 and dtype is not _F32):
        raise TypeError(f"logits: expected a CUDA tensor of bfloat16 or float32, got {dtype} on {logits.device}")
    shape, device = logits.shape, _current_device()
    if len(shape) != 2 or logits.stride(1) != 1 or logits.get_device() != device:
        _explain_devices(device, (logits, "logits"))
        raise ValueError("logits: expected [n_rows, vocab], innermost stride 1")
    rows, vocab = shape
    stride = logits.stride(0) if rows > 1 else (vocab + 7) // 8 * 8  # (of one row any will do)
    if (top_ids is None) != (top_logprobs is None) or (targets is None) != (logprob is None):
        raise ValueError("targets and logprob, top_ids and top_logprobs go together")
    one = shape[:1]
    top_n, many = 0, one
    if top_ids is not None:
        many = top_ids.shape
        top_n = many[1] if len(many) == 2 else -1
    if not (_fits(targets, _I32, device, one) and _fits(logprob, _F32, device, one) and _fits(entropy, _F32, device, one) and _fits(top_ids, _I32, device, (rows, top_n))
            and _fits(top_logprobs, _F32, device, many)):
        for t, kind, sizes, name in ((targets, _I32, one, "targets"), (logprob, _F32, one, "logprob"), (entropy, _F32, one, "entropy"),
                                     (top_ids, _I32, (rows, top_n), "top_ids"), (top_logprobs, _F32, (rows, top_n), "top_logprobs")):
            if not _fits(t, kind, device, sizes):
                _need(t, kind, name)
                _explain_devices(device, (t, name))
                raise ValueError(f"{name}: expected {list(sizes)} next to each other, got {list(t.shape)}, strides {t.stride()}")
    if masked is not None and (masked.get_device() != device or masked.element_size() != 1 or masked.shape != one or not masked.is_contiguous()):
        raise ValueError(f"masked: expected {rows} bytes on cuda:{device}, got {masked.dtype}, shape {tuple(masked.shape)} on {masked.device}")
    status = lib().focus_token_logprobs(logits.data_ptr(), dtype is _F32, stride, _ptr(targets), _ptr(masked), rows, vocab, top_n, _ptr(logprob), _ptr(entropy),
                                        _ptr(top_ids), _ptr(top_logprobs), _ptr(workspace), _space(workspace, device), _raw_stream(device))
    if status:
        _check(status)
