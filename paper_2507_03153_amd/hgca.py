"""Thin ctypes binding of libhgca.so (the C ABI declared in include/hgca.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Tensors are torch tensors on the GPU; torch is used for device
memory and streams.  There is no CPU fallback: without the built library, or
with a tensor that is not on a GPU, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch  # noqa: F401  (loads the HIP runtime the library binds to; must precede CDLL)

F32, BF16 = 0, 1
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_DEVICE = 0, -1, -2, -3, -4

# HGCA_LIB names another build of the same library (tuning experiments); the default is the in-tree one
_LIB_PATH = os.environ.get("HGCA_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhgca.so")

EXPORTS = ("hgca_status_string", "hgca_workspace_bytes", "hgca_dense_window_attn",
           "hgca_pool_scores", "hgca_select_salient", "hgca_sparse_attn", "hgca_lse_merge_splits", "hgca_lse_merge",
           "hgca_dense_window_attn_weights", "hgca_maw_update", "hgca_threshold_select", "hgca_select_topk",
           "hgca_kv_append", "hgca_kv_evict", "hgca_append_workspace_bytes", "hgca_append_attn",
           "hgca_append_tiers_workspace_bytes", "hgca_append_attn_tiers", "hgca_append_weights_tiers",
           "hgca_append_weights", "hgca_dense_window_attn_maw", "hgca_select_salient_grouped", "hgca_union_lists",
           "hgca_sparse_attn_grouped", "hgca_hybrid_decode_step", "hgca_ctx_compact",
           "hgca_managed_decode_step", "hgca_dense_window_attn_static", "hgca_hybrid_decode_step_selected", "hgca_kv_append_tokens",
           "hgca_managed_append_workspace_bytes", "hgca_managed_append_step",
           "hgca_qk_norm_rope", "hgca_tree_workspace_bytes", "hgca_tree_attn", "hgca_kv_commit", "hgca_kv8_write_tokens",
           "hgca_kv8_write_tier", "hgca_kv8_read", "hgca_kv8_workspace_bytes", "hgca_kv8_attn")
STATIC_SCRATCH_BYTES = 16 << 20                  # HGCA_STATIC_SCRATCH_BYTES of include/hgca.h
CACHE_WINDOW_FULL, CACHE_CONTEXT_FULL, CACHE_LIST_FULL = 1, 2, 4


class Shape(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("sm_scale", ctypes.c_float)]


class KvView(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("cap", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("first_block", ctypes.c_void_p)]


class Kv8View(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "seq_lens", "block_table")] + \
               [(n, ctypes.c_int32) for n in ("cap", "block_size", "max_blocks")] + [("first_block", ctypes.c_void_p)]


class CacheState(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_blocks", "v_blocks", "block_table", "first_win_block", "win_lens",
                                               "pool_lens", "a_maw", "ctx_idx", "ctx_cnt", "a_evicted", "plan",
                                               "status")] + \
               [(n, ctypes.c_int32) for n in ("block_size", "max_blocks", "win_blocks", "k_max", "pool_cap",
                                               "win_cap_blocks")]


class HgcaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (python -m paper_2507_03153_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(f"{_LIB_PATH} is missing: build it with "
                                    "`python -m paper_2507_03153_amd.build`; there is no fallback path")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        ps, pk = ctypes.POINTER(Shape), ctypes.POINTER(KvView)
        L.hgca_status_string.restype = ctypes.c_char_p
        L.hgca_status_string.argtypes = [ctypes.c_int]
        L.hgca_workspace_bytes.restype = sz
        L.hgca_workspace_bytes.argtypes = [ps, i32, i32, i32]
        L.hgca_dense_window_attn.restype = ctypes.c_int
        L.hgca_dense_window_attn.argtypes = [ps, vp, pk, vp, vp, vp, sz, vp]
        L.hgca_dense_window_attn_static.restype = ctypes.c_int
        L.hgca_dense_window_attn_static.argtypes = [ps, vp, pk, vp, vp, vp]
        L.hgca_pool_scores.restype = ctypes.c_int
        L.hgca_pool_scores.argtypes = [ps, vp, pk, vp, vp]
        L.hgca_select_salient.restype = ctypes.c_int
        L.hgca_select_salient.argtypes = [ps, vp, pk, vp, i32, i32, vp, vp, vp, vp, sz, vp]
        L.hgca_sparse_attn.restype = ctypes.c_int
        L.hgca_sparse_attn.argtypes = [ps, vp, pk, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.hgca_lse_merge_splits.restype = ctypes.c_int
        L.hgca_lse_merge_splits.argtypes = [ps, i32, vp, sz, i32, vp, sz, vp, i32, vp, vp]
        L.hgca_lse_merge.restype = ctypes.c_int
        L.hgca_lse_merge.argtypes = [ps, vp, vp, vp, vp, vp, i32, vp, vp]
        L.hgca_dense_window_attn_weights.restype = ctypes.c_int
        L.hgca_dense_window_attn_weights.argtypes = [ps, vp, pk, vp, vp, vp, vp, sz, vp]
        L.hgca_select_topk.restype = ctypes.c_int
        L.hgca_select_topk.argtypes = [ps, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp]
        L.hgca_append_workspace_bytes.restype = sz
        L.hgca_append_workspace_bytes.argtypes = [ps, i32, i32]
        L.hgca_append_attn.restype = ctypes.c_int
        L.hgca_append_attn.argtypes = [ps, vp, i32, pk, i32, vp, vp, vp, sz, vp]
        L.hgca_append_weights_tiers.restype = ctypes.c_int
        L.hgca_append_weights_tiers.argtypes = [ps, vp, i32, pk, pk, i32, vp, vp, vp, vp, vp]
        L.hgca_append_tiers_workspace_bytes.restype = ctypes.c_size_t
        L.hgca_append_tiers_workspace_bytes.argtypes = [ps, i32, i32, i32]
        L.hgca_append_attn_tiers.restype = ctypes.c_int
        L.hgca_append_attn_tiers.argtypes = [ps, vp, i32, pk, pk, i32, vp, vp, vp, vp, vp, sz, vp]
        L.hgca_append_weights.restype = ctypes.c_int
        L.hgca_append_weights.argtypes = [ps, vp, i32, pk, i32, vp, vp, vp]
        L.hgca_kv_append.restype = ctypes.c_int
        L.hgca_kv_append.argtypes = [ps, ctypes.POINTER(CacheState), vp, vp, vp, vp]
        L.hgca_kv_append_tokens.restype = ctypes.c_int
        L.hgca_kv_append_tokens.argtypes = [ps, ctypes.POINTER(CacheState), vp, vp, i32, vp, vp]
        L.hgca_managed_append_workspace_bytes.restype = sz
        L.hgca_managed_append_workspace_bytes.argtypes = [ps, ctypes.POINTER(CacheState), i32]
        L.hgca_managed_append_step.restype = ctypes.c_int
        L.hgca_managed_append_step.argtypes = [ps, ctypes.POINTER(CacheState), vp, vp, vp, i32, ctypes.c_float,
                                               ctypes.c_double, i32, vp, vp, vp, vp, vp, sz, vp]
        L.hgca_kv_evict.restype = ctypes.c_int
        L.hgca_kv_evict.argtypes = [ps, ctypes.POINTER(CacheState), ctypes.c_double, vp]
        L.hgca_select_salient_grouped.restype = ctypes.c_int
        L.hgca_select_salient_grouped.argtypes = [ps, vp, pk, vp, i32, i32, vp, vp, vp, sz, vp]
        L.hgca_union_lists.restype = ctypes.c_int
        L.hgca_union_lists.argtypes = [ps, vp, vp, i32, i32, vp, vp, i32, vp, vp]
        L.hgca_sparse_attn_grouped.restype = ctypes.c_int
        L.hgca_sparse_attn_grouped.argtypes = [ps, vp, pk, vp, vp, i32, vp, vp, vp, sz, vp]
        L.hgca_managed_decode_step.restype = ctypes.c_int
        L.hgca_managed_decode_step.argtypes = [ps, ctypes.POINTER(CacheState), vp, vp, vp, ctypes.c_float,
                                               ctypes.c_double, vp, vp, i32, vp, vp, sz, vp, sz, vp]
        L.hgca_ctx_compact.restype = ctypes.c_int
        L.hgca_ctx_compact.argtypes = [ps, pk, vp, vp, i32, vp, vp, vp, i32, vp, vp]
        L.hgca_hybrid_decode_step.restype = ctypes.c_int
        L.hgca_hybrid_decode_step.argtypes = [ps, vp, pk, pk, vp, i32, i32, vp, vp, vp, i32, vp, vp, sz, vp, sz, vp]
        L.hgca_hybrid_decode_step_selected.restype = ctypes.c_int
        L.hgca_hybrid_decode_step_selected.argtypes = [ps, vp, pk, pk, vp, vp, i32, vp, vp, i32, vp, vp, sz, vp, sz, vp]
        L.hgca_dense_window_attn_maw.restype = ctypes.c_int
        L.hgca_dense_window_attn_maw.argtypes = [ps, vp, pk, vp, vp, vp, vp, i32, ctypes.c_float, vp, sz, vp]
        L.hgca_maw_update.restype = ctypes.c_int
        L.hgca_maw_update.argtypes = [ps, vp, vp, vp, i32, i32, ctypes.c_float, vp]
        L.hgca_threshold_select.restype = ctypes.c_int
        L.hgca_threshold_select.argtypes = [ps, vp, vp, i32, vp, i32, ctypes.c_double, i32, vp, vp, vp, vp]
        p8, i64 = ctypes.POINTER(Kv8View), ctypes.c_int64
        L.hgca_qk_norm_rope.restype = ctypes.c_int
        L.hgca_qk_norm_rope.argtypes = [ps, vp, i64, vp, i64, i32, vp, vp, ctypes.c_float, vp, i32, vp, vp, i32, vp, vp, vp]
        L.hgca_tree_workspace_bytes.restype = sz
        L.hgca_tree_workspace_bytes.argtypes = [ps, i32, i32]
        L.hgca_tree_attn.restype = ctypes.c_int
        L.hgca_tree_attn.argtypes = [ps, vp, i32, pk, vp, vp, i32, vp, vp, sz, vp]
        L.hgca_kv_commit.restype = ctypes.c_int
        L.hgca_kv_commit.argtypes = [ps, pk, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        L.hgca_kv8_write_tokens.restype = ctypes.c_int
        L.hgca_kv8_write_tokens.argtypes = [ps, p8, vp, vp, vp, i32, vp, vp]
        L.hgca_kv8_write_tier.restype = ctypes.c_int
        L.hgca_kv8_write_tier.argtypes = [ps, p8, vp, pk, i32, vp, vp]
        L.hgca_kv8_read.restype = ctypes.c_int
        L.hgca_kv8_read.argtypes = [ps, p8, vp, i32, vp, vp, vp]
        L.hgca_kv8_workspace_bytes.restype = sz
        L.hgca_kv8_workspace_bytes.argtypes = [ps, i32, i32]
        L.hgca_kv8_attn.restype = ctypes.c_int
        L.hgca_kv8_attn.argtypes = [ps, vp, i32, p8, vp, i32, vp, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().hgca_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise HgcaError(status, where)


@dataclass
class Tier:
    """One KV tier on the GPU.  k/v: contiguous [B,Hkv,cap,d] or paged [n_blocks,Hkv,bs,d]."""
    k: torch.Tensor
    v: Optional[torch.Tensor]
    cap: int
    seq_lens: Optional[torch.Tensor] = None      # int32 [B]
    block_table: Optional[torch.Tensor] = None   # int32 [B,max_blocks]
    block_size: int = 0
    first_block: Optional[torch.Tensor] = None   # int32 [B]: the tier starts at this entry of its table row

    def view(self) -> KvView:
        for t in (self.k, self.v, self.seq_lens, self.block_table, self.first_block):
            if t is not None:
                _require_gpu(t)
        mb = 0 if self.block_table is None else int(self.block_table.shape[1])
        return KvView(_ptr(self.k), _ptr(self.v), _ptr(self.seq_lens), _ptr(self.block_table),
                      int(self.cap), int(self.block_size), mb, _ptr(self.first_block))


def _require_gpu(t: torch.Tensor) -> None:
    if not t.is_cuda:
        raise ValueError("libhgca takes GPU tensors only (no CPU path exists)")
    if not t.is_contiguous():
        raise ValueError("libhgca takes contiguous tensors")


def _ptr(t: Optional[torch.Tensor]):
    """The address as ctypes takes it for a pointer argument (None and 0: null)."""
    return None if t is None else t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"q/K/V must be float32 or bfloat16, got {t.dtype}")


def make_shape(q: torch.Tensor, n_kv_heads: int, sm_scale: float) -> Shape:
    _require_gpu(q)
    B, Hq, d = q.shape
    return Shape(_dtype_code(q), B, Hq, int(n_kv_heads), d, float(sm_scale))


# The current stream's handle without a Stream object around it, as addresses are passed without ctypes objects: small steps
# wait for the host (4 heads over 2 K tokens: 16.8 us of host time per step with those objects, 13.6 without, 8 of them
# the two launches).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def workspace_bytes(shape: Shape, max_window: int, max_pool: int, k_max: int) -> int:
    return int(lib().hgca_workspace_bytes(ctypes.byref(shape), int(max_window), int(max_pool), int(k_max)))


def alloc_workspace(shape: Shape, max_window: int, max_pool: int, k_max: int, device) -> torch.Tensor:
    n = workspace_bytes(shape, max_window, max_pool, k_max)
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def dense_window_attn(shape: Shape, q, window: Tier, o_out, lse_out, ws, stream=None) -> None:
    """o_out = lse_out = None defers the result: the split partials stay in ws for lse_merge_splits."""
    for t in (q, ws) + (() if o_out is None else (o_out, lse_out)):
        _require_gpu(t)
    kv = window.view()
    _check(lib().hgca_dense_window_attn(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(o_out), _ptr(lse_out),
                                        _ptr(ws), ws.numel(), _stream(stream)), "hgca_dense_window_attn")


def dense_window_attn_static(shape: Shape, q, window: Tier, o_out, lse_out, stream=None) -> None:
    """dense_window_attn without a workspace: the split partials live in the library's own device array."""
    for t in (q, o_out, lse_out):
        _require_gpu(t)
    kv = window.view()
    _check(lib().hgca_dense_window_attn_static(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(o_out),
                                               _ptr(lse_out), _stream(stream)), "hgca_dense_window_attn_static")


def pool_scores(shape: Shape, q, pool: Tier, scores_out, stream=None) -> None:
    for t in (q, scores_out):
        _require_gpu(t)
    kv = pool.view()
    _check(lib().hgca_pool_scores(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(scores_out), _stream(stream)),
           "hgca_pool_scores")


def select_salient(shape: Shape, q, pool: Tier, k, k_max: int, idx_out, cnt_out, ws, stream=None,
                   sel_scores_out=None) -> None:
    """k: int (uniform budget) or int32 GPU tensor [B] (per-sequence budgets)."""
    for t in (q, idx_out, cnt_out, ws) + (() if sel_scores_out is None else (sel_scores_out,)):
        _require_gpu(t)
    kv = pool.view()
    if isinstance(k, torch.Tensor):
        _require_gpu(k)
        k_ptr, k_uni = _ptr(k), 0
    else:
        k_ptr, k_uni = None, int(k)
    _check(lib().hgca_select_salient(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), k_ptr, k_uni, int(k_max),
                                     _ptr(idx_out), _ptr(cnt_out), _ptr(sel_scores_out), _ptr(ws), ws.numel(),
                                     _stream(stream)),
           "hgca_select_salient")


def sparse_attn(shape: Shape, q, pool: Tier, idx, cnt, k_max: int, o_out, lse_out, ws, stream=None,
                sel_scores=None) -> None:
    """sel_scores: scores of the listed entries for this q (from select_salient); K is then not re-read."""
    for t in (q, idx, cnt, ws) + (() if sel_scores is None else (sel_scores,)) + \
            (() if o_out is None else (o_out, lse_out)):
        _require_gpu(t)
    kv = pool.view()
    _check(lib().hgca_sparse_attn(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(idx), _ptr(cnt), int(k_max),
                                  _ptr(sel_scores), _ptr(o_out), _ptr(lse_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_sparse_attn")


def lse_merge_splits(shape: Shape, window_cap: int, ws_dense, k_max: int, ws_sparse, o_out, lse_out=None,
                     stream=None) -> None:
    """Folds the deferred split partials of a dense and a sparse call into the final O (and lse)."""
    for t in (o_out,) + tuple(x for x in (ws_dense, ws_sparse, lse_out) if x is not None):
        _require_gpu(t)
    nb = lambda w: 0 if w is None else w.numel()
    _check(lib().hgca_lse_merge_splits(ctypes.byref(shape), int(window_cap), _ptr(ws_dense), nb(ws_dense), int(k_max),
                                       _ptr(ws_sparse), nb(ws_sparse), _ptr(o_out), _dtype_code(o_out),
                                       _ptr(lse_out), _stream(stream)), "hgca_lse_merge_splits")


def lse_merge(shape: Shape, o_a, lse_a, o_b, lse_b, o_out, lse_out=None, stream=None) -> None:
    for t in (o_a, lse_a, o_b, lse_b, o_out):
        _require_gpu(t)
    _check(lib().hgca_lse_merge(ctypes.byref(shape), _ptr(o_a), _ptr(lse_a), _ptr(o_b), _ptr(lse_b), _ptr(o_out),
                                _dtype_code(o_out), _ptr(lse_out), _stream(stream)), "hgca_lse_merge")


def dense_window_attn_weights(shape: Shape, q, window: Tier, o_out, lse_out, a_out, ws, stream=None) -> None:
    """Dense window attention that also returns the window's softmax weights a_out [B,Hq,cap] (fp32)."""
    for t in (q, ws, o_out, lse_out, a_out):
        _require_gpu(t)
    kv = window.view()
    _check(lib().hgca_dense_window_attn_weights(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(o_out),
                                                _ptr(lse_out), _ptr(a_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_dense_window_attn_weights")


def maw_update(shape: Shape, a_maw, a_gpu, seq_lens, cap: int, n_new: int, alpha: float, stream=None) -> None:
    """a_maw <- (1 - alpha) a_maw + alpha a_gpu in place; the last n_new valid entries take a_gpu."""
    for t in (a_maw, a_gpu) + (() if seq_lens is None else (seq_lens,)):
        _require_gpu(t)
    _check(lib().hgca_maw_update(ctypes.byref(shape), _ptr(a_maw), _ptr(a_gpu), _ptr(seq_lens), int(cap), int(n_new),
                                 float(alpha), _stream(stream)), "hgca_maw_update")


def threshold_select(shape: Shape, weights, seq_lens, cap: int, size, beta: float, k_max: int, idx_out, cnt_out,
                     w_norm_out=None, stream=None) -> None:
    """size: int (uniform) or int32 GPU tensor [B]: the number of entries the weights were taken over."""
    for t in (weights, idx_out, cnt_out) + tuple(x for x in (seq_lens, w_norm_out) if x is not None):
        _require_gpu(t)
    if isinstance(size, torch.Tensor):
        _require_gpu(size)
        size_ptr, size_uni = _ptr(size), 0
    else:
        size_ptr, size_uni = None, int(size)
    _check(lib().hgca_threshold_select(ctypes.byref(shape), _ptr(weights), _ptr(seq_lens), int(cap), size_ptr,
                                       size_uni, float(beta), int(k_max), _ptr(idx_out), _ptr(cnt_out),
                                       _ptr(w_norm_out), _stream(stream)), "hgca_threshold_select")


def select_topk(shape: Shape, scores, seq_lens, cap: int, k, k_max: int, idx_out, cnt_out, sel_scores_out=None,
                stream=None) -> None:
    """Per-head top-k of caller-supplied fp32 scores [B,Hq,cap]; k: int or int32 GPU tensor [B]."""
    for t in (scores, idx_out, cnt_out) + tuple(x for x in (seq_lens, sel_scores_out) if x is not None):
        _require_gpu(t)
    if isinstance(k, torch.Tensor):
        _require_gpu(k)
        k_ptr, k_uni = _ptr(k), 0
    else:
        k_ptr, k_uni = None, int(k)
    _check(lib().hgca_select_topk(ctypes.byref(shape), _ptr(scores), _ptr(seq_lens), int(cap), k_ptr, k_uni, int(k_max),
                                  _ptr(idx_out), _ptr(cnt_out), _ptr(sel_scores_out), _stream(stream)),
           "hgca_select_topk")


def kv_append(shape: Shape, cache: CacheState, k_in, v_in, active=None, stream=None) -> None:
    """Writes the new token's K/V rows [B,Hkv,d] at the end of every (active) sequence's window."""
    for t in (k_in, v_in) + (() if active is None else (active,)):
        _require_gpu(t)
    _check(lib().hgca_kv_append(ctypes.byref(shape), ctypes.byref(cache), _ptr(k_in), _ptr(v_in), _ptr(active),
                                _stream(stream)), "hgca_kv_append")


def kv_append_tokens(shape: Shape, cache: CacheState, k_in, v_in, active=None, stream=None) -> None:
    """Writes a prompt's K/V rows [B,N,Hkv,d] behind every (active) sequence's window."""
    for t in (k_in, v_in) + (() if active is None else (active,)):
        _require_gpu(t)
    _check(lib().hgca_kv_append_tokens(ctypes.byref(shape), ctypes.byref(cache), _ptr(k_in), _ptr(v_in),
                                       int(k_in.shape[1]), _ptr(active), _stream(stream)), "hgca_kv_append_tokens")


def managed_append_workspace(shape: Shape, cache: CacheState, n_q: int, device) -> torch.Tensor:
    n = int(lib().hgca_managed_append_workspace_bytes(ctypes.byref(shape), ctypes.byref(cache), int(n_q)))
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_managed_append_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def managed_append_step(shape: Shape, cache: CacheState, q, k_in, v_in, alpha: float, beta: float, a_gpu, a_cpu,
                        o_out, lse_out, ws, stream=None, one_part_p: bool = False) -> None:
    """One append turn over the managed cache (insert N tokens, attend to window and complete pool, merge, moving
    averages, re-evaluation of the salient lists, eviction) in one call.  q [B,N,Hq,d], k_in / v_in [B,N,Hkv,d]."""
    for t in (q, k_in, v_in, a_gpu, o_out, lse_out, ws) + (() if a_cpu is None else (a_cpu,)):
        _require_gpu(t)
    _check(lib().hgca_managed_append_step(ctypes.byref(shape), ctypes.byref(cache), _ptr(q), _ptr(k_in), _ptr(v_in),
                                          int(q.shape[1]), float(alpha), float(beta),
                                          APPEND_ONE_PART_P if one_part_p else 0, _ptr(a_gpu), _ptr(a_cpu), _ptr(o_out),
                                          _ptr(lse_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_managed_append_step")


def kv_evict(shape: Shape, cache: CacheState, beta: float, stream=None) -> None:
    """Sequences whose window reached l_max hand their oldest block(s) to the pool and sparsify them."""
    _check(lib().hgca_kv_evict(ctypes.byref(shape), ctypes.byref(cache), float(beta), _stream(stream)),
           "hgca_kv_evict")


def append_workspace(shape: Shape, n_q: int, max_tokens: int, device) -> torch.Tensor:
    n = int(lib().hgca_append_workspace_bytes(ctypes.byref(shape), int(n_q), int(max_tokens)))
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_append_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


APPEND_CAUSAL_TAIL, APPEND_ONE_PART_P = 1, 2


def append_attn(shape: Shape, q, tier: Tier, causal_tail: bool, o_out, lse_out, ws, stream=None,
                one_part_p: bool = False) -> None:
    """q [B,N,Hq,d] bf16; o_out [B,N,Hq,d], lse_out [B,N,Hq] fp32."""
    for t in (q, o_out, lse_out, ws):
        _require_gpu(t)
    kv = tier.view()
    flags = (APPEND_CAUSAL_TAIL if causal_tail else 0) | (APPEND_ONE_PART_P if one_part_p else 0)
    _check(lib().hgca_append_attn(ctypes.byref(shape), _ptr(q), int(q.shape[1]), ctypes.byref(kv), flags,
                                  _ptr(o_out), _ptr(lse_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_append_attn")


def append_tiers_workspace(shape: Shape, n_q: int, window_cap: int, pool_cap: int, device) -> torch.Tensor:
    n = int(lib().hgca_append_tiers_workspace_bytes(ctypes.byref(shape), int(n_q), int(window_cap), int(pool_cap)))
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_append_tiers_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def append_attn_tiers(shape: Shape, q, window: Tier, pool: Tier, o_out, lse_out, ws, lse_window_out=None,
                      lse_pool_out=None, causal_tail: bool = True, one_part_p: bool = False, stream=None) -> None:
    """Attention of q [B,N,Hq,d] bf16 over the window (causal among its last N tokens) and over the whole pool, merged:
    o_out [B,N,Hq,d], lse_out [B,N,Hq] fp32; the per-tier lse rows are optional outputs."""
    for t in (q, o_out, lse_out, ws):
        _require_gpu(t)
    for t in (lse_window_out, lse_pool_out):
        if t is not None:
            _require_gpu(t)
    kw, kp = window.view(), pool.view()
    flags = (APPEND_CAUSAL_TAIL if causal_tail else 0) | (APPEND_ONE_PART_P if one_part_p else 0)
    _check(lib().hgca_append_attn_tiers(ctypes.byref(shape), _ptr(q), int(q.shape[1]), ctypes.byref(kw), ctypes.byref(kp),
                                        flags, _ptr(o_out), _ptr(lse_out),
                                        _ptr(lse_window_out) if lse_window_out is not None else None,
                                        _ptr(lse_pool_out) if lse_pool_out is not None else None,
                                        _ptr(ws), ws.numel(), _stream(stream)), "hgca_append_attn_tiers")


def append_weights(shape: Shape, q, tier: Tier, causal_tail: bool, lse, a_out, stream=None) -> None:
    """Query-averaged softmax weights of the tier, a_out [B,Hq,cap] fp32; lse from append_attn on the same tier."""
    for t in (q, lse, a_out):
        _require_gpu(t)
    kv = tier.view()
    _check(lib().hgca_append_weights(ctypes.byref(shape), _ptr(q), int(q.shape[1]), ctypes.byref(kv), int(causal_tail),
                                     _ptr(lse), _ptr(a_out), _stream(stream)), "hgca_append_weights")


def append_weights_tiers(shape: Shape, q, window: Tier, pool: Tier, lse_window, lse_pool, a_gpu, a_cpu,
                         causal_tail: bool = True, stream=None) -> None:
    """Query-averaged weights of window and pool in one launch (bf16); the lse rows from append_attn_tiers."""
    for t in (q, lse_window, lse_pool, a_gpu, a_cpu):
        _require_gpu(t)
    kw, kp = window.view(), pool.view()
    _check(lib().hgca_append_weights_tiers(ctypes.byref(shape), _ptr(q), int(q.shape[1]), ctypes.byref(kw), ctypes.byref(kp),
                                           int(causal_tail), _ptr(lse_window), _ptr(lse_pool), _ptr(a_gpu), _ptr(a_cpu),
                                           _stream(stream)), "hgca_append_weights_tiers")


def dense_window_attn_maw(shape: Shape, q, window: Tier, o_out, lse_out, a_out, a_maw, n_new: int, alpha: float, ws,
                          stream=None) -> None:
    """dense_window_attn_weights and maw_update(a_maw, a_out, ...) in one call."""
    for t in (q, ws, o_out, lse_out, a_out, a_maw):
        _require_gpu(t)
    kv = window.view()
    _check(lib().hgca_dense_window_attn_maw(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(o_out), _ptr(lse_out),
                                            _ptr(a_out), _ptr(a_maw), int(n_new), float(alpha), _ptr(ws), ws.numel(),
                                            _stream(stream)), "hgca_dense_window_attn_maw")


def select_salient_grouped(shape: Shape, q, pool: Tier, k, k_max: int, idx_out, cnt_out, ws, stream=None) -> None:
    """One list per KV head (idx_out [B,Hkv,k_max], cnt_out [B,Hkv]): top-k of the maximum score over the group."""
    for t in (q, idx_out, cnt_out, ws):
        _require_gpu(t)
    kv = pool.view()
    if isinstance(k, torch.Tensor):
        _require_gpu(k)
        k_ptr, k_uni = _ptr(k), 0
    else:
        k_ptr, k_uni = None, int(k)
    _check(lib().hgca_select_salient_grouped(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), k_ptr, k_uni, int(k_max),
                                             _ptr(idx_out), _ptr(cnt_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_select_salient_grouped")


def union_lists(shape: Shape, idx, cnt, k_max: int, n_positions: int, idx_out, cnt_out, k_max_out: int, status=None,
                stream=None) -> None:
    """Per KV head, the ascending union of its heads' lists."""
    for t in (idx, cnt, idx_out, cnt_out) + (() if status is None else (status,)):
        _require_gpu(t)
    _check(lib().hgca_union_lists(ctypes.byref(shape), _ptr(idx), _ptr(cnt), int(k_max), int(n_positions), _ptr(idx_out),
                                  _ptr(cnt_out), int(k_max_out), _ptr(status), _stream(stream)), "hgca_union_lists")


def sparse_attn_grouped(shape: Shape, q, pool: Tier, idx, cnt, k_max: int, o_out, lse_out, ws, stream=None) -> None:
    """sparse_attn with idx [B,Hkv,k_max], cnt [B,Hkv]: the heads of a group share the list."""
    for t in (q, idx, cnt, ws) + (() if o_out is None else (o_out, lse_out)):
        _require_gpu(t)
    kv = pool.view()
    _check(lib().hgca_sparse_attn_grouped(ctypes.byref(shape), _ptr(q), ctypes.byref(kv), _ptr(idx), _ptr(cnt), int(k_max),
                                          _ptr(o_out), _ptr(lse_out), _ptr(ws), ws.numel(), _stream(stream)),
           "hgca_sparse_attn_grouped")


def hybrid_decode_step(shape: Shape, q, window: Tier, pool: Tier, k, k_max: int, idx_out, cnt_out, o_out, lse_out,
                       ws_dense, ws_sparse, stream=None) -> None:
    """The whole decode step (dense, select, sparse, merge) in one library call."""
    for t in (q, idx_out, cnt_out, o_out, ws_dense, ws_sparse) + (() if lse_out is None else (lse_out,)):
        _require_gpu(t)
    kw, kp = window.view(), pool.view()
    if isinstance(k, torch.Tensor):
        _require_gpu(k)
        k_ptr, k_uni = _ptr(k), 0
    else:
        k_ptr, k_uni = None, int(k)
    _check(lib().hgca_hybrid_decode_step(ctypes.byref(shape), _ptr(q), ctypes.byref(kw), ctypes.byref(kp), k_ptr, k_uni,
                                         int(k_max), _ptr(idx_out), _ptr(cnt_out), _ptr(o_out), _dtype_code(o_out),
                                         _ptr(lse_out), _ptr(ws_dense), ws_dense.numel(), _ptr(ws_sparse),
                                         ws_sparse.numel(), _stream(stream)), "hgca_hybrid_decode_step")


def hybrid_decode_step_selected(shape: Shape, q, window: Tier, pool: Tier, idx, cnt, k_max: int, o_out, lse_out,
                                ws_dense, ws_sparse, stream=None, sel_scores=None) -> None:
    """The decode step over an existing selection (dense window part beside sparse part, merge) in one call."""
    for t in (q, idx, cnt, o_out, ws_dense, ws_sparse) + tuple(x for x in (lse_out, sel_scores) if x is not None):
        _require_gpu(t)
    kw, kp = window.view(), pool.view()
    _check(lib().hgca_hybrid_decode_step_selected(ctypes.byref(shape), _ptr(q), ctypes.byref(kw), ctypes.byref(kp),
                                                  _ptr(idx), _ptr(cnt), int(k_max), _ptr(sel_scores), _ptr(o_out),
                                                  _dtype_code(o_out), _ptr(lse_out), _ptr(ws_dense), ws_dense.numel(),
                                                  _ptr(ws_sparse), ws_sparse.numel(), _stream(stream)),
           "hgca_hybrid_decode_step_selected")


def ctx_compact(shape: Shape, pool: Tier, idx, cnt, k_max: int, k_ctx, v_ctx, ctx_cap: int, first_row=None,
                cnt_out=None, stream=None) -> None:
    """Copies the listed pool entries into per-head contiguous storage k_ctx / v_ctx [B,Hq,ctx_cap,d]."""
    for t in (idx, cnt, k_ctx, v_ctx) + tuple(x for x in (first_row, cnt_out) if x is not None):
        _require_gpu(t)
    kv = pool.view()
    _check(lib().hgca_ctx_compact(ctypes.byref(shape), ctypes.byref(kv), _ptr(idx), _ptr(cnt), int(k_max),
                                  _ptr(first_row), _ptr(k_ctx), _ptr(v_ctx), int(ctx_cap), _ptr(cnt_out),
                                  _stream(stream)), "hgca_ctx_compact")


def managed_decode_step(shape: Shape, state: "CacheState", q, k_in, v_in, alpha: float, beta: float, a_gpu, o_out,
                        lse_out, ws_dense, ws_sparse, stream=None) -> None:
    """One decode step over the managed cache (insert, attend, merge, moving average, eviction) in one call."""
    for t in (q, k_in, v_in, a_gpu, o_out, ws_dense, ws_sparse) + (() if lse_out is None else (lse_out,)):
        _require_gpu(t)
    _check(lib().hgca_managed_decode_step(ctypes.byref(shape), ctypes.byref(state), _ptr(q), _ptr(k_in), _ptr(v_in),
                                          float(alpha), float(beta), _ptr(a_gpu), _ptr(o_out),
                                          _dtype_code(o_out), _ptr(lse_out), _ptr(ws_dense), ws_dense.numel(),
                                          _ptr(ws_sparse), ws_sparse.numel(), _stream(stream)),
           "hgca_managed_decode_step")


# ---- what a step needs beside its attention: norm and rotation, drafted tokens, an 8-bit tier ----

ROPE_INTERLEAVED = 1
MAX_DRAFTS = 64                                  # HGCA_MAX_DRAFTS of include/hgca.h


@dataclass
class Kv8Tier:
    """A tier in 8 bits: k, v uint8 [B,Hkv,cap,d] or [n_blocks,Hkv,bs,d] (E4M3), k_scale, v_scale uint8 [...,d/32] (E8M0)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    cap: int
    seq_lens: Optional[torch.Tensor] = None      # int32 [B]
    block_table: Optional[torch.Tensor] = None   # int32 [B,max_blocks]
    block_size: int = 0
    first_block: Optional[torch.Tensor] = None   # int32 [B]

    @staticmethod
    def like(tier: "Tier") -> "Kv8Tier":
        """Zeroed 8-bit storage for the rows of `tier`, with its lengths and block table."""
        rows, d = tier.k.shape[:-1], int(tier.k.shape[-1])
        z = lambda n: torch.zeros(*rows, n, dtype=torch.uint8, device=tier.k.device)
        return Kv8Tier(z(d), z(d), z(d // 32), z(d // 32), tier.cap, tier.seq_lens, tier.block_table, tier.block_size,
                       tier.first_block)

    def view(self) -> Kv8View:
        mb = 0 if self.block_table is None else int(self.block_table.shape[1])
        return Kv8View(_ptr(self.k), _ptr(self.v), _ptr(self.k_scale), _ptr(self.v_scale), _ptr(self.seq_lens),
                       _ptr(self.block_table), int(self.cap), int(self.block_size), mb, _ptr(self.first_block))


def _need(name: str, t: torch.Tensor, dtype, size: tuple, dev: int) -> None:
    """The tensor has this type and size, is dense and lies on GPU `dev`."""
    if t.shape != size or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _refuse(name, t, dtype, size, dev)


def _refuse(name: str, t: torch.Tensor, dtype, size: tuple, dev: int) -> None:
    if t.dtype is not dtype or t.shape != size:
        raise ValueError(f"{name} must be {dtype} of size {list(size)}, got {t.dtype} of size {list(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the other tensors on cuda:{dev}")
    raise ValueError(f"{name}: libhgca takes contiguous tensors")


def _gpu_of(t: torch.Tensor) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("libhgca takes GPU tensors only (no CPU path exists)")
    return dev


def _tier_view(tier, B: int, H: int, d: int, dtype, dev: int):
    """The view of a tier whose tensors have been checked: rows of every sequence and KV head, lengths, table."""
    k, v, lens, table, first, cap, bs = tier.k, tier.v, tier.seq_lens, tier.block_table, tier.first_block, int(tier.cap), 0
    rows, mb = (B, H, cap), 0
    if table is not None:
        bs = int(tier.block_size)
        rows, mb = (k.shape[0], H, bs), int(table.shape[1])
        _need("tier.block_table", table, torch.int32, (B, mb), dev)
        if first is not None:
            _need("tier.first_block", first, torch.int32, (B,), dev)
    _need("tier.k", k, dtype, rows + (d,), dev)
    _need("tier.v", v, dtype, rows + (d,), dev)
    if lens is not None:
        _need("tier.seq_lens", lens, torch.int32, (B,), dev)
    if dtype is torch.uint8:
        ks, vs = tier.k_scale, tier.v_scale
        _need("tier.k_scale", ks, dtype, rows + (d // 32,), dev)
        _need("tier.v_scale", vs, dtype, rows + (d // 32,), dev)
        return Kv8View(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), _ptr(lens), _ptr(table), cap, bs, mb, _ptr(first))
    return KvView(k.data_ptr(), v.data_ptr(), _ptr(lens), _ptr(table), cap, bs, mb, _ptr(first))


def _launch(where: str, stream, dev: int, *args) -> None:
    """Calls `where` on GPU `dev`, on the given stream or the current one there.  (A call's checks and views take the host about as
    long as the launch: 4 of 8 us.)"""
    call = getattr(_lib or lib(), where)
    if stream is None and _raw_stream is not None and _device is not None and _device() == dev:
        status = call(*args, _raw_stream(dev))
    else:
        if stream is not None and stream.device.index != dev:
            raise ValueError(f"{where}: tensors on cuda:{dev}, stream on {stream.device}")
        with torch.cuda.device(dev):
            status = call(*args, _stream(stream))
    if status:
        raise HgcaError(status, where)


_TORCH_DTYPE = {F32: torch.float32, BF16: torch.bfloat16}


def _heads(shape: Shape):
    """Sizes and the tensors' type; another dtype code is the library's to refuse."""
    return shape.batch, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, _TORCH_DTYPE.get(shape.dtype, torch.bfloat16)


def _token_stride(name: str, t: torch.Tensor) -> int:
    """Elements between consecutive tokens of [B,n,H,d], whose heads lie side by side."""
    (B, n, H, d), (s0, s1, s2, s3) = t.shape, t.stride()
    step = s1 if n > 1 else s0 if B > 1 else H * d
    # (an expanded tensor's distance is 0, which the library takes as rows one behind the other)
    if s3 != 1 or (s2 != d and H > 1) or (s0 != n * step and B > 1 and n > 1) or (step < H * d and B * n > 1):
        raise ValueError(f"{name}: heads have to lie side by side and tokens at one distance")
    return step


def qk_norm_rope(shape: Shape, q, k, q_out, k_out, inv_freq, q_weight=None, k_weight=None, eps: float = 1e-6,
                 positions=None, first_pos=None, interleaved: bool = False, stream=None) -> None:
    """q [B,n,Hq,d] and k [B,n,Hkv,d] normed per head and rotated by position into q_out, k_out (dense; may be q, k where
    those are).  q and k may be parts of wider rows (a fused projection's).  inv_freq fp32 [rot/2]; positions int32 [B,n], or
    first_pos int32 [B] for consecutive ones."""
    B, Hq, Hkv, d, dt = _heads(shape)
    dev, n = _gpu_of(q), q.shape[1]
    if q.dtype is not dt or q.shape != (B, n, Hq, d) or k.dtype is not dt or k.shape != (B, n, Hkv, d) or k.get_device() != dev:
        raise ValueError(f"q and k must be {dt} of sizes {[B, n, Hq, d]} and {[B, n, Hkv, d]} on one GPU, got {q.dtype} {list(q.shape)} "
                         f"and {k.dtype} {list(k.shape)}")
    _need("q_out", q_out, dt, (B, n, Hq, d), dev)
    _need("k_out", k_out, dt, (B, n, Hkv, d), dev)
    half = inv_freq.numel()
    _need("inv_freq", inv_freq, torch.float32, (half,), dev)
    if q_weight is not None:
        _need("q_weight", q_weight, dt, (d,), dev)
    if k_weight is not None:
        _need("k_weight", k_weight, dt, (d,), dev)
    if positions is not None:
        _need("positions", positions, torch.int32, (B, n), dev)
    if first_pos is not None:
        _need("first_pos", first_pos, torch.int32, (B,), dev)
    _launch("hgca_qk_norm_rope", stream, dev, ctypes.byref(shape), q.data_ptr(), _token_stride("q", q), k.data_ptr(),
            _token_stride("k", k), n, _ptr(q_weight), _ptr(k_weight), eps, inv_freq.data_ptr(), 2 * half, _ptr(positions),
            _ptr(first_pos), ROPE_INTERLEAVED if interleaved else 0, q_out.data_ptr(), k_out.data_ptr())


def tree_workspace(shape: Shape, n_q: int, max_tokens: int, device) -> torch.Tensor:
    n = int(lib().hgca_tree_workspace_bytes(ctypes.byref(shape), int(n_q), int(max_tokens)))
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_tree_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _rows_call(where: str, shape: Shape, q, tier, tier_dtype, mask, o_out, lse_out, ws, stream) -> None:
    B, Hq, Hkv, d, dt = _heads(shape)
    dev, n = _gpu_of(q), q.shape[1]
    _need("q", q, dt, (B, n, Hq, d), dev)
    _need("o_out", o_out, torch.bfloat16 if o_out.dtype is torch.bfloat16 else torch.float32, (B, n, Hq, d), dev)
    _need("lse_out", lse_out, torch.float32, (B, n, Hq), dev)
    _need("ws", ws, torch.uint8, (ws.numel(),), dev)
    kv = _tier_view(tier, B, Hkv, d, tier_dtype or dt, dev)
    if tier_dtype is None:
        if mask is not None:
            _need("mask", mask, torch.int64, (B, n), dev)
        _launch(where, stream, dev, ctypes.byref(shape), q.data_ptr(), n, ctypes.byref(kv), _ptr(mask), o_out.data_ptr(),
                _dtype_code(o_out), lse_out.data_ptr(), ws.data_ptr(), ws.numel())
    else:
        _launch(where, stream, dev, ctypes.byref(shape), q.data_ptr(), n, ctypes.byref(kv), o_out.data_ptr(), _dtype_code(o_out),
                lse_out.data_ptr(), ws.data_ptr(), ws.numel())


def tree_attn(shape: Shape, q, tier: Tier, mask, o_out, lse_out, ws, stream=None) -> None:
    """Attention of q [B,n,Hq,d], n <= MAX_DRAFTS drafted tokens that are the tier's last n, over the tier; mask int64 [B,n]: bit
    j of mask[b,i] = query i sees draft j (None: all).  o_out [B,n,Hq,d] fp32 or bf16, lse_out [B,n,Hq] fp32."""
    _rows_call("hgca_tree_attn", shape, q, tier, None, mask, o_out, lse_out, ws, stream)


def _first_and_status(B: int, dev: int, first, status=None) -> None:
    if first is not None:
        _need("first", first, torch.int32, (B,), dev)
    if status is not None:
        _need("status", status, torch.int32, (1,), dev)


def kv_commit(shape: Shape, tier: Tier, first, k_in, v_in, lens_out, path=None, cnt=None, status=None, stream=None) -> None:
    """Rows path[b,i], i < cnt[b], of k_in / v_in [B,n,Hkv,d] go to positions first[b] + i of the tier; lens_out[b] = first[b] +
    cnt[b].  path int32 [B,n] (None: row i), cnt int32 [B] (None: n), first int32 [B] (None: 0).  With n = 0 nothing is written,
    lens_out neither."""
    B, _, Hkv, d, dt = _heads(shape)
    dev, n = _gpu_of(k_in), k_in.shape[1]
    _need("k_in", k_in, dt, (B, n, Hkv, d), dev)
    _need("v_in", v_in, dt, (B, n, Hkv, d), dev)
    _need("lens_out", lens_out, torch.int32, (B,), dev)
    if path is not None:
        _need("path", path, torch.int32, (B, n), dev)
    if cnt is not None:
        _need("cnt", cnt, torch.int32, (B,), dev)
    _first_and_status(B, dev, first, status)
    kv = _tier_view(tier, B, Hkv, d, dt, dev)
    _launch("hgca_kv_commit", stream, dev, ctypes.byref(shape), ctypes.byref(kv), _ptr(first), k_in.data_ptr(), v_in.data_ptr(), n,
            _ptr(path), _ptr(cnt), _ptr(lens_out), _ptr(status))


def kv8_write_tokens(shape: Shape, tier: Kv8Tier, first, k_in, v_in, status=None, stream=None) -> None:
    """k_in / v_in [B,n,Hkv,d] in 8 bits to positions first[b] .. (int32 [B], None: 0)."""
    B, _, Hkv, d, dt = _heads(shape)
    dev, n = _gpu_of(k_in), k_in.shape[1]
    _need("k_in", k_in, dt, (B, n, Hkv, d), dev)
    _need("v_in", v_in, dt, (B, n, Hkv, d), dev)
    _first_and_status(B, dev, first, status)
    kv8 = _tier_view(tier, B, Hkv, d, torch.uint8, dev)
    _launch("hgca_kv8_write_tokens", stream, dev, ctypes.byref(shape), ctypes.byref(kv8), _ptr(first), k_in.data_ptr(),
            v_in.data_ptr(), n, _ptr(status))


def kv8_write_tier(shape: Shape, tier: Kv8Tier, first, src: Tier, max_tokens: int, status=None, stream=None) -> None:
    """Tokens first[b] .. src.seq_lens[b] - 1 of src (max_tokens per sequence at most) in 8 bits to the same positions."""
    B, _, Hkv, d, dt = _heads(shape)
    dev = _gpu_of(src.k)
    _first_and_status(B, dev, first, status)
    kv8, kv = _tier_view(tier, B, Hkv, d, torch.uint8, dev), _tier_view(src, B, Hkv, d, dt, dev)
    _launch("hgca_kv8_write_tier", stream, dev, ctypes.byref(shape), ctypes.byref(kv8), _ptr(first), ctypes.byref(kv),
            int(max_tokens), _ptr(status))


def kv8_read(shape: Shape, tier: Kv8Tier, first, k_out, v_out, stream=None) -> None:
    """Tokens first[b] .. of an 8-bit tier as rows k_out / v_out [B,n,Hkv,d]; rows of tokens beyond the length stay."""
    B, _, Hkv, d, dt = _heads(shape)
    dev, n = _gpu_of(k_out), k_out.shape[1]
    _need("k_out", k_out, dt, (B, n, Hkv, d), dev)
    _need("v_out", v_out, dt, (B, n, Hkv, d), dev)
    _first_and_status(B, dev, first)
    kv8 = _tier_view(tier, B, Hkv, d, torch.uint8, dev)
    _launch("hgca_kv8_read", stream, dev, ctypes.byref(shape), ctypes.byref(kv8), _ptr(first), n, k_out.data_ptr(), v_out.data_ptr())


def kv8_workspace(shape: Shape, n_q: int, max_tokens: int, device) -> torch.Tensor:
    n = int(lib().hgca_kv8_workspace_bytes(ctypes.byref(shape), int(n_q), int(max_tokens)))
    if n == 0:
        raise HgcaError(ERR_INVALID_ARG, "hgca_kv8_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def kv8_attn(shape: Shape, q, tier: Kv8Tier, o_out, lse_out, ws, stream=None) -> None:
    """Attention of q [B,n,Hq,d] over every valid token of an 8-bit tier; o_out [B,n,Hq,d] fp32 or bf16, lse_out fp32."""
    _rows_call("hgca_kv8_attn", shape, q, tier, torch.uint8, None, o_out, lse_out, ws, stream)
