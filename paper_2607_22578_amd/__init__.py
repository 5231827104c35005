"""Python binding of libhsmerge.so (merged retrieval on MI355X / gfx950).

Argument marshalling only: every step runs in the HIP kernels of the shared
library.  Functions carry the C names of include/hs_merge.h and take device
buffers as torch tensors (or raw integer addresses); PyTorch serves only to
own device memory and streams.  Importing fails loudly when the library has
not been built -- there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhsmerge.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                      "(hipcc --offload-arch=gfx950)")

# torch ships its own HIP runtime.  Load it first so that the library binds to
# the same runtime instance (by soname) instead of bringing a second runtime
# into the process; two runtimes cannot share the device.
try:
    import torch as _torch  # noqa: F401
except ImportError:  # plain C-ABI use without torch
    _torch = None

_lib = ctypes.CDLL(LIB_PATH)

HS_OK, HS_ERR_INVALID_ARG, HS_ERR_UNSUPPORTED, HS_ERR_WORKSPACE, HS_ERR_ALIGNMENT, \
    HS_ERR_DEVICE = range(6)
HS_F32, HS_BF16, HS_FP8_E4M3, HS_FP4_E2M1 = 0, 1, 2, 3
ABI_VERSION = 3

EXPORTS = ["hs_merge_plan", "hs_plan_destroy", "hs_workflow_rows", "hs_dedup", "hs_score_topk",
           "hs_score_topk_noalloc", "hs_score_partial", "hs_topk_merge", "hs_corpus_tiled_bytes",
           "hs_tile_corpus", "hs_scatter", "hs_deliver",
           "hs_cache_bytes", "hs_cache_reset", "hs_cache_lookup",
           "hs_cache_insert", "hs_signature", "hs_priority",
           "hs_pack_rows", "hs_embed", "hs_embed_grad_bytes", "hs_embed_grad",
           "hs_score_packed", "hs_adjust_scores", "hs_topk_rows_bytes", "hs_topk_rows",
           "hs_status_string", "hs_last_error", "hs_abi_version"]
HS_SIG_NORMALIZE_TEXT = 1
HS_FLAG_TILED_CORPUS = 1


class hs_merge_desc(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("n_corpus", ctypes.c_int64), ("k", ctypes.c_int32),
                ("query_dtype", ctypes.c_int32), ("corpus_dtype", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("max_unique", ctypes.c_int64),
                ("n_workflows", ctypes.c_int64),
                ("workflow_offsets", ctypes.POINTER(ctypes.c_int64))]


class hs_sig_nodes(ctypes.Structure):
    _fields_ = [("op_type", ctypes.c_void_p), ("params", ctypes.c_void_p),
                ("param_off", ctypes.c_void_p), ("param_bytes", ctypes.c_int64),
                ("text", ctypes.c_void_p), ("text_off", ctypes.c_void_p),
                ("text_bytes", ctypes.c_int64), ("pred_off", ctypes.c_void_p),
                ("pred_idx", ctypes.c_void_p), ("pred_count", ctypes.c_int64),
                ("n_nodes", ctypes.c_int64)]


class hs_row_table(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("dim", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("scale_dtype", ctypes.c_int32), ("group", ctypes.c_int32)]


class hs_adjust(ctypes.Structure):
    _fields_ = [("seen_off", ctypes.c_void_p), ("seen", ctypes.c_void_p),
                ("n_seen", ctypes.c_int64), ("prompt_len", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("bias_off", ctypes.c_void_p),
                ("bias_id", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("n_bias", ctypes.c_int64), ("allow", ctypes.c_void_p),
                ("allow_stride", ctypes.c_int64)]


_vp, _i64, _i32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
_lib.hs_merge_plan.argtypes = [ctypes.POINTER(hs_merge_desc), ctypes.POINTER(_vp),
                               ctypes.POINTER(_sz)]
_lib.hs_merge_plan.restype = ctypes.c_int
_lib.hs_plan_destroy.argtypes = [_vp]
_lib.hs_plan_destroy.restype = None
_lib.hs_workflow_rows.argtypes = [_vp, _i64, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
_lib.hs_workflow_rows.restype = ctypes.c_int
_lib.hs_deliver.argtypes = [_vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp]
_lib.hs_deliver.restype = ctypes.c_int
_lib.hs_dedup.argtypes = [_vp] + [_vp] * 7 + [_vp, _sz, _vp]
_lib.hs_dedup.restype = ctypes.c_int
_lib.hs_score_topk.argtypes = [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.hs_score_topk.restype = ctypes.c_int
_lib.hs_score_topk_noalloc.argtypes = [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.hs_score_topk_noalloc.restype = ctypes.c_int
_lib.hs_score_partial.argtypes = [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.hs_score_partial.restype = ctypes.c_int
_lib.hs_topk_merge.argtypes = [_vp, _i64, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.hs_topk_merge.restype = ctypes.c_int
_lib.hs_corpus_tiled_bytes.argtypes = [_vp, ctypes.POINTER(_sz)]
_lib.hs_corpus_tiled_bytes.restype = ctypes.c_int
_lib.hs_tile_corpus.argtypes = [_vp, _vp, _vp, _sz, _vp]
_lib.hs_tile_corpus.restype = ctypes.c_int
_lib.hs_scatter.argtypes = [_vp, _i64, _i64, _vp, _i32, _i64, _vp, _vp, _vp]
_lib.hs_scatter.restype = ctypes.c_int
_lib.hs_cache_bytes.argtypes = [_vp, _i64, ctypes.POINTER(_sz)]
_lib.hs_cache_bytes.restype = ctypes.c_int
_lib.hs_cache_reset.argtypes = [_vp, _vp, _sz, _i64, _vp]
_lib.hs_cache_reset.restype = ctypes.c_int
_lib.hs_cache_lookup.argtypes = [_vp, _vp, _sz, _i64, _vp, _vp, _i64] + [_vp] * 7
_lib.hs_cache_lookup.restype = ctypes.c_int
_lib.hs_cache_insert.argtypes = [_vp, _vp, _sz, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _vp]
_lib.hs_cache_insert.restype = ctypes.c_int
_lib.hs_signature.argtypes = [ctypes.POINTER(hs_sig_nodes), _i64, _i64, _i32, _vp, _vp, _vp]
_lib.hs_signature.restype = ctypes.c_int
_dbl = ctypes.c_double
_lib.hs_priority.argtypes = ([_vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _dbl, _dbl, _dbl, _dbl]
                             + [_vp] * 4 + [_sz, _vp])
_lib.hs_priority.restype = ctypes.c_int
_flt = ctypes.c_float
_lib.hs_pack_rows.argtypes = [_vp, _i32, _i64, _i64, _i32, _i32, _vp, _vp, _vp]
_lib.hs_pack_rows.restype = ctypes.c_int
_lib.hs_embed.argtypes = [ctypes.POINTER(hs_row_table), _vp, _i32, _i64, _flt, _i64, _vp, _i32,
                          _vp]
_lib.hs_embed.restype = ctypes.c_int
_lib.hs_embed_grad_bytes.argtypes = [_i64, _i64, _i64, ctypes.POINTER(_sz)]
_lib.hs_embed_grad_bytes.restype = ctypes.c_int
_lib.hs_embed_grad.argtypes = [_vp, _i32, _vp, _i32, _i64, _i64, _i64, _flt, _i64, _i32, _vp, _i32,
                               _vp, _sz, _vp]
_lib.hs_embed_grad.restype = ctypes.c_int
_lib.hs_score_packed.argtypes = [ctypes.POINTER(hs_row_table), _vp, _i32, _i64, _vp, _i32, _i64,
                                 _vp]
_lib.hs_score_packed.restype = ctypes.c_int
_lib.hs_adjust_scores.argtypes = [ctypes.POINTER(hs_adjust), _vp, _i64, _vp, _i64, _i32, _i64,
                                  _i64, _vp]
_lib.hs_adjust_scores.restype = ctypes.c_int
_lib.hs_topk_rows_bytes.argtypes = [_i64, _i64, _i32, ctypes.POINTER(_sz)]
_lib.hs_topk_rows_bytes.restype = ctypes.c_int
_lib.hs_topk_rows.argtypes = [_vp, _i32, _i64, _i64, _i64, _i32, _vp, _vp, _vp, _sz, _vp]
_lib.hs_topk_rows.restype = ctypes.c_int
_lib.hs_status_string.argtypes = [ctypes.c_int]
_lib.hs_status_string.restype = ctypes.c_char_p
_lib.hs_last_error.argtypes = []
_lib.hs_last_error.restype = ctypes.c_char_p
_lib.hs_abi_version.argtypes = []
_lib.hs_abi_version.restype = ctypes.c_int32


class HsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{hs_status_string(status)}: {msg}")
        self.status = status


def hs_status_string(status: int) -> str:
    return _lib.hs_status_string(status).decode()


def hs_last_error() -> str:
    return _lib.hs_last_error().decode()


def hs_abi_version() -> int:
    return int(_lib.hs_abi_version())


def _check(status: int):
    if status != HS_OK:
        raise HsError(status, hs_last_error())


def _ptr(x):
    """Device/host address of a torch tensor, an int address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dtype_code(t) -> int:
    """HS dtype of a torch tensor (float32, bfloat16, uint8/float8_e4m3fn)."""
    import torch
    m = {torch.float32: HS_F32, torch.bfloat16: HS_BF16, torch.uint8: HS_FP8_E4M3,
         torch.float8_e4m3fn: HS_FP8_E4M3}
    if t.dtype not in m:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return m[t.dtype]


@dataclass
class Plan:
    handle: int
    workspace_bytes: int
    desc: hs_merge_desc

    def __del__(self):
        # (at interpreter exit the module's globals may already be gone)
        if self.handle and _lib is not None:
            _lib.hs_plan_destroy(self.handle)
            self.handle = 0


def hs_merge_plan(n_requests: int, dim: int, n_corpus: int, k: int, query_dtype: int,
                  corpus_dtype: int, max_unique: int = 0, flags: int = 0,
                  n_workflows: int = 1, workflow_offsets=None) -> Plan:
    """workflow_offsets: None (uniform) or a sequence of n_workflows + 1
    request offsets (host CSR)."""
    off = None
    if workflow_offsets is not None:
        vals = [int(x) for x in workflow_offsets]
        off = (ctypes.c_int64 * max(len(vals), 1))(*vals)
    d = hs_merge_desc(n_requests, dim, n_corpus, k, query_dtype, corpus_dtype, flags, max_unique,
                      n_workflows, ctypes.cast(off, ctypes.POINTER(ctypes.c_int64))
                      if off is not None else None)
    h = _vp()
    ws = _sz()
    _check(_lib.hs_merge_plan(ctypes.byref(d), ctypes.byref(h), ctypes.byref(ws)))
    d.workflow_offsets = None   # the plan keeps its own copy
    return Plan(h.value, int(ws.value), d)


def hs_workflow_rows(plan: Plan, w: int):
    """(first, count): rows of workflow w in the per-request outputs."""
    a, b = _i64(), _i64()
    _check(_lib.hs_workflow_rows(plan.handle, w, ctypes.byref(a), ctypes.byref(b)))
    return int(a.value), int(b.value)


def hs_deliver(plan: Plan, topk_score, topk_index, topk_rows: int, inverse, out_score, out_index,
               stream=None):
    _check(_lib.hs_deliver(plan.handle, _ptr(topk_score), _ptr(topk_index), topk_rows,
                           _ptr(inverse), _ptr(out_score), _ptr(out_index), _stream(stream)))


def hs_dedup(plan: Plan, keys, unique_keys, first_index, counts, inverse, n_unique_dev,
             n_unique_host=None, ws=None, ws_bytes: Optional[int] = None, stream=None):
    host = None
    if n_unique_host is True:
        host = ctypes.c_int64(-1)
        hptr = ctypes.addressof(host)
    else:
        hptr = _ptr(n_unique_host)
    _check(_lib.hs_dedup(plan.handle, _ptr(keys), _ptr(unique_keys), _ptr(first_index),
                         _ptr(counts), _ptr(inverse), _ptr(n_unique_dev), hptr, _ptr(ws),
                         _ws_bytes(ws, ws_bytes), _stream(stream)))
    return None if host is None else int(host.value)


def _ws_bytes(ws, ws_bytes):
    if ws_bytes is not None:
        return ws_bytes
    if ws is None or isinstance(ws, int):
        return 0
    return ws.numel() * ws.element_size()


def hs_score_topk(plan: Plan, q_unique, n_unique: int, n_unique_dev, corpus, row_scale,
                  topk_score, topk_index, ws=None, ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_score_topk(plan.handle, _ptr(q_unique), n_unique, _ptr(n_unique_dev),
                              _ptr(corpus), _ptr(row_scale), _ptr(topk_score), _ptr(topk_index),
                              _ptr(ws), _ws_bytes(ws, ws_bytes), _stream(stream)))


def hs_corpus_tiled_bytes(plan: Plan) -> int:
    n = _sz()
    _check(_lib.hs_corpus_tiled_bytes(plan.handle, ctypes.byref(n)))
    return int(n.value)


def hs_tile_corpus(plan: Plan, corpus, tiled, tiled_bytes: Optional[int] = None, stream=None):
    if tiled_bytes is None:
        tiled_bytes = tiled.numel() * tiled.element_size() if tiled is not None else 0
    _check(_lib.hs_tile_corpus(plan.handle, _ptr(corpus), _ptr(tiled), tiled_bytes,
                               _stream(stream)))


def hs_score_topk_noalloc(plan: Plan, q_unique, n_unique: int, n_unique_dev, corpus, row_scale,
                          topk_score, topk_index, stream=None):
    _check(_lib.hs_score_topk_noalloc(plan.handle, _ptr(q_unique), n_unique, _ptr(n_unique_dev),
                                      _ptr(corpus), _ptr(row_scale), _ptr(topk_score),
                                      _ptr(topk_index), _stream(stream)))


def hs_score_partial(plan: Plan, q_unique, n_unique: int, n_unique_dev, corpus, row_scale,
                     ws=None, ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_score_partial(plan.handle, _ptr(q_unique), n_unique, _ptr(n_unique_dev),
                                 _ptr(corpus), _ptr(row_scale), _ptr(ws),
                                 _ws_bytes(ws, ws_bytes), _stream(stream)))


def hs_topk_merge(plan: Plan, n_unique: int, n_unique_dev, topk_score, topk_index, ws=None,
                  ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_topk_merge(plan.handle, n_unique, _ptr(n_unique_dev), _ptr(topk_score),
                              _ptr(topk_index), _ptr(ws), _ws_bytes(ws, ws_bytes),
                              _stream(stream)))


def hs_scatter(src, src_rows: int, row_bytes: int, index, index_is_i64: int, n_out: int,
               n_out_dev, dst, stream=None):
    _check(_lib.hs_scatter(_ptr(src), src_rows, row_bytes, _ptr(index), index_is_i64, n_out,
                           _ptr(n_out_dev), _ptr(dst), _stream(stream)))


def hs_cache_bytes(plan: Plan, capacity: int) -> int:
    b = _sz()
    _check(_lib.hs_cache_bytes(plan.handle, capacity, ctypes.byref(b)))
    return int(b.value)


def hs_cache_reset(plan: Plan, cache, capacity: int, cache_bytes: Optional[int] = None,
                   stream=None):
    _check(_lib.hs_cache_reset(plan.handle, _ptr(cache), _ws_bytes(cache, cache_bytes), capacity,
                               _stream(stream)))


def hs_cache_lookup(plan: Plan, cache, capacity: int, unique_keys, first_index, n_unique: int,
                    n_unique_dev, topk_score, topk_index, miss_pos, miss_first, n_miss_dev,
                    cache_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_cache_lookup(plan.handle, _ptr(cache), _ws_bytes(cache, cache_bytes), capacity,
                                _ptr(unique_keys), _ptr(first_index), n_unique,
                                _ptr(n_unique_dev), _ptr(topk_score), _ptr(topk_index),
                                _ptr(miss_pos), _ptr(miss_first), _ptr(n_miss_dev),
                                _stream(stream)))


def hs_cache_insert(plan: Plan, cache, capacity: int, unique_keys, miss_pos, n_unique: int,
                    n_unique_dev, topk_score, topk_index, cache_bytes: Optional[int] = None,
                    stream=None):
    _check(_lib.hs_cache_insert(plan.handle, _ptr(cache), _ws_bytes(cache, cache_bytes), capacity,
                                _ptr(unique_keys), _ptr(miss_pos), n_unique, _ptr(n_unique_dev),
                                _ptr(topk_score), _ptr(topk_index), _stream(stream)))


def _nbytes(x):
    if x is None or isinstance(x, int):
        return 0
    return x.numel() * x.element_size()


def hs_signature(op_type, n_nodes: int, first: int, count: int, digest, keys=None, params=None,
                 param_off=None, text=None, text_off=None, pred_off=None, pred_idx=None,
                 flags: int = 0, param_bytes: Optional[int] = None,
                 text_bytes: Optional[int] = None, pred_count: Optional[int] = None,
                 stream=None):
    """Signatures of nodes [first, first + count) (digests and 64-bit keys);
    buffer sizes default to the tensors' sizes."""
    nd = hs_sig_nodes(_ptr(op_type), _ptr(params), _ptr(param_off),
                      _nbytes(params) if param_bytes is None else param_bytes,
                      _ptr(text), _ptr(text_off), _nbytes(text) if text_bytes is None else text_bytes,
                      _ptr(pred_off), _ptr(pred_idx),
                      (_nbytes(pred_idx) // 4) if pred_count is None else pred_count, n_nodes)
    _check(_lib.hs_signature(ctypes.byref(nd), first, count, flags, _ptr(digest), _ptr(keys),
                             _stream(stream)))


def hs_priority(plan: Plan, inverse, first_index, n_unique: int, n_unique_dev, phi, s_hat, heavy,
                alpha: float, gamma: float, delta: float, eps: float, phi_fused, pi, order,
                ws=None, ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_priority(plan.handle, _ptr(inverse), _ptr(first_index), n_unique,
                            _ptr(n_unique_dev), _ptr(phi), _ptr(s_hat), _ptr(heavy), alpha, gamma,
                            delta, eps, _ptr(phi_fused), _ptr(pi), _ptr(order), _ptr(ws),
                            _ws_bytes(ws, ws_bytes), _stream(stream)))


def hs_pack_rows(src, src_dtype: int, rows: int, dim: int, group: int, scale_dtype: int, codes,
                 scale, stream=None):
    _check(_lib.hs_pack_rows(_ptr(src), src_dtype, rows, dim, group, scale_dtype, _ptr(codes),
                             _ptr(scale), _stream(stream)))


def hs_embed(table: hs_row_table, ids, ids_is_i64: int, n: int, scale: float, pad_id: int, out,
             out_dtype: int, stream=None):
    _check(_lib.hs_embed(ctypes.byref(table), _ptr(ids), ids_is_i64, n, scale, pad_id, _ptr(out),
                         out_dtype, _stream(stream)))


def hs_embed_grad_bytes(n: int, rows: int, dim: int) -> int:
    b = _sz()
    _check(_lib.hs_embed_grad_bytes(n, rows, dim, ctypes.byref(b)))
    return int(b.value)


def hs_embed_grad(d_out, d_out_dtype: int, ids, ids_is_i64: int, n: int, rows: int, dim: int,
                  scale: float, pad_id: int, accumulate: int, d_table, d_table_dtype: int,
                  ws=None, ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_embed_grad(_ptr(d_out), d_out_dtype, _ptr(ids), ids_is_i64, n, rows, dim, scale,
                              pad_id, accumulate, _ptr(d_table), d_table_dtype, _ptr(ws),
                              _ws_bytes(ws, ws_bytes), _stream(stream)))


def hs_score_packed(table: hs_row_table, x, x_dtype: int, n_x: int, out, out_dtype: int,
                    out_stride: int, stream=None):
    _check(_lib.hs_score_packed(ctypes.byref(table), _ptr(x), x_dtype, n_x, _ptr(out), out_dtype,
                                out_stride, _stream(stream)))


def hs_adjust_scores(adjust: hs_adjust, scores, stride: int, out, out_stride: int, dtype: int,
                     n_rows: int, n_cols: int, stream=None):
    _check(_lib.hs_adjust_scores(ctypes.byref(adjust), _ptr(scores), stride, _ptr(out), out_stride,
                                 dtype, n_rows, n_cols, _stream(stream)))


def hs_topk_rows_bytes(n_rows: int, n_cols: int, k: int) -> int:
    b = _sz()
    _check(_lib.hs_topk_rows_bytes(n_rows, n_cols, k, ctypes.byref(b)))
    return int(b.value)


def hs_topk_rows(scores, dtype: int, stride: int, n_rows: int, n_cols: int, k: int, topk_score,
                 topk_index, ws=None, ws_bytes: Optional[int] = None, stream=None):
    _check(_lib.hs_topk_rows(_ptr(scores), dtype, stride, n_rows, n_cols, k, _ptr(topk_score),
                             _ptr(topk_index), _ptr(ws), _ws_bytes(ws, ws_bytes),
                             _stream(stream)))


# ---------------------------------------------------------------- composition

class MergedRetrieval:
    """Owns the plan, workspace and per-window buffers for one shape and runs
    the whole path (dedup -> representative rows -> score/top-k -> delivery)
    on one stream.  All outputs are torch tensors on the device."""

    def __init__(self, n_requests: int, dim: int, n_corpus: int, k: int, query_dtype: int,
                 corpus_dtype: int, device="cuda", max_unique: int = 0, n_workflows: int = 1,
                 workflow_offsets=None, tiled_corpus: bool = False):
        """tiled_corpus: the score calls take the corpus in the tiled layout
        (make it once with tile_corpus)."""
        import torch
        self.R, self.d, self.N, self.k = n_requests, dim, n_corpus, k
        self.qdt, self.cdt = query_dtype, corpus_dtype
        self.tiled_corpus = tiled_corpus
        self.plan = hs_merge_plan(n_requests, dim, n_corpus, k, query_dtype, corpus_dtype,
                                  max_unique, flags=HS_FLAG_TILED_CORPUS if tiled_corpus else 0,
                                  n_workflows=n_workflows,
                                  workflow_offsets=workflow_offsets)
        self.n_workflows = n_workflows
        cap = max_unique if max_unique > 0 else n_requests
        self.cap = cap
        dev = torch.device(device)
        R1 = max(n_requests, 1)
        qt = torch.float32 if query_dtype == HS_F32 else torch.bfloat16
        self.ws = torch.empty(max(self.plan.workspace_bytes, 256), dtype=torch.uint8, device=dev)
        self.unique_keys = torch.empty(R1, dtype=torch.int64, device=dev)
        self.first_index = torch.empty(R1, dtype=torch.int32, device=dev)
        self.counts = torch.empty(R1, dtype=torch.int32, device=dev)
        self.inverse = torch.empty(R1, dtype=torch.int32, device=dev)
        self.n_unique = torch.zeros(1, dtype=torch.int64, device=dev)
        # rows for every distinct query of a window (more than one batch of
        # max_unique when the window has more distinct keys)
        self.q_unique = torch.empty((R1, dim), dtype=qt, device=dev)
        self.topk_score = torch.empty((R1, k), dtype=torch.float32, device=dev)
        self.topk_index = torch.empty((R1, k), dtype=torch.int32, device=dev)
        self.out_score = torch.empty((R1, k), dtype=torch.float32, device=dev)
        self.out_index = torch.empty((R1, k), dtype=torch.int32, device=dev)
        self.q_row_bytes = dim * (4 if query_dtype == HS_F32 else 2)

    def tile_corpus(self, corpus, stream=None):
        """The tiled copy of a row-major BF16/FP8 corpus (a new device tensor),
        for a MergedRetrieval made with tiled_corpus=True."""
        import torch
        out = torch.empty(max(hs_corpus_tiled_bytes(self.plan), 16), dtype=torch.uint8,
                          device=corpus.device)
        hs_tile_corpus(self.plan, corpus, out, stream=stream)
        return out

    def dedup(self, keys, stream=None, host_count: bool = False):
        return hs_dedup(self.plan, keys, self.unique_keys, self.first_index, self.counts,
                        self.inverse, self.n_unique, True if host_count else None, self.ws,
                        stream=stream)

    def gather_queries(self, q_req, stream=None):
        hs_scatter(q_req, self.R, self.q_row_bytes, self.first_index, 0, self.cap,
                   self.n_unique, self.q_unique, stream=stream)

    def score_partial(self, corpus, scale=None, n_unique: int = -1, stream=None):
        hs_score_partial(self.plan, self.q_unique, n_unique, self.n_unique, corpus, scale,
                         self.ws, stream=stream)

    def topk_merge(self, n_unique: int = -1, stream=None):
        hs_topk_merge(self.plan, n_unique, self.n_unique, self.topk_score, self.topk_index,
                      self.ws, stream=stream)

    def deliver(self, stream=None):
        hs_deliver(self.plan, self.topk_score, self.topk_index, self.topk_score.shape[0],
                   self.inverse, self.out_score, self.out_index, stream=stream)

    def workflow_results(self, w: int):
        """(scores, indices) of workflow w's requests: views of its rows of
        the per-request outputs."""
        first, count = hs_workflow_rows(self.plan, w)
        return (self.out_score[first:first + count], self.out_index[first:first + count])

    def run(self, keys, q_req, corpus, scale=None, stream=None, n_unique: int = -1):
        """The whole window; n_unique = -1 keeps the distinct count on the
        device (no host synchronisation).  With max_unique below the number
        of requests, the distinct count is read on the host (one
        synchronisation) and the distinct queries are scored in batches of at
        most max_unique (B_r), so that no group is left unscored."""
        if self.cap < self.R:
            nu = self.dedup(keys, stream, host_count=True)
            hs_scatter(q_req, self.R, self.q_row_bytes, self.first_index, 0, self.R,
                       self.n_unique, self.q_unique, stream=stream)
            self.score_chunked(corpus, nu, self.cap, scale, stream)
            self.deliver(stream)
            return
        self.dedup(keys, stream)
        self.gather_queries(q_req, stream)
        self.score_partial(corpus, scale, n_unique, stream)
        self.topk_merge(n_unique, stream)
        self.deliver(stream)

    # ------------------------------------------------ cross-window reuse

    def enable_cache(self, capacity: int, stream=None):
        """Allocates and empties a result store of `capacity` entries (a
        power of two) and the per-window miss buffers of run_cached."""
        import torch
        dev = self.ws.device
        self.cache_capacity = capacity
        self.cache = torch.empty(max(hs_cache_bytes(self.plan, capacity), 256), dtype=torch.uint8,
                                 device=dev)
        c1 = max(self.cap, 1)
        self.miss_pos = torch.empty(c1, dtype=torch.int32, device=dev)
        self.miss_first = torch.empty(c1, dtype=torch.int32, device=dev)
        self.n_miss = torch.zeros(1, dtype=torch.int64, device=dev)
        self.q_miss = torch.empty_like(self.q_unique)
        self.miss_score = torch.empty_like(self.topk_score)
        self.miss_index = torch.empty_like(self.topk_index)
        hs_cache_reset(self.plan, self.cache, capacity, stream=stream)

    def run_cached(self, keys, q_req, corpus, scale=None, stream=None, score_events=None):
        """The whole window with reuse of earlier windows' results: dedup ->
        store lookup (hit rows filled) -> representative rows of the misses ->
        score/top-k of the misses -> miss rows put in place -> store insert ->
        delivery.  Distinct and miss counts stay on the device.  score_events
        = (start, end) events recorded around the score step, if given."""
        if self.cap < self.R:
            raise ValueError("run_cached scores one batch per window: it needs max_unique = 0 "
                             "(or n_requests)")
        self.dedup(keys, stream)
        hs_cache_lookup(self.plan, self.cache, self.cache_capacity, self.unique_keys,
                        self.first_index, -1, self.n_unique, self.topk_score, self.topk_index,
                        self.miss_pos, self.miss_first, self.n_miss, stream=stream)
        hs_scatter(q_req, self.R, self.q_row_bytes, self.miss_first, 0, self.cap, self.n_miss,
                   self.q_miss, stream=stream)
        if score_events is not None:
            score_events[0].record(stream)
        hs_score_partial(self.plan, self.q_miss, -1, self.n_miss, corpus, scale, self.ws,
                         stream=stream)
        if score_events is not None:
            score_events[1].record(stream)
        hs_topk_merge(self.plan, -1, self.n_miss, self.miss_score, self.miss_index, self.ws,
                      stream=stream)
        row = self.k * 4
        hs_scatter(self.miss_score, self.cap, row, self.miss_pos, 0, self.cap, self.n_unique,
                   self.topk_score, stream=stream)
        hs_scatter(self.miss_index, self.cap, row, self.miss_pos, 0, self.cap, self.n_unique,
                   self.topk_index, stream=stream)
        hs_cache_insert(self.plan, self.cache, self.cache_capacity, self.unique_keys,
                        self.miss_pos, -1, self.n_unique, self.topk_score, self.topk_index,
                        stream=stream)
        self.deliver(stream)

    # ------------------------------------------------ packed 4-bit corpus

    def enable_packed(self, batch: int = 64):
        """Allocates the scores and workspace of run_packed: `batch` distinct queries are
        scored at a time, [batch x n_corpus] fp32 scores (rows padded to 128 bytes)."""
        import torch
        if batch < 1:
            raise ValueError("batch must be at least 1")
        dev = self.ws.device
        self.packed_batch = max(min(batch, self.R), 1)
        self.packed_stride = max((self.N + 31) // 32 * 32, 32)
        self.packed_scores = torch.empty((self.packed_batch, self.packed_stride),
                                         dtype=torch.float32, device=dev)
        self.packed_allow = None   # (made for the first masks per request)
        self.packed_ws = torch.empty(hs_topk_rows_bytes(self.packed_batch, self.N, self.k),
                                     dtype=torch.uint8, device=dev)

    def run_packed(self, keys, q_req, table: "RowTable", allow=None, stream=None):
        """The whole window over a corpus packed into four bits (RowTable): dedup ->
        representative rows -> scores of the distinct queries with every chunk -> chunks
        that are not allowed set to -inf -> top-k -> delivery.  `allow` (int32 words, bit
        c % 32 of word c / 32 for chunk c): [words] for the window, or [R x words] per
        request (a filter is part of what makes two requests equal: the mask of a
        group is that of its first request).  Reads the distinct count on the host (one
        synchronisation).  A request with fewer than k allowed chunks has (-inf, -1) in
        the slots left."""
        if table.c.dtype != HS_FP4_E2M1:
            raise TypeError("the table must be packed (pack_rows)")
        if (table.rows, table.dim) != (self.N, self.d):
            raise ValueError(f"a table of {table.rows} x {table.dim} for a corpus of "
                             f"{self.N} x {self.d}")
        dev = self.ws.device
        if table.device != dev:
            raise ValueError(f"table is on {table.device}, not on {dev}")
        words = (self.N + 31) // 32
        if allow is not None and words > 0:
            if tuple(allow.shape) not in ((words,), (self.R, words)):
                raise ValueError(f"allow has shape {tuple(allow.shape)}, not ({words},) or "
                                 f"({self.R}, {words})")
            _tensor(allow, "allow", dev, dtypes=(_torch.int32,))
        if not hasattr(self, "packed_scores"):
            self.enable_packed()
            # (`stream` must not overtake what still uses the memory just taken)
            _torch.cuda.current_stream(dev).synchronize()
        if allow is not None and allow.dim() == 2 and self.packed_allow is None:
            self.packed_allow = _torch.empty((self.packed_batch, max(words, 1)),
                                             dtype=_torch.int32, device=dev)
            _torch.cuda.current_stream(dev).synchronize()
        nu = self.dedup(keys, stream, host_count=True)
        hs_scatter(q_req, self.R, self.q_row_bytes, self.first_index, 0, self.R, self.n_unique,
                   self.q_unique, stream=stream)
        adj = hs_adjust()
        if allow is not None and words > 0:
            adj.allow = _ptr(allow)
            if allow.dim() == 2:
                adj.allow = _ptr(self.packed_allow)
                adj.allow_stride = words
        for b0 in range(0, nu, self.packed_batch):
            nb = min(self.packed_batch, nu - b0)
            q = self.q_unique.data_ptr() + b0 * self.q_row_bytes
            hs_score_packed(table.c, q, self.qdt, nb, self.packed_scores, HS_F32,
                            self.packed_stride, stream=stream)
            if adj.allow:
                if adj.allow_stride:
                    hs_scatter(allow, self.R, words * 4, self.first_index.data_ptr() + b0 * 4, 0,
                               nb, None, self.packed_allow, stream=stream)
                hs_adjust_scores(adj, self.packed_scores, self.packed_stride, self.packed_scores,
                                 self.packed_stride, HS_F32, nb, self.N, stream=stream)
            hs_topk_rows(self.packed_scores, HS_F32, self.packed_stride, nb, self.N, self.k,
                         self.topk_score.data_ptr() + b0 * self.k * 4,
                         self.topk_index.data_ptr() + b0 * self.k * 4, self.packed_ws,
                         stream=stream)
        self.deliver(stream)

    # ------------------------------------------------ ready-queue priorities

    def priority(self, phi, s_hat, heavy=None, alpha=1.0, gamma=1.0, delta=0.0, eps=1e-6,
                 stream=None):
        """Eq. 3 / Eq. 7 priorities of this window's fused nodes (after dedup)
        and their ready-queue order; results in self.phi_fused, self.pi,
        self.order (first n_u entries)."""
        import torch
        dev = self.ws.device
        if not hasattr(self, "order"):
            c1 = max(self.cap, 1)
            self.phi_fused = torch.empty(c1, dtype=torch.float64, device=dev)
            self.pi = torch.empty(c1, dtype=torch.float64, device=dev)
            self.order = torch.empty(c1, dtype=torch.int32, device=dev)
        hs_priority(self.plan, self.inverse, self.first_index, -1, self.n_unique, phi, s_hat,
                    heavy, alpha, gamma, delta, eps, self.phi_fused, self.pi, self.order, self.ws,
                    stream=stream)

    # ------------------------------------------------ micro-batching (Eq. 8)

    def score_chunked(self, corpus, n_unique: int, chunk: int, scale=None, stream=None,
                      events=None):
        """Scores the window's n_unique distinct queries (host count) as
        consecutive sub-batches of at most `chunk` queries, one after the
        other on `stream` (the batch limit B_r of Appendix A; small batches
        finish their queries earlier).  Results land in topk_score/index as
        for one batch.  `events`, if given, is a list that receives one
        (start, end) event pair per sub-batch."""
        import torch
        row_q = self.q_row_bytes
        for b0 in range(0, n_unique, chunk):
            nb = min(chunk, n_unique - b0)
            if events is not None:
                ev = (torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True))
                ev[0].record(stream)
            q = self.q_unique.data_ptr() + b0 * row_q
            ts = self.topk_score.data_ptr() + b0 * self.k * 4
            ti = self.topk_index.data_ptr() + b0 * self.k * 4
            hs_score_topk(self.plan, q, nb, None, corpus, scale, ts, ti, self.ws, stream=stream)
            if events is not None:
                ev[1].record(stream)
                events.append(ev)

    def score_split(self, corpus, n_unique: int, parts: int, streams, scale=None):
        """Scores the distinct queries as `parts` near-equal sub-batches, each
        on its own stream with its own workspace (the split k_v of Appendix
        A: sub-batches that may run side by side).  The caller orders the
        streams after the current producer and synchronises them."""
        import torch
        if not hasattr(self, "_split_ws") or len(self._split_ws) < parts:
            self._split_ws = [torch.empty_like(self.ws) for _ in range(parts)]
        row_q = self.q_row_bytes
        base = 0
        for j in range(parts):
            nb = n_unique // parts + (1 if j < n_unique % parts else 0)
            if nb == 0:
                continue
            q = self.q_unique.data_ptr() + base * row_q
            ts = self.topk_score.data_ptr() + base * self.k * 4
            ti = self.topk_index.data_ptr() + base * self.k * 4
            hs_score_topk(self.plan, q, nb, None, corpus, scale, ts, ti, self._split_ws[j],
                          stream=streams[j])
            base += nb



# ---------------------------------------------------------------- one call

def dedup(keys, stream=None):
    """Step 1 alone (Sec. 3.3 (I) signature matching) on a device int64
    tensor of R keys: returns (unique_keys, first_index, counts, inverse),
    the per-group tensors trimmed to the n_u groups.  Reads n_u on the host
    (one synchronisation of `stream`)."""
    import torch
    if keys.dtype != torch.int64 or keys.dim() != 1:
        raise TypeError("keys must be a 1-D int64 tensor")
    R = keys.shape[0]
    dev = keys.device
    stream = stream if stream is not None else torch.cuda.current_stream(dev)
    plan = hs_merge_plan(R, 8, 1, 1, HS_BF16, HS_BF16)
    R1 = max(R, 1)
    ws = torch.empty(max(plan.workspace_bytes, 256), dtype=torch.uint8, device=dev)
    uk = torch.empty(R1, dtype=torch.int64, device=dev)
    fi = torch.empty(R1, dtype=torch.int32, device=dev)
    ct = torch.empty(R1, dtype=torch.int32, device=dev)
    inv = torch.empty(R1, dtype=torch.int32, device=dev)
    nu_dev = torch.zeros(1, dtype=torch.int64, device=dev)
    nu = hs_dedup(plan, keys if R else None, uk, fi, ct, inv, nu_dev, True, ws, stream=stream)
    return uk[:nu], fi[:nu], ct[:nu], inv[:R]


def merge_retrieval(keys, q_req, corpus, k: int, scale=None, workflow_offsets=None,
                    max_unique: int = 0, stream=None):
    """The whole window in one call: dedup (Sec. 3.3 (I)), one batched exact
    top-k retrieval per distinct query (Appendix A batching), delivery of each
    group's result to every request (Sec. 3.3 (I)).  keys [R] int64,
    q_req [R x d] (float32 or bfloat16), corpus [N x d] (float32, bfloat16, or
    float8_e4m3fn / uint8 codes with scale [N] float32), all on one device;
    workflow_offsets: host CSR of W + 1 request offsets, or None for one
    workflow.  Returns a dict of device tensors: out_score / out_index
    [R x k] (per request), unique_keys / first_index / counts [n_u],
    inverse [R], topk_score / topk_index [n_u x k], and n_unique (an int:
    the call reads it on the host once) and `retrieval`, the MergedRetrieval
    that owns them (workflow_results(w) gives workflow w's rows)."""
    import torch
    stream = stream if stream is not None else torch.cuda.current_stream(keys.device)
    R, d = q_req.shape
    N = corpus.shape[0]
    offs = None if workflow_offsets is None else [int(x) for x in workflow_offsets]
    W = 1 if offs is None else len(offs) - 1
    m = MergedRetrieval(R, d, N, k, dtype_code(q_req), dtype_code(corpus), device=keys.device,
                        max_unique=max_unique, n_workflows=W, workflow_offsets=offs)
    m.run(keys, q_req, corpus, scale, stream=stream)
    stream.synchronize()
    nu = int(m.n_unique.item())
    return {"out_score": m.out_score[:R], "out_index": m.out_index[:R],
            "unique_keys": m.unique_keys[:nu], "first_index": m.first_index[:nu],
            "counts": m.counts[:nu], "inverse": m.inverse[:R],
            "topk_score": m.topk_score[:nu], "topk_index": m.topk_index[:nu],
            "n_unique": nu, "retrieval": m}


# ---------------------------------------------------------------- row tables
#
# As everything here these work on memory: no result has an autograd history.  A program
# that trains calls embed and embed_grad from an autograd function of its own.

class _Here:
    """The context of a call on the current device and stream."""

    def __enter__(self):
        return None

    def __exit__(self, *exc):
        return False


_HERE_CONTEXT = _Here()


def _on(stream, device):
    """(context, stream) of a one-call operator: launches and new tensors belong to
    `stream` (a torch stream; default: the current one of the tensors' device) whatever
    device and stream are current."""
    if device.type != "cuda":
        raise TypeError("tensors must be on a GPU")
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"stream on {stream.device}, tensors on {device}")
        return _torch.cuda.stream(stream), stream
    here = device.index == _torch.cuda.current_device()
    # (the handle alone: a Stream object takes 1.8 us to make, more than the checks)
    return (_HERE_CONTEXT if here else _torch.cuda.device(device),
            _torch._C._cuda_getCurrentRawStream(device.index))


_FLOAT_CODES = {} if _torch is None else {_torch.float32: HS_F32, _torch.bfloat16: HS_BF16}


def _float_code(dtype, what: str) -> int:
    code = _FLOAT_CODES.get(dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16, not {dtype}")
    return code


def _tensor(t, what: str, device, shape=None, dtypes=None):
    """Checks one contiguous device tensor (shape, dtypes: tuples)."""
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    if dtypes is not None and t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _arg(t, what: str, device, shape, dtype):
    """Address of one checked contiguous device tensor."""
    if t.dtype is dtype and t.get_device() == device.index and \
            (shape is None or t.shape == shape) and t.is_contiguous():
        return t.data_ptr()
    return _tensor(t, what, device, shape, (dtype,)).data_ptr()


def _rows_of(t, what: str):
    """(rows, columns, row stride) of a 2-D tensor whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be 2-D")
    rows, cols = t.shape
    stride, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{what} must have contiguous rows")
    if rows > 1:
        if stride < cols:
            raise ValueError(f"{what} has overlapping rows")
        return rows, cols, stride
    return rows, cols, cols


class RowTable:
    """A table of rows in device memory (hs_row_table) and the tensors behind it:
    data [rows x dim] float32 or bfloat16; float8_e4m3fn or uint8 codes with scales
    [rows] float32; or, with group = 32, 64 or 128, packed E2M1 codes [rows x dim / 2]
    uint8 with scales [rows x dim / group] float32 or bfloat16."""

    def __init__(self, data, scales=None, group: int = 0):
        import torch
        if data.dim() != 2:
            raise ValueError("data must be 2-D")
        _tensor(data, "data", data.device)
        rows, width = data.shape
        f32, bf16 = torch.float32, torch.bfloat16
        sdt = 0
        if group:
            _tensor(data, "data", data.device, dtypes=(torch.uint8,))
            dim, code = 2 * width, HS_FP4_E2M1
            if scales is None:
                raise ValueError("a packed table needs scales")
            if group not in (32, 64, 128) or dim % group:
                raise ValueError(f"group {group} does not fit {dim} columns")
            _tensor(scales, "scales", data.device, (rows, dim // group), (f32, bf16))
            sdt = _float_code(scales.dtype, "scales")
        else:
            dim, code = width, dtype_code(data)
            if code == HS_FP8_E4M3:
                if scales is None:
                    raise ValueError("an fp8 table needs scales")
                _tensor(scales, "scales", data.device, (rows,), (f32,))
            elif scales is not None:
                raise ValueError("scales belong to fp8 and packed tables")
        self.data, self.scales, self.group = data, scales, group
        self.rows, self.dim, self.device = rows, dim, data.device
        self.c = hs_row_table(_ptr(data), _ptr(scales), rows, dim, code, sdt, group)


def pack_rows(rows, group: int = 32, scale_dtype=None, stream=None) -> RowTable:
    """The packed 4-bit table of rows [n x dim] (float32 or bfloat16), dim a multiple of
    group (32, 64 or 128); scale_dtype bfloat16 (the default) or float32."""
    torch = _torch
    scale_dtype = torch.bfloat16 if scale_dtype is None else scale_dtype
    if rows.dim() != 2:
        raise ValueError("rows must be 2-D")
    _tensor(rows, "rows", rows.device)
    code, sdt = _float_code(rows.dtype, "rows"), _float_code(scale_dtype, "scale_dtype")
    if group not in (32, 64, 128) or rows.shape[1] == 0 or rows.shape[1] % group:
        raise ValueError(f"group {group} does not fit {rows.shape[1]} columns")
    n, d = rows.shape
    ctx, stream = _on(stream, rows.device)
    with ctx:
        data = torch.empty((n, d // 2), dtype=torch.uint8, device=rows.device)
        scales = torch.empty((n, d // group), dtype=scale_dtype, device=rows.device)
        hs_pack_rows(rows, code, n, d, group, sdt, data, scales, stream=stream)
    return RowTable(data, scales, group)


def _ids(ids, device):
    _tensor(ids, "ids", device, dtypes=(_torch.int32, _torch.int64))
    return int(ids.dtype == _torch.int64), ids.numel()


def embed(table: RowTable, ids, scale: float = 1.0, pad_id: int = -1, out_dtype=None, out=None,
          stream=None):
    """Embedding lookup with scaling: scale * table[ids] for ids of any shape (int32 or
    int64), as ids.shape + [dim] in out_dtype (default: the table's type, bfloat16 for
    quantised tables).  Ids outside the table and pad_id give rows of zeros.  `out`:
    a contiguous tensor for the result.  The result is not differentiable by itself;
    embed_grad is its gradient."""
    torch = _torch
    device = table.device
    is64, n = _ids(ids, device)
    shape = ids.shape + (table.dim,)
    ctx, stream = _on(stream, device)
    with ctx:
        if out is None:
            if out_dtype is None:
                out_dtype = torch.float32 if table.c.dtype == HS_F32 else torch.bfloat16
            out = torch.empty(shape, dtype=out_dtype, device=device)
        else:
            _tensor(out, "out", device, shape, None if out_dtype is None else (out_dtype,))
        hs_embed(table.c, ids, is64, n, scale, pad_id, out, _float_code(out.dtype, "out"),
                 stream=stream)
    return out


def embed_grad(d_out, ids, rows: int, scale: float = 1.0, pad_id: int = -1, out_dtype=None,
               out=None, accumulate: bool = False, ws=None, stream=None):
    """Gradient of embed with respect to its table of `rows` rows: d_out is ids.shape +
    [dim] (float32 or bfloat16), the result [rows x dim] in out_dtype (default: that of
    d_out).  accumulate adds to `out`.  `ws`: a uint8 workspace of hs_embed_grad_bytes'
    size to use instead of a new one."""
    torch = _torch
    device = d_out.device
    is64, n = _ids(ids, device)
    if d_out.dim() < 1:
        raise ValueError("d_out needs a column dimension")
    dim = d_out.shape[-1]
    _tensor(d_out, "d_out", device, ids.shape + (dim,))
    code = _float_code(d_out.dtype, "d_out")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    ctx, stream = _on(stream, device)
    with ctx:
        if out is None:
            out = torch.empty((rows, dim), dtype=out_dtype or d_out.dtype, device=device)
        if ws is None:
            ws = torch.empty(hs_embed_grad_bytes(n, rows, dim), dtype=torch.uint8, device=device)
        _tensor(out, "out", device, (rows, dim), None if out_dtype is None else (out_dtype,))
        _tensor(ws, "ws", device)
        hs_embed_grad(d_out, code, ids, is64, n, rows, dim, scale, pad_id, int(accumulate), out,
                      _float_code(out.dtype, "out"), ws, stream=stream)
    return out


def score_packed(table: RowTable, x, out_dtype=None, out=None, stream=None):
    """Products of rows x [m x dim] (float32 or bfloat16) with every row of a packed
    table, [m x table.rows] in out_dtype (default float32).  `out` may have a row
    stride above table.rows."""
    torch = _torch
    device = table.device
    if table.c.dtype != HS_FP4_E2M1:
        raise TypeError("the table must be packed (pack_rows)")
    if x.dim() != 2:
        raise ValueError("x must be 2-D")
    m = x.shape[0]
    _tensor(x, "x", device, (m, table.dim))
    code = _float_code(x.dtype, "x")
    ctx, stream = _on(stream, device)
    with ctx:
        if out is None:
            out = torch.empty((m, table.rows), dtype=out_dtype or torch.float32, device=device)
        stride = _rows_of(out, "out")[2]
        if out.device != device or out.shape != (m, table.rows) or \
                out_dtype not in (None, out.dtype):
            raise ValueError("out does not fit the table, x and out_dtype")
        hs_score_packed(table.c, x, code, m, out, _float_code(out.dtype, "out"), stride,
                        stream=stream)
    return out


def adjust_scores(scores, allow=None, seen=None, seen_off=None, prompt_len=None, repetition=None,
                  frequency=None, presence=None, bias_id=None, bias=None, bias_off=None, out=None,
                  stream=None):
    """Penalties for repeated tokens, biases and allow masks on scores [rows x cols]
    (float32 or bfloat16; hs_adjust_scores gives the formulas).  seen [any] int32 with
    seen_off [rows + 1] int64; prompt_len [rows] int32; repetition, frequency, presence
    [rows] float32; bias_id [any] int32 and bias float32 with bias_off [rows + 1] int64;
    allow: int32 words, bit c % 32 of word c / 32 for column c, [words] for all rows or
    [rows x words].  `out` may be scores; by default a new tensor."""
    torch = _torch
    device = scores.device
    rows, cols, stride = _rows_of(scores, "scores")
    code = _float_code(scores.dtype, "scores")
    if (seen is None) != (seen_off is None):
        raise ValueError("seen and seen_off belong together")
    if not (bias_id is None) == (bias is None) == (bias_off is None):
        raise ValueError("bias_id, bias and bias_off belong together")
    f32, i32, i64 = torch.float32, torch.int32, torch.int64
    per_row, offsets = (rows,), (rows + 1,)
    a = hs_adjust()
    if seen is not None:
        a.seen = _arg(seen, "seen", device, None, i32)
        a.seen_off = _arg(seen_off, "seen_off", device, offsets, i64)
        a.n_seen = seen.numel()
    if bias_id is not None:
        a.bias_id = _arg(bias_id, "bias_id", device, None, i32)
        a.bias = _arg(bias, "bias", device, bias_id.shape, f32)
        a.bias_off = _arg(bias_off, "bias_off", device, offsets, i64)
        a.n_bias = bias_id.numel()
    if prompt_len is not None:
        a.prompt_len = _arg(prompt_len, "prompt_len", device, per_row, i32)
    if repetition is not None:
        a.repetition = _arg(repetition, "repetition", device, per_row, f32)
    if frequency is not None:
        a.frequency = _arg(frequency, "frequency", device, per_row, f32)
    if presence is not None:
        a.presence = _arg(presence, "presence", device, per_row, f32)
    if allow is not None:
        words = (cols + 31) // 32
        if allow.dim() == 1:
            a.allow = _arg(allow, "allow", device, (words,), i32)
        else:
            a.allow = _arg(allow, "allow", device, (rows, words), i32)
            a.allow_stride = words
    ctx, stream = _on(stream, device)
    with ctx:
        if out is None:
            out = torch.empty((rows, cols), dtype=scores.dtype, device=device)
            out_stride = cols
        else:
            *shape, out_stride = _rows_of(out, "out")
            if out.device != device or shape != [rows, cols] or out.dtype != scores.dtype:
                raise ValueError("out does not fit scores")
        hs_adjust_scores(a, scores, stride, out, out_stride, code, rows, cols, stream=stream)
    return out


def topk_rows(scores, k: int, out=None, ws=None, stream=None):
    """The k best columns of every row of scores [rows x cols] (float32 or bfloat16):
    (score [rows x k] float32, column [rows x k] int32), score descending, equal scores by
    ascending column; entries of -inf and NaN are never taken, slots left are (-inf, -1).
    `out`: the two tensors for the result, `ws`: a uint8 workspace of
    hs_topk_rows_bytes' size."""
    torch = _torch
    device = scores.device
    rows, cols, stride = _rows_of(scores, "scores")
    code = _float_code(scores.dtype, "scores")
    need = hs_topk_rows_bytes(rows, cols, k) if ws is None else 0
    ctx, stream = _on(stream, device)
    with ctx:
        if out is None:
            out = (torch.empty((rows, k), dtype=torch.float32, device=device),
                   torch.empty((rows, k), dtype=torch.int32, device=device))
        if ws is None:
            ws = torch.empty(need, dtype=torch.uint8, device=device)
        score = _arg(out[0], "out[0]", device, (rows, k), torch.float32)
        index = _arg(out[1], "out[1]", device, (rows, k), torch.int32)
        _tensor(ws, "ws", device)
        hs_topk_rows(scores, code, stride, rows, cols, k, score, index, ws, stream=stream)
    return out
