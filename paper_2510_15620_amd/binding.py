"""ctypes binding of libprism.so: argument marshalling only - every step of the path runs in the
library's HIP kernels.  Function names follow include/prism.h.  PyTorch tensors are used as
device-memory handles (data_ptr) and for the caller's stream."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass, field
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprism.so")

OK, EINVAL, ECAP, EHIP, ENOMEM, EUNSUPPORTED = 0, -1, -2, -3, -4, -5
WFMT_PLAIN, WFMT_W4G128 = 0, 1
DTYPE_FP32, DTYPE_BF16, DTYPE_F16 = 0, 1, 2
MODE_DROP_ONLY, MODE_THREE_WAY, MODE_NO_PRUNING = 0, 1, 2
EPI_STORE, EPI_RESIDUAL, EPI_SWIGLU, EPI_STORE_F32 = 0, 1, 2, 3
FATE_NOT_LIVE, FATE_DROPPED, FATE_DEFERRED, FATE_SELECTED = -1, 0, 1, 2
KIND_TRANSFERS = 8          # bit of prism_report.kind_mask that asks for ms_transfers (PRISM_KIND_MASK_TRANSFERS)
MAX_CANDS, MAX_CLUSTERS, MAX_SEQ = 4096, 8, 8192

EXPORTS = ["prism_create", "prism_select", "prism_set_forced_keep", "prism_destroy", "prism_strerror",
           "prism_last_error", "prism_op_embed", "prism_op_rmsnorm", "prism_op_gemm", "prism_op_qkv_finish", "prism_op_qkv_project", "prism_w4_bytes", "prism_op_quantize_w4", "prism_op_dequantize_w4",
           "prism_op_attention", "prism_op_score", "prism_op_route", "prism_op_route_static", "prism_op_compact", "prism_op_topk", "prism_vt_column_of_key",
           "prism_page_plan_bytes", "prism_op_page_plan", "prism_op_qkv_finish_paged", "prism_attention_paged_workspace",
           "prism_op_attention_paged",
           "prism_op_quantize_q8", "prism_op_dequantize_q8", "prism_op_rmsnorm_q8", "prism_op_gemm_q8"]


class PrismError(RuntimeError):
    def __init__(self, code: int, detail: str):
        super().__init__(f"prism error {code}: {detail}")
        self.code = code


class prism_model(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] + \
               [("rms_eps", C.c_float), ("rope_base", C.c_float), ("dtype", C.c_int32), ("qk_norm", C.c_int32)]


LAYER_FIELDS = ("attn_norm", "wq", "wk", "wv", "q_norm", "k_norm", "wo", "ffn_norm", "w_gate", "w_up", "w_down")


class prism_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYER_FIELDS]


class prism_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("layers", C.POINTER(prism_layer_weights)), ("final_norm", C.c_void_p),
                ("w_yes", C.c_void_p), ("w_no", C.c_void_p), ("layer_residency", C.c_int32), ("embed_residency", C.c_int32), ("layer_format", C.c_int32)]


class prism_options(C.Structure):
    _fields_ = [("checkpoint_layers", C.POINTER(C.c_int32)), ("n_checkpoints", C.c_int32), ("cv_threshold", C.c_float),
                ("n_clusters", C.c_int32), ("mode", C.c_int32), ("chunk_cands", C.c_int32), ("hbm_cap_bytes", C.c_int64),
                ("stream", C.c_void_p), ("operand", C.c_int32), ("offload_hidden", C.c_int32), ("embed_cache_rows", C.c_int32), ("stream_slots", C.c_int32),
                ("no_query_sharing", C.c_int32), ("single_pass_checks", C.c_int32)]


class prism_kv_cache(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("page_stride", C.c_int64)] + \
               [(n, C.c_int32) for n in ("dtype", "n_kv_heads", "head_dim", "page_size", "n_pages")]


class prism_page_shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_tokens", "n_q_heads", "n_kv_heads", "page_size", "n_pages", "max_pages", "window")]


class prism_q8(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("stride", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32)]


class prism_report(C.Structure):
    _fields_ = [("cap_events", C.c_int32), ("n_cands", C.c_int32), ("n_events", C.c_int32),
                ("ev_layer", C.POINTER(C.c_int32)), ("ev_n_before", C.POINTER(C.c_int32)),
                ("ev_n_after", C.POINTER(C.c_int32)), ("ev_tokens_after", C.POINTER(C.c_int32)),
                ("ev_gate", C.POINTER(C.c_int32)), ("ev_n_clusters", C.POINTER(C.c_int32)),
                ("ev_mean", C.POINTER(C.c_double)), ("ev_std", C.POINTER(C.c_double)),
                ("ev_scores", C.POINTER(C.c_float)), ("ev_fate", C.POINTER(C.c_int8)),
                ("ms_total", C.c_double), ("ms_layers", C.c_double), ("ms_checks", C.c_double),
                ("token_layers", C.c_int64), ("peak_hbm_bytes", C.c_int64), ("bytes_streamed", C.c_int64),
                ("layers_run", C.c_int32), ("kind_launches", C.c_int32 * 6), ("kind_ms", C.c_double * 6),
                ("kind_flops", C.c_double * 6), ("bytes_hidden_moved", C.c_int64), ("embed_rows_hit", C.c_int64),
                ("embed_rows_missed", C.c_int64), ("span_cap", C.c_int32), ("n_spans", C.c_int32),
                ("span_kind", C.POINTER(C.c_int32)), ("span_rows", C.POINTER(C.c_int32)), ("span_ms", C.POINTER(C.c_float)),
                ("span_flops", C.POINTER(C.c_double)), ("kind_mask", C.c_int32), ("ms_transfers", C.c_double)]


_lib = None


def lib() -> C.CDLL:
    """The HIP library.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise PrismError(EHIP, f"{LIB_PATH} is not built; run `python -m paper_2510_15620_amd.build`")
        # PyTorch ships its own copy of the HIP runtime.  Streams and device pointers cross between it and this library,
        # so both must use ONE runtime instance: load PyTorch's first and let the library bind to it.  (Loaded the other
        # way round, the second copy finds no device.)
        import torch  # noqa: F401
        _lib = C.CDLL(LIB_PATH)
        _lib.prism_strerror.restype = C.c_char_p
        _lib.prism_last_error.restype = C.c_char_p
        _lib.prism_destroy.restype = None
        vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
        _lib.prism_create.argtypes = [C.POINTER(prism_model), C.POINTER(prism_weights), C.POINTER(prism_options), C.POINTER(vp)]
        _lib.prism_select.argtypes = [vp, C.POINTER(i32), i32, C.POINTER(C.POINTER(i32)), C.POINTER(i32), i32, i32,
                                      C.POINTER(i32), C.POINTER(f32), C.POINTER(i32), C.POINTER(prism_report)]
        _lib.prism_set_forced_keep.argtypes = [vp, C.POINTER(C.c_int8), i32, i32]
        _lib.prism_destroy.argtypes = [vp]
        _lib.prism_strerror.argtypes = [i32]
        _lib.prism_op_embed.argtypes = [vp, i32, vp, i32, i32, vp, vp]
        _lib.prism_op_rmsnorm.argtypes = [vp, vp, i32, i32, f32, i32, vp, vp]
        _lib.prism_op_gemm.argtypes = [i32, i32, vp, vp, vp, i32, i32, i32, vp]
        _lib.prism_op_qkv_finish.argtypes = [i32, vp, vp, i32, vp, vp, i32, i32, i32, i32, f32, f32, i32, vp, vp, vp, C.c_int64, vp]
        _lib.prism_op_qkv_project.argtypes = [i32, vp, vp, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32, f32, i32, vp, vp, vp,
                                              C.c_int64, vp]
        _lib.prism_op_attention.argtypes = [i32, vp, vp, C.c_int64, C.POINTER(i32), C.POINTER(i32), i32, i32, i32, i32, vp, vp]
        _lib.prism_op_score.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, f32, vp, vp]
        _lib.prism_op_route.argtypes = [vp, i32, i32, i32, f32, vp, vp, vp]
        _lib.prism_op_route_static.argtypes = [vp, i32, i32, i32, f32, vp, vp, vp]
        _lib.prism_op_compact.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
        _lib.prism_op_topk.argtypes = [vp, i32, i32, vp, vp, vp]
        _lib.prism_w4_bytes.restype = C.c_int64
        _lib.prism_w4_bytes.argtypes = [i32, i32]
        _lib.prism_op_quantize_w4.argtypes = [vp, i32, i32, vp, vp]
        _lib.prism_op_dequantize_w4.argtypes = [vp, i32, i32, i32, vp, vp]
        i64, shape, cache = C.c_int64, C.POINTER(prism_page_shape), C.POINTER(prism_kv_cache)
        _lib.prism_page_plan_bytes.restype = i64
        _lib.prism_page_plan_bytes.argtypes = [shape]
        _lib.prism_op_page_plan.argtypes = [shape, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib.prism_op_qkv_finish_paged.argtypes = [cache, i32, vp, i64, i32, vp, vp, i32, vp, vp, f32, f32, i32, vp, i64, vp]
        _lib.prism_attention_paged_workspace.restype = i64
        _lib.prism_attention_paged_workspace.argtypes = [shape, i32]
        _lib.prism_op_attention_paged.argtypes = [shape, cache, vp, vp, vp, i64, f32, f32, vp, vp, i64, vp, i64, vp]
        q8 = C.POINTER(prism_q8)
        _lib.prism_op_quantize_q8.argtypes = [i32, vp, i64, q8, vp]
        _lib.prism_op_dequantize_q8.argtypes = [q8, i32, vp, i64, vp]
        _lib.prism_op_rmsnorm_q8.argtypes = [vp, i64, i32, vp, i64, i32, vp, f32, q8, vp]
        _lib.prism_op_gemm_q8.argtypes = [i32, q8, q8, i32, vp, i64, vp]
    return _lib


def _check(rc: int):
    if rc != OK:
        l = lib()
        raise PrismError(rc, f"{l.prism_strerror(rc).decode()}: {l.prism_last_error().decode()}")


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


def _i32_array(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


@dataclass
class Report:
    layer: np.ndarray
    n_before: np.ndarray
    n_after: np.ndarray
    tokens_after: np.ndarray
    gate: np.ndarray
    n_clusters: np.ndarray
    mean: np.ndarray
    std: np.ndarray
    scores: np.ndarray          # [n_events, n_cands], NaN where not live
    fate: np.ndarray            # [n_events, n_cands]
    ms_total: float
    ms_layers: float
    ms_checks: float
    token_layers: int
    peak_hbm_bytes: int
    bytes_streamed: int
    layers_run: int
    kind_launches: List[int] = field(default_factory=list)   # QKV, O, gate/up, down GEMMs, attention, elementwise
    kind_ms: List[float] = field(default_factory=list)
    kind_flops: List[float] = field(default_factory=list)
    bytes_hidden_moved: int = 0
    embed_rows_hit: int = 0
    embed_rows_missed: int = 0
    ms_transfers: float = 0.0   # side-stream time spent copying streamed layer weights
    spans: Optional[np.ndarray] = None   # per launch, in order: structured array (kind, rows, ms, flops); None unless asked for


class Prism:
    """prism_create / prism_select / prism_set_forced_keep / prism_destroy."""

    def __init__(self, model, weights, *, checkpoints: Sequence[int] = (), cv_threshold: float = 0.0, n_clusters: int = 3,
                 mode: int = MODE_DROP_ONLY, chunk_cands: int = 0, hbm_cap_bytes: int = 0, stream_weights: bool = False,
                 stream: Optional[int] = None, operand: str = "f16", offload_hidden: bool = False, embed_on_host: bool = False,
                 embed_cache_rows: int = 0, w4: bool = False, stream_slots: int = 0, share_query: bool = True,
                 two_pass_checks: bool = True):
        """model: object with n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab, rms_eps, rope_base,
        qk_norm, dtype ("fp32" | "bf16": storage type of the weights).  operand ("f16" | "bf16"): 16-bit type of the
        matrix-core operands when the weights are bf16.  weights: object with embed, final_norm, w_yes, w_no (device tensors) and
        layers: list of dicts of tensors (device, or pinned host when stream_weights).  embed_on_host: weights.embed is a
        pinned host tensor (w_yes / w_no stay device tensors) read through a device LRU cache of embed_cache_rows rows.
        offload_hidden: the residual stream lives in pinned host memory, three chunks at a time on the device.
        w4: the seven matrices of every layer dict are uint8 blobs from quantize_w4 (gains stay bf16).
        share_query=False: every sequence carries its own copy of the query (prism_options.no_query_sharing).
        two_pass_checks=False: a checked layer runs completely before its check (prism_options.single_pass_checks)."""
        self._ctx = C.c_void_p()
        m = prism_model(model.n_layers, model.hidden, model.n_q_heads, model.n_kv_heads, model.head_dim, model.ffn,
                        model.vocab, model.rms_eps, model.rope_base, DTYPE_FP32 if model.dtype == "fp32" else DTYPE_BF16,
                        int(model.qk_norm))
        layers = (prism_layer_weights * model.n_layers)()
        for l, lw in enumerate(weights.layers):
            for n in LAYER_FIELDS:
                setattr(layers[l], n, _ptr(lw[n]))
        self._keep = (weights, layers)      # borrowed by the library for the context's lifetime
        w = prism_weights(_ptr(weights.embed), layers, _ptr(weights.final_norm), _ptr(weights.w_yes), _ptr(weights.w_no),
                          1 if stream_weights else 0, 1 if embed_on_host else 0, WFMT_W4G128 if w4 else WFMT_PLAIN)
        ck, ckp = _i32_array(list(checkpoints))
        o = prism_options(ckp, len(ck), cv_threshold, n_clusters, mode, chunk_cands, hbm_cap_bytes,
                          _stream() if stream is None else stream, DTYPE_BF16 if operand == "bf16" else DTYPE_F16,
                          int(offload_hidden), embed_cache_rows, stream_slots, 0 if share_query else 1,
                          0 if two_pass_checks else 1)
        self.n_checkpoints = len(ck)
        _check(lib().prism_create(C.byref(m), C.byref(w), C.byref(o), C.byref(self._ctx)))

    def select(self, query_tokens, cand_tokens: Sequence, K: int, report: bool = True, spans: int = 0, kinds=None):
        """spans: capacity of the per-launch detail of the report (0 = none).  kinds: the kernel kinds that get event spans
        (iterable of kind numbers; None = all); KIND_TRANSFERS in it additionally times the streamed layers' copies."""
        q, qp = _i32_array(query_tokens)
        cands = [np.ascontiguousarray(c, dtype=np.int32) for c in cand_tokens]
        n = len(cands)
        cptrs = (C.POINTER(C.c_int32) * max(n, 1))(*[c.ctypes.data_as(C.POINTER(C.c_int32)) for c in cands])
        lens, lp = _i32_array([len(c) for c in cands])
        kk = max(K, 1)
        out_idx = np.full(kk, -1, np.int32)
        out_scores = np.full(kk, np.nan, np.float32)
        count = C.c_int32(0)
        rep = None
        if report:
            cap = self.n_checkpoints + 1
            arrs = {k: np.zeros(cap, np.int32) for k in ("layer", "n_before", "n_after", "tokens_after", "gate", "n_clusters")}
            arrs["mean"], arrs["std"] = np.zeros(cap, np.float64), np.zeros(cap, np.float64)
            arrs["scores"] = np.zeros((cap, max(n, 1)), np.float32)
            arrs["fate"] = np.zeros((cap, max(n, 1)), np.int8)
            P = lambda a, t: a.ctypes.data_as(C.POINTER(t))
            rep = prism_report(cap, max(n, 1), 0, P(arrs["layer"], C.c_int32), P(arrs["n_before"], C.c_int32),
                               P(arrs["n_after"], C.c_int32), P(arrs["tokens_after"], C.c_int32), P(arrs["gate"], C.c_int32),
                               P(arrs["n_clusters"], C.c_int32), P(arrs["mean"], C.c_double), P(arrs["std"], C.c_double),
                               P(arrs["scores"], C.c_float), P(arrs["fate"], C.c_int8))
            if spans > 0:
                sp = {"kind": np.zeros(spans, np.int32), "rows": np.zeros(spans, np.int32), "ms": np.zeros(spans, np.float32),
                      "flops": np.zeros(spans, np.float64)}
                rep.span_cap = spans
                rep.span_kind, rep.span_rows = P(sp["kind"], C.c_int32), P(sp["rows"], C.c_int32)
                rep.span_ms, rep.span_flops = P(sp["ms"], C.c_float), P(sp["flops"], C.c_double)
            if kinds is not None:
                rep.kind_mask = sum(1 << int(k) for k in kinds)
        _check(lib().prism_select(self._ctx, qp, len(q), cptrs, lp, n, K, out_idx.ctypes.data_as(C.POINTER(C.c_int32)),
                                  out_scores.ctypes.data_as(C.POINTER(C.c_float)), C.byref(count),
                                  C.byref(rep) if rep is not None else None))
        k = count.value
        r = None
        if rep is not None:
            e = rep.n_events
            r = Report(arrs["layer"][:e], arrs["n_before"][:e], arrs["n_after"][:e], arrs["tokens_after"][:e],
                       arrs["gate"][:e].astype(bool), arrs["n_clusters"][:e], arrs["mean"][:e], arrs["std"][:e],
                       arrs["scores"][:e], arrs["fate"][:e], rep.ms_total, rep.ms_layers, rep.ms_checks,
                       rep.token_layers, rep.peak_hbm_bytes, rep.bytes_streamed, rep.layers_run,
                       list(rep.kind_launches), list(rep.kind_ms), list(rep.kind_flops), rep.bytes_hidden_moved,
                       rep.embed_rows_hit, rep.embed_rows_missed, rep.ms_transfers)
            if spans > 0:
                n = rep.n_spans
                r.spans = np.rec.fromarrays([sp["kind"][:n], sp["rows"][:n], sp["ms"][:n], sp["flops"][:n]],
                                            names="kind,rows,ms,flops")
        return out_idx[:k].copy(), out_scores[:k].copy(), r

    def set_forced_keep(self, masks: Optional[np.ndarray]):
        if masks is None:
            _check(lib().prism_set_forced_keep(self._ctx, None, 0, 0))
            return
        m = np.ascontiguousarray(masks, dtype=np.int8)
        _check(lib().prism_set_forced_keep(self._ctx, m.ctypes.data_as(C.POINTER(C.c_int8)), m.shape[0], m.shape[1]))

    def destroy(self):
        if self._ctx:
            lib().prism_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---- kernel-level entry points (device tensors in, device tensors out) ---------------------------------------------

def _dt(t) -> int:
    import torch
    return {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}[t.dtype]


def op_embed(tokens, table, X):
    _check(lib().prism_op_embed(_ptr(tokens), tokens.numel(), _ptr(table), table.shape[1], _dt(table), _ptr(X), _stream()))


def op_rmsnorm(X, gain, eps, out):
    _check(lib().prism_op_rmsnorm(_ptr(X), _ptr(gain), X.shape[0], X.shape[1], eps, _dt(gain), _ptr(out), _stream()))


def op_gemm(epilogue, A, W, out):
    _check(lib().prism_op_gemm(_dt(A), epilogue, _ptr(A), _ptr(W), _ptr(out), A.shape[0], W.shape[0], A.shape[1], _stream()))


def op_qkv_finish(dtype, QKV, pos, max_pos, q_gain, k_gain, nq, nkv, hd, eps, base, qk_norm, QK=None, Vt=None,
                  vt_col=None, vt_stride=0):
    _check(lib().prism_op_qkv_finish(dtype, _ptr(QKV), _ptr(pos), max_pos, _ptr(q_gain), _ptr(k_gain), QKV.shape[0],
                                     nq, nkv, hd, eps, base, int(qk_norm), _ptr(QK), _ptr(Vt), _ptr(vt_col), vt_stride,
                                     _stream()))


def op_qkv_project(Xn, Wqkv, pos, max_pos, q_gain, k_gain, nq, nkv, hd, eps, base, qk_norm, QK, Vt, vt_col, vt_stride):
    _check(lib().prism_op_qkv_project(_dt(Xn), _ptr(Xn), _ptr(Wqkv), _ptr(pos), max_pos, _ptr(q_gain), _ptr(k_gain),
                                      Xn.shape[0], Xn.shape[1], nq, nkv, hd, eps, base, int(qk_norm), _ptr(QK), _ptr(Vt),
                                      _ptr(vt_col), vt_stride, _stream()))


def w4_bytes(N: int, K: int) -> int:
    return int(lib().prism_w4_bytes(N, K))


def quantize_w4(W):
    """W [N, K] bf16 device tensor -> uint8 device tensor holding the 4-bit blob (codes, then bf16 scales)."""
    import torch
    N, K = W.shape
    blob = torch.empty(w4_bytes(N, K), dtype=torch.uint8, device=W.device)
    _check(lib().prism_op_quantize_w4(_ptr(W), N, K, _ptr(blob), _stream()))
    return blob


def dequantize_w4(blob, N: int, K: int, out):
    _check(lib().prism_op_dequantize_w4(_ptr(blob), N, K, _dt(out), _ptr(out), _stream()))


MATRICES = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


def quantize_layers_w4(layers):
    """Layer dicts with the seven matrices replaced by their 4-bit blobs (device tensors in, device tensors out)."""
    return [{k: (quantize_w4(v) if k in MATRICES else v) for k, v in l.items()} for l in layers]


def vt_column_of_key(p):
    """Column, relative to its sequence's first, of the key at position p in the transposed V buffer: the library's
    prism_vt_column_of_key applied to an int or elementwise to an integer array (its 16 values per group, tiled)."""
    perm = np.array([lib().prism_vt_column_of_key(i) for i in range(16)], dtype=np.int64)
    p = np.asarray(p)
    out = (p & ~15) | perm[p & 15]
    return int(out) if out.ndim == 0 else out.astype(p.dtype)


def op_attention(dtype, QK, Vt, vt_stride, cu_seqlens, vt_col0, nq, nkv, hd, out):
    cu, cup = _i32_array(cu_seqlens)
    c0, c0p = _i32_array(vt_col0 if vt_col0 is not None else np.zeros(len(cu) - 1))
    _check(lib().prism_op_attention(dtype, _ptr(QK), _ptr(Vt), vt_stride, cup, c0p, len(cu) - 1, nq, nkv, hd, _ptr(out),
                                    _stream()))


def op_score(X, last_row, final_norm, w_yes, w_no, eps, scores):
    _check(lib().prism_op_score(_ptr(X), _ptr(last_row), last_row.numel(), X.shape[1], _ptr(final_norm), _ptr(w_yes),
                                _ptr(w_no), _dt(final_norm), eps, _ptr(scores), _stream()))


def op_route(scores, K_rem, n_clusters, tau, fate, stats):
    _check(lib().prism_op_route(_ptr(scores), scores.numel(), K_rem, n_clusters, tau, _ptr(fate), _ptr(stats), _stream()))


def op_route_static(scores, K_rem, n_clusters, tau, fate, stats):
    """prism_op_route on the library's static workspace: allocates nothing and does not synchronise."""
    _check(lib().prism_op_route_static(_ptr(scores), scores.numel(), K_rem, n_clusters, tau, _ptr(fate), _ptr(stats), _stream()))


def op_compact(X_src, X_dst, src_start, dst_start, length):
    _check(lib().prism_op_compact(_ptr(X_src), _ptr(X_dst), _ptr(src_start), _ptr(dst_start), _ptr(length),
                                  length.numel(), X_src.shape[1], _stream()))


def op_topk(scores, K, out_pos, out_scores):
    _check(lib().prism_op_topk(_ptr(scores), scores.numel(), K, _ptr(out_pos), _ptr(out_scores), _stream()))


# ---- paged K/V cache ----------------------------------------------------------------------------------------------------

def _need(ok: bool, what: str):
    if not ok:
        raise PrismError(EINVAL, what)


def _ints(t, n: int, device: int, what: str) -> int:
    """Address of a dense int32 device tensor of at least n values."""
    if t.dtype is _torch.int32 and t.numel() >= n and t.is_contiguous() and t.get_device() == device:
        return t.data_ptr()
    raise PrismError(EINVAL, f"{what}: a dense int32 tensor of {n} values on the current device")


def _table(t, plan, device: int) -> int:
    """Address of a page table: rows of plan.max_pages entries, or a flat tensor of them."""
    if t.dim() > 1 and t.shape[-1] != plan.max_pages:
        raise PrismError(EINVAL, f"table: rows of {t.shape[-1]} pages for a plan of {plan.max_pages}")
    return _ints(t, plan.n_seqs * plan.max_pages, device, "table")


def _rows(t, dtype, device: int, what: str):
    """Address, row stride, rows and width of a two-dimensional device tensor whose rows are dense."""
    if t.dim() == 2 and t.dtype is dtype and t.get_device() == device:
        n, width = t.shape
        stride, one = t.stride()
        if one == 1 or width < 2:
            return t.data_ptr(), stride if n > 1 else width, n, width
    raise PrismError(EINVAL, f"{what}: rows of {dtype}, dense, on the current device")


def _gain(t, hd: int, dtype, device: int) -> int:
    if t is not None and t.dtype is dtype and t.numel() == hd and t.is_contiguous() and t.get_device() == device:
        return t.data_ptr()
    raise PrismError(EINVAL, f"a gain of {hd} values of {dtype} on the current device")


_torch = None               # set with the first cache or plan: the calls below have both at hand and are short


def _here():
    """Current device and its current stream's handle (without making a Stream object)."""
    d = _torch.cuda.current_device()
    return d, _torch._C._cuda_getCurrentRawStream(d)


class KVCache:
    """A pool of pages: K and V [n_pages, n_kv_heads, page_size, head_dim] device tensors of one dtype.  Pages are dense; the stride
    from page to page is free, and the same for both (K and V may be views into one allocation)."""

    def __init__(self, K, V):
        global _torch
        import torch
        _torch = torch
        _need(K.dim() == 4 and K.shape == V.shape and K.dtype is V.dtype and K.is_cuda and K.device == V.device, "KVCache: K and V alike")
        n, heads, size, hd = K.shape
        _need(K.dtype in (torch.float32, torch.bfloat16, torch.float16), "KVCache: fp32, bf16 or half")
        for t in (K, V):
            _need(all(t.shape[i] < 2 or t.stride(i) == s for i, s in ((1, size * hd), (2, hd), (3, 1))), "KVCache: pages have to be dense")
        stride = K.stride(0) if n > 1 else heads * size * hd
        _need(n < 2 or V.stride(0) == stride, "KVCache: K and V have the same stride between pages")
        self.K, self.V, self.dtype, self.device = K, V, K.dtype, K.get_device()
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = n, heads, size, hd
        self._c = prism_kv_cache(K.data_ptr(), V.data_ptr(), stride, _dt(K), heads, hd, size, n)
        self._ref = C.byref(self._c)


class PagePlan:
    """The shape of a step (see prism_page_shape) and the device buffer of its plan.  Filled by op_page_plan, read by
    op_attention_paged; may be filled again for another step of the same shape.  The buffer is made, and cleared, on the current
    stream: as with any tensor, another stream waits for that one before it uses the plan."""

    def __init__(self, n_seqs: int, n_tokens: int, n_q_heads: int, n_kv_heads: int, page_size: int, n_pages: int, max_pages: int,
                 window: int = 0):
        global _torch
        import torch
        _torch = torch
        self._c = prism_page_shape(n_seqs, n_tokens, n_q_heads, n_kv_heads, page_size, n_pages, max_pages, window)
        self._ref = C.byref(self._c)
        size = int(lib().prism_page_plan_bytes(self._ref))
        if size < 0:
            raise PrismError(EINVAL, lib().prism_last_error().decode())
        self.n_seqs, self.n_tokens, self.n_q_heads, self.max_pages = n_seqs, n_tokens, n_q_heads, max_pages
        self.buffer = torch.zeros(size, dtype=torch.uint8, device="cuda")
        self.device = self.buffer.get_device()


def op_page_plan(plan: PagePlan, cached, fresh, table, free_pages, n_free, n_free_left, cu, pos, slot, status=None):
    """cached, fresh [n_seqs]; table [n_seqs, max_pages]; free_pages [any]; n_free, n_free_left [1]; cu [n_seqs + 1]; pos, slot
    [n_tokens]; status [4] or None: int32 device tensors."""
    d, stream = _here()
    n, T = plan.n_seqs, plan.n_tokens
    if plan.device != d:
        raise PrismError(EINVAL, "op_page_plan: the plan is on another device than the current one")
    _check(lib().prism_op_page_plan(
        plan._ref, _ints(cached, n, d, "cached"), _ints(fresh, n, d, "fresh"), _table(table, plan, d),
        _ints(free_pages, 0, d, "free_pages"), free_pages.numel(), _ints(n_free, 1, d, "n_free"), _ints(n_free_left, 1, d, "n_free_left"),
        _ints(cu, n + 1, d, "cu"), _ints(pos, T, d, "pos"), _ints(slot, T, d, "slot"),
        0 if status is None else _ints(status, 4, d, "status"), plan.buffer.data_ptr(), stream))


def op_qkv_finish_paged(QKV, pos, slot, cache: KVCache, q_gain, k_gain, eps, base, qk_norm, Q):
    """QKV [T, (nq + 2 nkv) * hd] fp32 or in the cache's dtype -> Q [T, nq * hd] and the cache's slots."""
    d, stream = _here()
    hd, nkv, dtype = cache.head_dim, cache.n_kv_heads, cache.dtype
    if cache.device != d:
        raise PrismError(EINVAL, "op_qkv_finish_paged: the cache is on another device than the current one")
    wide = QKV.dtype is _torch.float32
    x, x_stride, T, x_width = _rows(QKV, _torch.float32 if wide else dtype, d, "QKV")
    q, q_stride, q_rows, q_width = _rows(Q, dtype, d, "Q")
    if q_rows != T or q_width % hd or x_width != q_width + 2 * nkv * hd:
        raise PrismError(EINVAL, f"op_qkv_finish_paged: QKV [{T}, {x_width}], Q [{q_rows}, {q_width}], {nkv} KV heads of {hd}")
    _check(lib().prism_op_qkv_finish_paged(
        cache._ref, DTYPE_FP32 if wide else cache._c.dtype, x, x_stride, T, _ints(pos, T, d, "pos"), _ints(slot, T, d, "slot"), q_width // hd,
        _gain(q_gain, hd, dtype, d) if qk_norm else 0, _gain(k_gain, hd, dtype, d) if qk_norm else 0, eps, base, 1 if qk_norm else 0, q, q_stride, stream))


def attention_paged_workspace(plan: PagePlan, cache: KVCache):
    """A workspace for op_attention_paged: calls that may overlap need one each."""
    import torch
    size = int(lib().prism_attention_paged_workspace(plan._ref, cache.head_dim))
    if size < 0:
        raise PrismError(EINVAL, lib().prism_last_error().decode())
    return torch.empty(size, dtype=torch.uint8, device="cuda")


def op_attention_paged(plan: PagePlan, Q, cache: KVCache, table, out, workspace, scale: float = 0.0, softcap: float = 0.0, slopes=None):
    """Q, out [n_tokens, n_q_heads * hd] in the cache's dtype; table as op_page_plan left it; slopes [n_q_heads] fp32 or None."""
    d, stream = _here()
    if plan.device != d or cache.device != d or workspace.get_device() != d or not workspace.is_contiguous():
        raise PrismError(EINVAL, "op_attention_paged: a plan, a cache and a dense workspace on the current device")
    q, q_stride, T, width = _rows(Q, cache.dtype, d, "Q")
    o, o_stride, o_rows, o_width = _rows(out, cache.dtype, d, "out")
    if T != plan.n_tokens or o_rows != T or width != plan.n_q_heads * cache.head_dim or o_width != width:
        raise PrismError(EINVAL, f"op_attention_paged: Q [{T}, {width}], out [{o_rows}, {o_width}] for {plan.n_tokens} rows of {plan.n_q_heads} heads")
    if slopes is not None and (slopes.dtype is not _torch.float32 or slopes.numel() != plan.n_q_heads or not slopes.is_contiguous() or slopes.get_device() != d):
        raise PrismError(EINVAL, "op_attention_paged: slopes of n_q_heads fp32 values")
    _check(lib().prism_op_attention_paged(
        plan._ref, cache._ref, plan.buffer.data_ptr(), _table(table, plan, d), q, q_stride, scale, softcap,
        0 if slopes is None else slopes.data_ptr(), o, o_stride, workspace.data_ptr(), workspace.nbytes, stream))


# ---- 8-bit rows ---------------------------------------------------------------------------------------------------------

# Set with the first rows, by which every call gets here: a step of a few tokens waits for the host, so these calls look nothing up twice.
# torch dtype -> PRISM_DTYPE_*; the current stream of a device; the current device, where there are several
_DTYPES = {}
_raw_stream = None


def _only_device():
    return 0


_device = _only_device


class Q8:
    """Rows of 8-bit codes with a scale each (see prism_q8), on the current device: made by op_rmsnorm_q8 and op_quantize_q8, read by
    op_gemm_q8 and op_dequantize_q8.  codes [rows, stride] int8, stride being cols rounded up to 128; scales [rows] fp32.  Uninitialised.
    Keep weights in one for as long as they are used, and activations in one for each place that may be in use at the same time."""

    def __init__(self, rows: int, cols: int):
        import torch
        _need(rows >= 0 and cols > 0, f"Q8: {rows} rows of {cols} codes")
        self._set(torch.empty(rows, (cols + 127) // 128 * 128, dtype=torch.int8, device="cuda"),
                  torch.empty(rows, dtype=torch.float32, device="cuda"), cols)

    def _set(self, codes, scales, cols):
        global _device, _raw_stream
        if not _DTYPES:
            import torch
            lib()
            _raw_stream = torch._C._cuda_getCurrentRawStream
            if torch.cuda.device_count() > 1:
                _device = torch._C._cuda_getDevice
            _DTYPES.update({torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16})
        self.codes, self.scales, self.rows, self.cols, self.shape = codes, scales, codes.shape[0], cols, (codes.shape[0], cols)
        self.device = codes.get_device()
        self._c = prism_q8(codes.data_ptr(), scales.data_ptr(), codes.shape[1], self.rows, cols)
        self._ref = C.byref(self._c)

    @classmethod
    def of(cls, codes, scales) -> "Q8":
        """A copy of codes [rows, cols] int8 and scales [rows] fp32 (weights quantised elsewhere, say) in this layout."""
        import torch
        _need(codes.dim() == 2 and codes.dtype is torch.int8 and codes.is_cuda and codes.get_device() == torch.cuda.current_device(),
              "Q8.of: codes [rows, cols] int8 on the current device")
        _need(scales.shape == codes.shape[:1] and scales.dtype is torch.float32 and scales.device == codes.device, "Q8.of: a fp32 scale for each row")
        rows, cols = codes.shape
        _need(cols > 0, f"Q8: {rows} rows of {cols} codes")
        if cols % 128:
            padded = codes.new_zeros(rows, (cols + 127) // 128 * 128)
            padded[:, :cols] = codes
        else:
            padded = codes.clone(memory_format=torch.contiguous_format)
        q = cls.__new__(cls)
        q._set(padded, scales.clone(memory_format=torch.contiguous_format), cols)
        return q

    def first(self, rows: int) -> "Q8":
        """The first `rows` rows, in place: a buffer made for the largest batch serves smaller ones."""
        _need(0 <= rows <= self.rows, f"Q8.first: {rows} of {self.rows} rows")
        q = Q8.__new__(Q8)
        q._set(self.codes[:rows], self.scales[:rows], self.cols)
        return q


def _any_rows(t, shape, device: int, what: str):
    """Address, row stride and dtype number of a device tensor of that shape whose rows are dense."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is not None and t.shape == shape and t.get_device() == device:
        stride, one = t.stride()
        if one == 1 or shape[1] < 2:
            return t.data_ptr(), stride if shape[0] > 1 else shape[1], dtype
    raise PrismError(EINVAL, f"{what}: {list(shape)} in fp32, bf16 or half, rows dense, on the current device")


def _elsewhere():
    raise PrismError(EINVAL, "8-bit rows on another device than the current one")


def op_quantize_q8(X, out: Q8):
    """X [rows, cols] fp32, bf16 or half -> out."""
    d = _device()
    x, x_stride, dtype = _any_rows(X, out.shape, d, "op_quantize_q8: X")
    if out.device != d:
        _elsewhere()
    rc = _lib.prism_op_quantize_q8(dtype, x, x_stride, out._ref, _raw_stream(d))
    if rc:
        _check(rc)


def op_dequantize_q8(q: Q8, out):
    """q -> out [rows, cols] fp32, bf16 or half."""
    d = _device()
    o, o_stride, dtype = _any_rows(out, q.shape, d, "op_dequantize_q8: out")
    if q.device != d:
        _elsewhere()
    rc = _lib.prism_op_dequantize_q8(q._ref, dtype, o, o_stride, _raw_stream(d))
    if rc:
        _check(rc)


def op_rmsnorm_q8(X, gain, eps, out: Q8, add=None):
    """X [rows, cols] fp32 (+= add, any dtype, where given), normed and quantised to out; gain [cols], any dtype."""
    d = _device()
    x, x_stride, dtype = _any_rows(X, out.shape, d, "op_rmsnorm_q8: X")
    gain_dtype = _DTYPES.get(gain.dtype)
    if dtype or gain_dtype is None or gain.numel() != out.cols or not gain.is_contiguous() or gain.get_device() != d:
        raise PrismError(EINVAL, f"op_rmsnorm_q8: X in fp32 and a gain of {out.cols} values on the current device")
    a, a_stride, add_dtype = (0, 0, 0) if add is None else _any_rows(add, out.shape, d, "op_rmsnorm_q8: add")
    if out.device != d:
        _elsewhere()
    rc = _lib.prism_op_rmsnorm_q8(x, x_stride, add_dtype, a, a_stride, gain_dtype, gain.data_ptr(), eps, out._ref, _raw_stream(d))
    if rc:
        _check(rc)


def op_gemm_q8(epilogue, A: Q8, W: Q8, out):
    """out [A.rows, W.rows] (EPI_SWIGLU: W.rows / 2 columns) = epilogue of A W^T: bf16 or half for EPI_STORE and EPI_SWIGLU, else fp32."""
    d = _device()
    o, o_stride, dtype = _any_rows(out, (A.rows, W.rows // 2 if epilogue == EPI_SWIGLU else W.rows), d, "op_gemm_q8: out")
    if A.device != d or W.device != d:
        _elsewhere()
    rc = _lib.prism_op_gemm_q8(epilogue, A._ref, W._ref, dtype, o, o_stride, _raw_stream(d))
    if rc:
        _check(rc)
