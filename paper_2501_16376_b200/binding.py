"""Thin ctypes binding of libswiftprune.so: same names as the C ABI, argument marshalling only.

Every step of the pruning pass runs in the library's CUDA kernels.  PyTorch tensors are used
for device memory and streams; this module reads their ``data_ptr()``, shape and stride and
passes them through.  If the compiled library is missing the import fails: there is no
fallback path.

A call works on the current stream, or on ``stream``.  What it makes itself (results that were not
given, scratch memory) is then that stream's memory; inputs are ordered by the caller.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
#: the compiled library; SWIFTPRUNE_LIBRARY may point at another build of the same ABI
LIB_PATH = os.environ.get("SWIFTPRUNE_LIBRARY") or os.path.join(_HERE, "libswiftprune.so")

SP_OK = 0
SP_ERR_INVALID_ARG, SP_ERR_SHAPE, SP_ERR_DTYPE, SP_ERR_STATE = 1, 2, 3, 4
SP_ERR_DEGENERATE, SP_ERR_CUDA, SP_ERR_NOMEM = 5, 6, 7
SP_F16, SP_BF16 = 0, 1
SP_S_GATED, SP_S_LITERAL_W2, SP_S_FROZEN, SP_S_READING_X2, SP_S_LITERAL_SCAN = 0, 1, 2, 3, 4
SP_COUNTER_KEPT, SP_COUNTER_S_HAZARD, SP_NUM_COUNTERS = 0, 1, 2
SP_CALIB_X_COMPLETE = 1
SP_MX4_A16, SP_MX4_A4 = 0, 1

#: every symbol include/swiftprune.h declares
EXPORTS = (
    "sp_create", "sp_destroy", "sp_calib_reset", "sp_calib_accumulate", "sp_calib_accumulate_ex", "sp_calib_accumulate_multi", "sp_finalize_multi",
    "sp_get_stats",
    "sp_set_stats", "sp_calib_stats_noalloc", "sp_score", "sp_la_for_sparsity", "sp_select_unstructured",
    "sp_select_unstructured_ex", "sp_search_la", "sp_ewma_trace", "sp_select_nm", "sp_select_24_compressed", "sp_apply_mask", "sp_calib_accumulate_host",
    "sp_select_nm_host", "sp_select_unstructured_host", "sp_select_unstructured_group",
    "sp_select_unstructured_group_ex", "sp_select_nm_group", "sp_select_unstructured_multi",
    "sp_select_unstructured_multi_ex", "sp_select_nm_multi", "sp_mx4_scale_bytes", "sp_mx4_quantize",
    "sp_mx4_dequantize", "sp_mx4_linear_workspace", "sp_mx4_linear", "sp_cache_append",
    "sp_cache_attention_workspace", "sp_cache_attention", "sp_cache_evict", "sp_qk_norm_rotary",
    "sp_cache_fork_workspace", "sp_cache_fork", "sp_cache_reserve_workspace", "sp_cache_reserve",
    "sp_cache_compact_workspace", "sp_cache_compact", "sp_cache_attention_shared_workspace",
    "sp_cache_attention_shared", "sp_wait_status",
    "sp_debug_status", "sp_status_string",
    "sp_last_cuda_error", "sp_launch_count",
)


class SpError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(what)


class EwmaParams(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("beta", ctypes.c_float), ("la", ctypes.c_float),
                ("s_update", ctypes.c_int)]


class Matrix(ctypes.Structure):
    """sp_matrix: one weight matrix of a grouped selection call."""
    _fields_ = [("W", ctypes.c_void_p), ("n_rows", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("mask_out", ctypes.c_void_p), ("W_out", ctypes.c_void_p), ("ldo", ctypes.c_int64)]


class Batch(ctypes.Structure):
    """sp_batch: one batch of calibration activations of a multi-input call."""
    _fields_ = [("X", ctypes.c_void_p), ("n_tokens", ctypes.c_int64), ("ldx", ctypes.c_int64)]


class CacheStruct(ctypes.Structure):
    """sp_cache: an 8-bit key/value cache."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("n_blocks", ctypes.c_int64), ("n_seqs", ctypes.c_int64),
                ("table_cols", ctypes.c_int64), ("ld_table", ctypes.c_int64),
                ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("block_tokens", ctypes.c_int)]


class Strides(ctypes.Structure):
    """sp_strides: strides in elements of a [sequence, token, head, head_dim] tensor."""
    _fields_ = [("seq", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


SP_MAX_GROUP = 8
SP_MAX_MULTI = 16


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libswiftprune.so is not built (%s); run `python -m paper_2501_16376_b200.build`. "
            "There is no CPU fallback." % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, ci, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    lib.sp_create.argtypes = [ctypes.POINTER(vp), i64, ci]
    lib.sp_destroy.argtypes = [vp]
    lib.sp_calib_reset.argtypes = [vp, vp]
    lib.sp_calib_accumulate.argtypes = [vp, vp, ci, i64, i64, vp]
    lib.sp_calib_accumulate_ex.argtypes = [vp, vp, ci, i64, i64, ctypes.c_uint, vp]
    lib.sp_get_stats.argtypes = [vp, vp, vp, vp, ctypes.POINTER(i64), vp]
    lib.sp_set_stats.argtypes = [vp, vp, i64, vp]
    lib.sp_score.argtypes = [vp, vp, ci, i64, i64, vp, vp]
    lib.sp_calib_stats_noalloc.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp, vp]
    lib.sp_la_for_sparsity.argtypes = [f32, ctypes.POINTER(f32)]
    lib.sp_select_unstructured.argtypes = [vp, vp, ci, i64, i64, f32, vp, vp, i64, vp, vp]
    lib.sp_select_unstructured_ex.argtypes = [vp, vp, ci, i64, i64, ctypes.POINTER(EwmaParams),
                                              vp, vp, i64, vp, vp]
    lib.sp_select_nm.argtypes = [vp, vp, ci, i64, i64, ci, ci, vp, vp, i64, vp]
    lib.sp_select_24_compressed.argtypes = [vp, vp, ci, i64, i64, vp, i64, vp, vp]
    lib.sp_ewma_trace.argtypes = [vp, vp, ci, i64, i64, ctypes.POINTER(EwmaParams), vp, vp, vp, vp]
    lib.sp_search_la.argtypes = [vp, vp, ci, i64, i64, f32, f32, f32, ci, ctypes.POINTER(f32),
                                 ctypes.POINTER(ctypes.c_double), vp]
    lib.sp_apply_mask.argtypes = [vp, ci, i64, i64, i64, vp, vp, i64, vp]
    lib.sp_calib_accumulate_host.argtypes = [vp, vp, ci, i64, i64, vp]
    lib.sp_select_nm_host.argtypes = [vp, vp, ci, i64, i64, ci, ci, vp, vp, i64, vp]
    lib.sp_select_unstructured_host.argtypes = [vp, vp, ci, i64, i64, f32, vp, vp, i64, vp]
    lib.sp_select_unstructured_group.argtypes = [vp, ctypes.POINTER(Matrix), ci, ci, f32, vp, vp]
    lib.sp_select_unstructured_group_ex.argtypes = [vp, ctypes.POINTER(Matrix), ci, ci,
                                                    ctypes.POINTER(EwmaParams), vp, vp]
    lib.sp_select_nm_group.argtypes = [vp, ctypes.POINTER(Matrix), ci, ci, ci, ci, vp]
    lib.sp_select_unstructured_multi.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Matrix), ci,
                                                 ci, f32, vp, vp]
    lib.sp_select_unstructured_multi_ex.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Matrix), ci,
                                                    ci, ctypes.POINTER(EwmaParams), vp, vp]
    lib.sp_calib_accumulate_multi.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Batch), ci, ci,
                                              ctypes.c_uint, vp]
    lib.sp_finalize_multi.argtypes = [ctypes.POINTER(vp), ci, vp]
    lib.sp_select_nm_multi.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Matrix), ci, ci, ci, ci,
                                       vp]
    pc, ps, pi64 = ctypes.POINTER(CacheStruct), ctypes.POINTER(Strides), ctypes.POINTER(i64)
    lib.sp_mx4_scale_bytes.argtypes = [i64, i64]
    lib.sp_mx4_scale_bytes.restype = i64
    lib.sp_mx4_quantize.argtypes = [vp, ci, i64, i64, i64, vp, vp, i64, vp, vp]
    lib.sp_mx4_dequantize.argtypes = [vp, i64, vp, i64, i64, ci, vp, i64, vp]
    lib.sp_mx4_linear_workspace.argtypes = [i64, i64, i64, ci, pi64]
    lib.sp_mx4_linear.argtypes = [vp, ci, i64, i64, vp, i64, vp, i64, i64, ci, vp, i64, vp, i64, vp]
    lib.sp_cache_append.argtypes = [pc, vp, ps, vp, ps, ci, i64, vp, vp, vp]
    lib.sp_cache_attention_workspace.argtypes = [pc, i64, ci, i64, ci, pi64]
    lib.sp_cache_attention.argtypes = [pc, vp, ps, ci, i64, ci, vp, i64, f32, vp, ps, vp, vp, vp,
                                       i64, vp, i64, vp]
    lib.sp_cache_evict.argtypes = [pc, vp, i64, vp, i64, i64, i64, pc, vp, vp, i64, vp, vp]
    lib.sp_qk_norm_rotary.argtypes = [vp, ps, ci, vp, ps, ci, ci, i64, i64, ci, vp, vp, f32, vp, vp,
                                      ci, ci, vp, ps, vp, ps, vp]
    lib.sp_cache_fork_workspace.argtypes = [pc, i64, pi64]
    lib.sp_cache_fork.argtypes = [pc, vp, vp, vp, i64, vp, i64, vp]
    lib.sp_cache_reserve_workspace.argtypes = [pc, i64, pi64]
    lib.sp_cache_reserve.argtypes = [pc, vp, vp, vp, i64, vp, vp, i64, vp]
    lib.sp_cache_compact_workspace.argtypes = [pc, pi64]
    lib.sp_cache_compact.argtypes = [pc, vp, vp, i64, vp, vp, vp, i64, vp]
    lib.sp_cache_attention_shared_workspace.argtypes = [pc, i64, ci, i64, i64, i64, i64, pi64]
    lib.sp_cache_attention_shared.argtypes = [pc, vp, ps, ci, i64, ci, vp, i64, vp, i64, vp, i64, i64,
                                              f32, vp, ps, vp, vp, i64, vp]
    lib.sp_wait_status.argtypes = [ctypes.POINTER(ci), ci]
    lib.sp_debug_status.argtypes = [ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(i64),
                                    ctypes.POINTER(i64), ci]
    lib.sp_status_string.argtypes = [ci]
    lib.sp_status_string.restype = ctypes.c_char_p
    lib.sp_last_cuda_error.restype = ctypes.c_char_p
    lib.sp_launch_count.restype = ctypes.c_uint64
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is ctypes.c_int and name not in ("sp_status_string",):
            fn.restype = ci
    return lib


lib = _load()


def _check(status: int):
    if status != SP_OK:
        msg = lib.sp_status_string(status).decode()
        if status in (SP_ERR_CUDA, SP_ERR_NOMEM):
            msg += " [" + lib.sp_last_cuda_error().decode() + "]"
        raise SpError(status, msg)


def _dtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return SP_F16
    if t.dtype == torch.bfloat16:
        return SP_BF16
    raise SpError(SP_ERR_DTYPE, "expected a float16 or bfloat16 tensor, got %s" % t.dtype)


def _matrix(t: torch.Tensor, what: str, host: bool = False):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise SpError(SP_ERR_SHAPE, "%s must be 2-D with unit stride along its rows" % what)
    if t.is_cuda == host:
        raise SpError(SP_ERR_INVALID_ARG,
                      "%s must be a %s tensor" % (what, "CPU" if host else "CUDA"))
    ld = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])
    return t.data_ptr(), t.shape[0], t.shape[1], ld


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _torch_stream(stream):
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()


def _scratch(stream, make, *args, **kw):
    """make(*args, **kw): a tensor that only the work of a call on `stream` (None: the current one)
    uses.  It comes from that stream's memory.  A block that the allocator hands out again on the
    current stream may still be in use by what is pending there, and a launch on another stream
    does not wait for that."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(_torch_stream(stream)):
        return make(*args, **kw)


def _result(stream, make, *args, **kw):
    """The same for a tensor that is returned: the caller's stream counts as using it, so that it is
    not handed out again while work there reads it."""
    t = _scratch(stream, make, *args, **kw)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream())
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def sp_launch_count() -> int:
    return int(lib.sp_launch_count())


def sp_debug_status(clear: bool = False):
    """(violations, first_code, first_index, first_limit) of the debug build's index checks;
    violations is -1 for the release build."""
    v, c = ctypes.c_int(), ctypes.c_int()
    i, lim = ctypes.c_int64(), ctypes.c_int64()
    _check(lib.sp_debug_status(ctypes.byref(v), ctypes.byref(c), ctypes.byref(i), ctypes.byref(lim),
                               1 if clear else 0))
    return v.value, c.value, i.value, lim.value


def sp_la_for_sparsity(sparsity: float) -> float:
    out = ctypes.c_float()
    _check(lib.sp_la_for_sparsity(sparsity, ctypes.byref(out)))
    return out.value


class Context:
    """Owns one ``sp_ctx`` (one layer input of ``d_in`` channels)."""

    def __init__(self, d_in: int, device: int | None = None):
        if device is None:
            device = torch.cuda.current_device()
        self.d_in = int(d_in)
        self.device = int(device)
        h = ctypes.c_void_p()
        _check(lib.sp_create(ctypes.byref(h), self.d_in, self.device))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib.sp_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- calibration ---------------------------------------------------------
    def sp_calib_reset(self, stream=None):
        _check(lib.sp_calib_reset(self._h, _stream(stream)))

    def sp_calib_accumulate(self, X: torch.Tensor, stream=None, x_complete: bool = False):
        """x_complete: X was complete before the preceding operation on the stream began
        (SP_CALIB_X_COMPLETE, see the C header)."""
        ptr, T, n, ld = _matrix(X, "X")
        if n != self.d_in:
            raise SpError(SP_ERR_SHAPE, "X has %d channels, context has %d" % (n, self.d_in))
        if x_complete:
            _check(lib.sp_calib_accumulate_ex(self._h, ptr, _dtype_of(X), T, ld,
                                              SP_CALIB_X_COMPLETE, _stream(stream)))
        else:
            _check(lib.sp_calib_accumulate(self._h, ptr, _dtype_of(X), T, ld, _stream(stream)))

    def sp_get_stats(self, stream=None):
        """Returns (colsq fp64 [d_in], S, factor fp32 [d_in], n_tokens) as CPU tensors/numbers."""
        colsq = torch.empty(self.d_in, dtype=torch.float64)
        factor = torch.empty(self.d_in, dtype=torch.float32)
        S = ctypes.c_double()
        ntok = ctypes.c_int64()
        _check(lib.sp_get_stats(self._h, colsq.data_ptr(), ctypes.addressof(S), factor.data_ptr(),
                                ctypes.byref(ntok), _stream(stream)))
        return colsq, S.value, factor, ntok.value

    def sp_set_stats(self, colsq: torch.Tensor, n_tokens: int, stream=None):
        colsq = colsq.detach().to("cpu", torch.float64).contiguous()
        if colsq.numel() != self.d_in:
            raise SpError(SP_ERR_SHAPE, "colsq must have d_in entries")
        _check(lib.sp_set_stats(self._h, colsq.data_ptr(), int(n_tokens), _stream(stream)))

    # -- metric --------------------------------------------------------------
    def sp_score(self, W: torch.Tensor | None = None, want_scores: bool = True, stream=None):
        """Finalises the statistics; with W, returns the fp32 score matrix L (Eq. 8)."""
        if W is None or not want_scores:
            _check(lib.sp_score(self._h, None, SP_F16, 0, self.d_in, None, _stream(stream)))
            return None
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        scores = _result(stream, torch.empty, R, n, dtype=torch.float32, device=W.device)
        _check(lib.sp_score(self._h, ptr, _dtype_of(W), R, ld, scores.data_ptr(), _stream(stream)))
        return scores

    def sp_select_24_compressed(self, W, values=None, meta=None, stream=None):
        """2:4 selection emitted as kept values [R, d_in/2] + 4-bit-per-group indices
        [R, ceil(d_in/32)] int32 (layout in the C header).  Returns (values, meta)."""
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        if values is None:
            values = _result(stream, torch.empty, R, n // 2, dtype=W.dtype, device=W.device)
        if meta is None:
            meta = _result(stream, torch.zeros, R, (n + 31) // 32, dtype=torch.int32, device=W.device)
        vptr, _, _, ldv = _matrix(values, "values")
        _check(lib.sp_select_24_compressed(self._h, ptr, _dtype_of(W), R, ld, vptr, ldv,
                                           meta.data_ptr(), _stream(stream)))
        return values, meta

    def _check_width(self, n):
        if n != self.d_in:
            raise SpError(SP_ERR_SHAPE, "W has %d columns, context has %d" % (n, self.d_in))

    def _outputs(self, W, mask, W_out, want_mask, inplace, stream):
        R, n = W.shape
        if mask is None and want_mask:
            mask = _result(stream, torch.empty, R, (n + 31) // 32, dtype=torch.int32, device=W.device)
        if inplace:
            W_out = W
        elif W_out is None:
            W_out = _result(stream, torch.empty_like, W)
        return mask, W_out

    # -- selection -----------------------------------------------------------
    def sp_select_unstructured(self, W, sparsity=None, *, params: EwmaParams | None = None,
                               mask=None, W_out=None, inplace=False, want_mask=True,
                               counters=None, stream=None):
        """Algorithm 1 on every row of W.  Returns (mask int32 [R, ceil(n/32)], W_out)."""
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        mask, W_out = self._outputs(W, mask, W_out, want_mask, inplace, stream)
        optr, _, _, ldo = _matrix(W_out, "W_out")
        if params is not None:
            _check(lib.sp_select_unstructured_ex(self._h, ptr, _dtype_of(W), R, ld,
                                                 ctypes.byref(params), _ptr(mask), optr, ldo,
                                                 _ptr(counters), _stream(stream)))
        else:
            _check(lib.sp_select_unstructured(self._h, ptr, _dtype_of(W), R, ld, float(sparsity),
                                              _ptr(mask), optr, ldo, _ptr(counters),
                                              _stream(stream)))
        return mask, W_out

    def sp_ewma_trace(self, W, params: EwmaParams, stream=None):
        """est, dev (state before each element's update) and L along every row: three fp32
        tensors [R, d_in].  Sequential diagnostic, meant for a few rows."""
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        est, dev, L = (_result(stream, torch.empty, R, n, dtype=torch.float32, device=W.device) for _ in range(3))
        _check(lib.sp_ewma_trace(self._h, ptr, _dtype_of(W), R, ld, ctypes.byref(params),
                                 est.data_ptr(), dev.data_ptr(), L.data_ptr(), _stream(stream)))
        return est, dev, L

    def sp_search_la(self, W, target_sparsity: float, alpha: float = 0.125, beta: float = 0.125,
                     iterations: int = 24, stream=None):
        """Bisects la so that Algorithm 1 prunes target_sparsity of W.  Returns (la, achieved)."""
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        la = ctypes.c_float()
        got = ctypes.c_double()
        _check(lib.sp_search_la(self._h, ptr, _dtype_of(W), R, ld, float(target_sparsity),
                                float(alpha), float(beta), int(iterations), ctypes.byref(la),
                                ctypes.byref(got), _stream(stream)))
        return la.value, got.value

    def sp_select_nm(self, W, N: int, M: int, *, mask=None, W_out=None, inplace=False,
                     want_mask=True, stream=None):
        """N:M selection (keep N of every M).  Returns (mask, W_out)."""
        ptr, R, n, ld = _matrix(W, "W")
        self._check_width(n)
        mask, W_out = self._outputs(W, mask, W_out, want_mask, inplace, stream)
        optr, _, _, ldo = _matrix(W_out, "W_out")
        _check(lib.sp_select_nm(self._h, ptr, _dtype_of(W), R, ld, int(N), int(M), _ptr(mask),
                                optr, ldo, _stream(stream)))
        return mask, W_out

    # -- grouped selection (layers that read this context's input) ----------------------
    def sp_select_unstructured_group(self, Ws, sparsity=None, *, params: EwmaParams | None = None,
                                     masks=None, W_outs=None, inplace=False, want_mask=True,
                                     counters=None, stream=None):
        """Algorithm 1 on several matrices that read this context's input, in one call.
        Returns (masks, W_outs)."""
        arr, k, dtype, masks, W_outs = _group(self, Ws, masks, W_outs, want_mask, inplace, stream)
        if params is not None:
            _check(lib.sp_select_unstructured_group_ex(self._h, arr, k, dtype, ctypes.byref(params),
                                                       _ptr(counters), _stream(stream)))
        else:
            _check(lib.sp_select_unstructured_group(self._h, arr, k, dtype, float(sparsity),
                                                    _ptr(counters), _stream(stream)))
        return masks, W_outs

    def sp_select_nm_group(self, Ws, N: int, M: int, *, masks=None, W_outs=None, inplace=False,
                           want_mask=True, stream=None):
        """N:M selection of several matrices that read this context's input, in one call.
        Returns (masks, W_outs)."""
        arr, k, dtype, masks, W_outs = _group(self, Ws, masks, W_outs, want_mask, inplace, stream)
        _check(lib.sp_select_nm_group(self._h, arr, k, dtype, int(N), int(M), _stream(stream)))
        return masks, W_outs

    # -- host-buffer variants: tensors are CPU tensors (pinned for overlap); see the C header

    def sp_calib_accumulate_host(self, X: torch.Tensor, stream=None):
        ptr, T, n, ld = _matrix(X, "X", host=True)
        if n != self.d_in:
            raise SpError(SP_ERR_SHAPE, "X has %d channels, context has %d" % (n, self.d_in))
        _check(lib.sp_calib_accumulate_host(self._h, ptr, _dtype_of(X), T, ld, _stream(stream)))

    def sp_select_nm_host(self, W, N, M, mask, W_out, stream=None):
        ptr, R, n, ld = _matrix(W, "W", host=True)
        self._check_width(n)
        optr, ldo = (None, ld) if W_out is None else (_matrix(W_out, "W_out", host=True)[0],
                                                      _matrix(W_out, "W_out", host=True)[3])
        _check(lib.sp_select_nm_host(self._h, ptr, _dtype_of(W), R, ld, int(N), int(M),
                                     _ptr(mask), optr, ldo, _stream(stream)))

    def sp_select_unstructured_host(self, W, sparsity, mask, W_out, stream=None):
        ptr, R, n, ld = _matrix(W, "W", host=True)
        self._check_width(n)
        optr, ldo = (None, ld) if W_out is None else (_matrix(W_out, "W_out", host=True)[0],
                                                      _matrix(W_out, "W_out", host=True)[3])
        _check(lib.sp_select_unstructured_host(self._h, ptr, _dtype_of(W), R, ld, float(sparsity),
                                               _ptr(mask), optr, ldo, _stream(stream)))


def _group(ctx, Ws, masks, W_outs, want_mask, inplace, stream):
    """Marshals a list of weight tensors (and optional outputs) into an sp_matrix array."""
    k = len(Ws)
    masks = list(masks) if masks is not None else [None] * k
    W_outs = list(W_outs) if W_outs is not None else [None] * k
    arr = (Matrix * k)()
    dtype = _dtype_of(Ws[0])
    for i, W in enumerate(Ws):
        ptr, R, n, ld = _matrix(W, "W")
        ctx._check_width(n)
        if _dtype_of(W) != dtype:
            raise SpError(SP_ERR_DTYPE, "all matrices of a group must have the same dtype")
        masks[i], W_outs[i] = ctx._outputs(W, masks[i], W_outs[i], want_mask, inplace, stream)
        optr, _, _, ldo = _matrix(W_outs[i], "W_out")
        arr[i] = Matrix(ptr, R, ld, _ptr(masks[i]), optr, ldo)
    return arr, k, dtype, masks, W_outs


def sp_calib_accumulate_multi(ctxs, Xs, stream=None, x_complete: bool = False):
    """One batch for each of several layer inputs in one call: Xs[i] ([tokens, d_in of ctxs[i]],
    all of one dtype) is added to the statistics of ctxs[i]; the contexts must all differ."""
    k = len(Xs)
    if k != len(ctxs) or k < 1:
        raise SpError(SP_ERR_INVALID_ARG, "one context per batch")
    arr = (Batch * k)()
    handles = (ctypes.c_void_p * k)()
    dtype = _dtype_of(Xs[0])
    for i, (ctx, X) in enumerate(zip(ctxs, Xs)):
        ptr, T, n, ld = _matrix(X, "X")
        if n != ctx.d_in:
            raise SpError(SP_ERR_SHAPE, "X has %d channels, context has %d" % (n, ctx.d_in))
        if _dtype_of(X) != dtype:
            raise SpError(SP_ERR_DTYPE, "all batches of a call must have the same dtype")
        arr[i] = Batch(ptr, T, ld)
        handles[i] = ctx._h
    _check(lib.sp_calib_accumulate_multi(handles, arr, k, dtype,
                                         SP_CALIB_X_COMPLETE if x_complete else 0,
                                         _stream(stream)))


def sp_finalize_multi(ctxs, stream=None):
    """S and the per-channel factors of every listed context with batches pending, one launch."""
    handles = (ctypes.c_void_p * len(ctxs))(*[c._h for c in ctxs])
    _check(lib.sp_finalize_multi(handles, len(ctxs), _stream(stream)))


def _multi(ctxs, Ws, masks, W_outs, want_mask, inplace, stream):
    """Marshals matrices with a context each into an sp_matrix array and a handle array."""
    k = len(Ws)
    if k != len(ctxs) or k < 1:
        raise SpError(SP_ERR_INVALID_ARG, "one context per matrix")
    masks = list(masks) if masks is not None else [None] * k
    W_outs = list(W_outs) if W_outs is not None else [None] * k
    arr = (Matrix * k)()
    handles = (ctypes.c_void_p * k)()
    dtype = _dtype_of(Ws[0])
    for i, (ctx, W) in enumerate(zip(ctxs, Ws)):
        ptr, R, n, ld = _matrix(W, "W")
        ctx._check_width(n)
        if _dtype_of(W) != dtype:
            raise SpError(SP_ERR_DTYPE, "all matrices of a call must have the same dtype")
        masks[i], W_outs[i] = ctx._outputs(W, masks[i], W_outs[i], want_mask, inplace, stream)
        optr, _, _, ldo = _matrix(W_outs[i], "W_out")
        arr[i] = Matrix(ptr, R, ld, _ptr(masks[i]), optr, ldo)
        handles[i] = ctx._h
    return handles, arr, k, dtype, masks, W_outs


def sp_select_unstructured_multi(ctxs, Ws, sparsity=None, *, params: EwmaParams | None = None,
                                 masks=None, W_outs=None, inplace=False, want_mask=True,
                                 counters=None, stream=None):
    """Algorithm 1 on matrices that read different layer inputs, in one call: Ws[i] is pruned
    with the statistics of ctxs[i] (contexts may repeat).  Returns (masks, W_outs)."""
    handles, arr, k, dtype, masks, W_outs = _multi(ctxs, Ws, masks, W_outs, want_mask, inplace, stream)
    if params is not None:
        _check(lib.sp_select_unstructured_multi_ex(handles, arr, k, dtype, ctypes.byref(params),
                                                   _ptr(counters), _stream(stream)))
    else:
        _check(lib.sp_select_unstructured_multi(handles, arr, k, dtype, float(sparsity),
                                                _ptr(counters), _stream(stream)))
    return masks, W_outs


def sp_select_nm_multi(ctxs, Ws, N: int, M: int, *, masks=None, W_outs=None, inplace=False,
                       want_mask=True, stream=None):
    """N:M selection of matrices that read different layer inputs, in one call: Ws[i] is pruned
    with the statistics of ctxs[i].  Returns (masks, W_outs)."""
    handles, arr, k, dtype, masks, W_outs = _multi(ctxs, Ws, masks, W_outs, want_mask, inplace, stream)
    _check(lib.sp_select_nm_multi(handles, arr, k, dtype, int(N), int(M), _stream(stream)))
    return masks, W_outs


def sp_apply_mask(W: torch.Tensor, mask: torch.Tensor, W_out: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    ptr, R, n, ld = _matrix(W, "W")
    if W_out is None:
        W_out = _result(stream, torch.empty_like, W)
    optr, _, _, ldo = _matrix(W_out, "W_out")
    if mask.dim() != 2 or tuple(mask.shape) != (R, (n + 31) // 32) or not mask.is_contiguous():
        raise SpError(SP_ERR_SHAPE, "mask must be contiguous [rows, ceil(cols/32)]")
    _check(lib.sp_apply_mask(ptr, _dtype_of(W), R, n, ld, mask.data_ptr(), optr, ldo,
                             _stream(stream)))
    return W_out


def sp_calib_stats_noalloc(X: torch.Tensor, colsq_out: torch.Tensor | None = None,
                           factor_out: torch.Tensor | None = None,
                           S_out: torch.Tensor | None = None, stream=None):
    """One-shot statistics of a single batch for callers that cannot allocate device memory:
    the library uses a fixed internal array instead of a context (d_in <= 16384).  The outputs
    are device tensors the caller already owns (fp64 [d_in], fp32 [d_in], fp64 [1]); this
    wrapper allocates nothing either.  Calls on one device must not overlap on the GPU."""
    ptr, T, n, ld = _matrix(X, "X")
    for t, dt, numel in ((colsq_out, torch.float64, n), (factor_out, torch.float32, n),
                         (S_out, torch.float64, 1)):
        if t is not None and (t.dtype != dt or t.numel() < numel or not t.is_cuda
                              or not t.is_contiguous()):
            raise SpError(SP_ERR_INVALID_ARG, "output buffers must be contiguous CUDA tensors "
                                              "of the documented type and size")
    with torch.cuda.device(X.device):
        _check(lib.sp_calib_stats_noalloc(ptr, _dtype_of(X), T, n, ld, _ptr(colsq_out),
                                          _ptr(factor_out), _ptr(S_out), _stream(stream)))


# ---------------------------------------------------------------- microscaled 4-bit weights

# These calls sit in decoding loops whose kernels take microseconds, so their checks are kept to
# a few hundred nanoseconds each: the current device is asked for once a call, and what depends on
# sizes alone is remembered.

def _on_device(t: torch.Tensor, what: str, device: int):
    if t.get_device() != device:
        raise SpError(SP_ERR_INVALID_ARG, "%s must be a CUDA tensor of the current device" % what)


def _rows(t: torch.Tensor, what: str, device: int):
    """_matrix for a tensor of the current device."""
    if t.get_device() != device:
        raise SpError(SP_ERR_INVALID_ARG, "%s must be a CUDA tensor of the current device" % what)
    shape = t.shape
    if len(shape) != 2:
        raise SpError(SP_ERR_SHAPE, "%s must be 2-D with unit stride along its rows" % what)
    R, n = shape
    ld, inner = t.stride()
    if n > 1 and inner != 1:
        raise SpError(SP_ERR_SHAPE, "%s must be 2-D with unit stride along its rows" % what)
    return t.data_ptr(), R, n, ld if R > 1 else max(ld, n)


_current_device = torch.cuda.current_device


def _raw_stream(stream, device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


def _codes(codes: torch.Tensor, scales: torch.Tensor, n_cols: int, device: int):
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
        raise SpError(SP_ERR_DTYPE, "codes and scales are uint8 tensors")
    ptr, R, width, ldc = _rows(codes, "codes", device)
    _on_device(scales, "scales", device)
    if width < (n_cols + 31) // 32 * 16:
        raise SpError(SP_ERR_SHAPE, "codes have %d bytes a row, %d columns need %d"
                      % (width, n_cols, (n_cols + 31) // 32 * 16))
    if scales.numel() < sp_mx4_scale_bytes(R, n_cols) or not scales.is_contiguous():
        raise SpError(SP_ERR_SHAPE, "scales must be contiguous with sp_mx4_scale_bytes entries")
    return ptr, R, ldc, scales.data_ptr()


@functools.lru_cache(maxsize=4096)
def sp_mx4_scale_bytes(n_rows: int, n_cols: int) -> int:
    return int(lib.sp_mx4_scale_bytes(int(n_rows), int(n_cols)))


def sp_mx4_quantize(W: torch.Tensor, mask: torch.Tensor | None = None, codes=None, scales=None,
                    stream=None):
    """Microscaled 4-bit form of W (with the keep mask of a selection applied on the way).
    Returns (codes uint8 [rows, 16 * ceil(cols / 32)], scales uint8 in tiles; layout in the C
    header)."""
    device = _current_device()
    ptr, R, n, ld = _rows(W, "W", device)
    if mask is not None:
        _on_device(mask, "mask", device)
        if (mask.dtype != torch.int32 or tuple(mask.shape) != (R, (n + 31) // 32)
                or not mask.is_contiguous()):
            raise SpError(SP_ERR_SHAPE, "mask must be contiguous int32 [rows, ceil(cols/32)]")
    if codes is None:
        codes = _result(stream, torch.empty, R, (n + 31) // 32 * 16, dtype=torch.uint8, device=W.device)
    if scales is None:
        scales = _result(stream, torch.empty, sp_mx4_scale_bytes(R, n), dtype=torch.uint8, device=W.device)
    cptr, rows, ldc, sptr = _codes(codes, scales, n, device)
    if rows != R:
        raise SpError(SP_ERR_SHAPE, "codes have %d rows, W has %d" % (rows, R))
    _check(lib.sp_mx4_quantize(ptr, _dtype_of(W), R, n, ld, _ptr(mask), cptr, ldc, sptr,
                               _raw_stream(stream, device)))
    return codes, scales


def sp_mx4_dequantize(codes: torch.Tensor, scales: torch.Tensor, n_cols: int, dtype=None,
                      W_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The values of a 4-bit matrix as a 16-bit one [rows, n_cols] (of W_out's type, or dtype)."""
    device = _current_device()
    cptr, R, ldc, sptr = _codes(codes, scales, n_cols, device)
    if W_out is None:
        W_out = _result(stream, torch.empty, R, n_cols, dtype=dtype or torch.bfloat16, device=codes.device)
    optr, rows, n, ldo = _rows(W_out, "W_out", device)
    if (rows, n) != (R, n_cols):
        raise SpError(SP_ERR_SHAPE, "W_out must be [%d, %d]" % (R, n_cols))
    _check(lib.sp_mx4_dequantize(cptr, ldc, sptr, R, n_cols, _dtype_of(W_out), optr, ldo,
                                 _raw_stream(stream, device)))
    return W_out


def _workspace(need: int, workspace, like, device: int, stream):
    """(pointer, bytes, tensor that keeps it alive) of a call's scratch memory."""
    if need == 0:
        return None, 0, None
    if workspace is None:
        workspace = _scratch(stream, torch.empty, need, dtype=torch.uint8, device=like.device)
    elif workspace.numel() * workspace.element_size() < need or not workspace.is_contiguous():
        raise SpError(SP_ERR_INVALID_ARG, "the workspace needs %d contiguous bytes" % need)
    else:
        _on_device(workspace, "the workspace", device)
    return workspace.data_ptr(), need, workspace


@functools.lru_cache(maxsize=4096)
def sp_mx4_linear_workspace(n_tokens: int, n_rows: int, n_cols: int, mode: int = SP_MX4_A16) -> int:
    need = ctypes.c_int64()
    _check(lib.sp_mx4_linear_workspace(int(n_tokens), int(n_rows), int(n_cols), int(mode),
                                       ctypes.byref(need)))
    return need.value


def sp_mx4_linear(X: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                  mode: int = SP_MX4_A16, Y: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y [tokens, rows] = X [tokens, cols] times the transposed 4-bit matrix.  SP_MX4_A16 takes
    X as it is, SP_MX4_A4 quantises it like the weights first."""
    device = _current_device()
    ptr, T, n, ldx = _rows(X, "X", device)
    cptr, R, ldc, sptr = _codes(codes, scales, n, device)
    if Y is None:
        Y = _result(stream, torch.empty, T, R, dtype=X.dtype, device=X.device)
    yptr, rows, cols, ldy = _rows(Y, "Y", device)
    if (rows, cols) != (T, R):
        raise SpError(SP_ERR_SHAPE, "Y must be [%d, %d]" % (T, R))
    if Y.dtype != X.dtype:
        raise SpError(SP_ERR_DTYPE, "X and Y must have the same dtype")
    if yptr == ptr and ptr:
        raise SpError(SP_ERR_INVALID_ARG, "Y is memory apart from X")
    need = sp_mx4_linear_workspace(T, R, n, mode)
    if mode == SP_MX4_A16 and ptr % 16 == 0 and ldx % 8 == 0:
        need = 0
    wptr, wbytes, keep = _workspace(need, workspace, X, device, stream)
    _check(lib.sp_mx4_linear(ptr, _dtype_of(X), T, ldx, cptr, ldc, sptr, R, n, mode, yptr, ldy,
                             wptr, wbytes, _raw_stream(stream, device)))
    return Y


# ---------------------------------------------------------------- 8-bit key/value cache

@functools.lru_cache(maxsize=4096)
def _strides(seq: int, token: int, head: int) -> Strides:
    return Strides(seq, token, head)


def _heads(t: torch.Tensor, what: str, n_seqs: int, head_dim: int, device: int) -> Strides:
    shape, s = t.shape, t.stride()
    if len(shape) != 4 or shape[0] != n_seqs or shape[3] != head_dim or s[3] != 1:
        raise SpError(SP_ERR_SHAPE, "%s must be [%d, tokens, heads, %d] with consecutive values"
                      % (what, n_seqs, head_dim))
    _on_device(t, what, device)
    return _strides(s[0], s[1], s[2])


@functools.lru_cache(maxsize=4096)
def _query_layout(q, qs, o, os_, n_seqs: int, head_dim: int):
    """Queries, heads and strides of a [n_seqs, n_q, heads, head size] tensor and an output like it,
    checked once for their shapes and strides."""
    for shape, stride, what in ((q, qs, "Q"), (o, os_, "O")):
        if len(shape) != 4 or shape[0] != n_seqs or shape[3] != head_dim or stride[3] != 1:
            raise SpError(SP_ERR_SHAPE, "%s must be [%d, tokens, heads, %d] with consecutive values"
                          % (what, n_seqs, head_dim))
    if o != q:
        raise SpError(SP_ERR_SHAPE, "O must have the shape of Q")
    return q[1], q[2], _strides(*qs[:3]), _strides(*os_[:3])


def _int32(t, what, shape, device: int):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise SpError(SP_ERR_INVALID_ARG, "%s must be contiguous int32 %s" % (what, list(shape)))
    if t.get_device() != device:
        _on_device(t, what, device)
    return t.data_ptr()


def _acc(t, what, n_seqs, n_heads, length, device: int):
    """Pointer and leading dimension of a float [n_seqs, kv heads, >= length] tensor."""
    shape = t.shape
    if (t.dtype != torch.float32 or len(shape) != 3 or shape[0] != n_seqs or shape[1] != n_heads
            or shape[2] < length or not t.is_contiguous()):
        raise SpError(SP_ERR_SHAPE, "%s must be contiguous float32 [%d, %d, >= %d]"
                      % (what, n_seqs, n_heads, length))
    _on_device(t, what, device)
    return t.data_ptr(), shape[2]


class KvCache:
    """An 8-bit key/value cache over tensors that the caller owns (``sp_cache``): codes uint8
    [n_blocks, kv heads, block tokens, head size] and float32 scales [n_blocks, kv heads] for K
    and V, and an int32 table [n_seqs, blocks of a sequence].  refs (int32 [n_blocks]) counts the
    table entries that name each block, for the calls that share and hand out blocks."""

    def __init__(self, k, v, k_scale, v_scale, table, refs=None):
        device = _current_device()
        for t, what in ((k, "k"), (v, "v")):
            if t.dtype != torch.uint8 or t.dim() != 4 or not t.is_contiguous():
                raise SpError(SP_ERR_INVALID_ARG, "%s must be contiguous uint8 [n_blocks, heads, "
                                                  "block tokens, head size]" % what)
            _on_device(t, what, device)
        if k.shape != v.shape:
            raise SpError(SP_ERR_SHAPE, "k and v must have the same shape")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.float32 or t.shape != k.shape[:2] or not t.is_contiguous():
                raise SpError(SP_ERR_INVALID_ARG, "%s must be contiguous float32 [n_blocks, heads]" % what)
            _on_device(t, what, device)
        if table.dtype != torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise SpError(SP_ERR_INVALID_ARG, "table must be int32 [n_seqs, blocks]")
        _on_device(table, "table", device)
        _int32(refs, "refs", k.shape[:1], device)
        self.device, self.refs = device, refs
        self.k, self.v, self.k_scale, self.v_scale, self.table = k, v, k_scale, v_scale, table
        self.n_seqs, (_, self.n_kv_heads, self.block_tokens, self.head_dim) = table.shape[0], k.shape
        ld = table.stride(0) if self.n_seqs > 1 else max(table.stride(0), table.shape[1])
        self._c = CacheStruct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                              table.data_ptr(), k.shape[0], self.n_seqs, table.shape[1], ld,
                              self.n_kv_heads, self.head_dim, self.block_tokens)
        self._workspaces = {}

    def _here(self, what: str = "the cache") -> int:
        """The current device, which must be the cache's."""
        device = _current_device()
        if self.device != device:
            raise SpError(SP_ERR_INVALID_ARG, "%s lies on device %d, the current one is %d"
                          % (what, self.device, device))
        return device

    @classmethod
    def empty(cls, n_seqs: int, max_tokens: int, n_kv_heads: int, head_dim: int,
              block_tokens: int = 32, device=None) -> "KvCache":
        """A cache with its own blocks for max_tokens tokens of each sequence."""
        device = device or torch.device("cuda", torch.cuda.current_device())
        per = (max_tokens + block_tokens - 1) // block_tokens
        shape = (n_seqs * per, n_kv_heads, block_tokens, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        ks, vs = (torch.ones(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        table = torch.arange(n_seqs * per, dtype=torch.int32, device=device).view(n_seqs, per)
        return cls(k, v, ks, vs, table)

    @classmethod
    def pool(cls, n_seqs: int, max_tokens: int, n_blocks: int, n_kv_heads: int, head_dim: int,
             block_tokens: int = 32, device=None) -> "KvCache":
        """A cache of n_blocks blocks that are all free (``sp_cache_reserve`` hands them out), with
        a table for max_tokens tokens of each sequence."""
        device = device or torch.device("cuda", torch.cuda.current_device())
        shape = (n_blocks, n_kv_heads, block_tokens, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        ks, vs = (torch.ones(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        per = (max_tokens + block_tokens - 1) // block_tokens
        table = torch.full((n_seqs, per), -1, dtype=torch.int32, device=device)
        return cls(k, v, ks, vs, table, torch.zeros(n_blocks, dtype=torch.int32, device=device))

    def sp_cache_append(self, K, V, start, count=None, stream=None):
        """Writes K, V [n_seqs, new, kv heads, head size] at the places start[b] and following
        (start, count: int32 [n_seqs]; count defaults to all the new tokens)."""
        device = self._here()
        ks = _heads(K, "K", self.n_seqs, self.head_dim, device)
        vs = _heads(V, "V", self.n_seqs, self.head_dim, device)
        if K.shape != V.shape or K.shape[2] != self.n_kv_heads:
            raise SpError(SP_ERR_SHAPE, "K and V must have the same shape and %d heads" % self.n_kv_heads)
        if K.dtype != V.dtype:
            raise SpError(SP_ERR_DTYPE, "K and V must have the same dtype")
        shape = (self.n_seqs,)
        _check(lib.sp_cache_append(self._c, K.data_ptr(), ks, V.data_ptr(), vs, _dtype_of(K),
                                   K.shape[1], _int32(start, "start", shape, device),
                                   _int32(count, "count", shape, device),
                                   _raw_stream(stream, device)))

    def sp_cache_attention_workspace(self, n_q: int, n_heads: int, max_len: int, want_acc: bool) -> int:
        key = (n_q, n_heads, max_len, want_acc)
        found = self._workspaces.get(key)
        if found is None:
            need = ctypes.c_int64()
            _check(lib.sp_cache_attention_workspace(self._c, n_q, n_heads, max_len, int(want_acc),
                                                    ctypes.byref(need)))
            if len(self._workspaces) > 4096:
                self._workspaces.clear()
            found = self._workspaces[key] = need.value
        return found

    def sp_cache_attention(self, Q, lens, max_len: int, scale: float | None = None, O=None,
                           lse=None, acc_in=None, acc_out=None, workspace=None, stream=None):
        """Attention of Q [n_seqs, n_q, heads, head size] over the cache, whose lens (int32
        [n_seqs]) count the call's own n_q tokens; max_len bounds them.  scale defaults to
        1 / sqrt(head size).  acc_out (float32 [n_seqs, kv heads, >= max_len]) accumulates the
        attention every token received on top of acc_in.  Returns O."""
        device = self._here()
        qs = _heads(Q, "Q", self.n_seqs, self.head_dim, device)
        if O is None:
            O = _result(stream, torch.empty, Q.shape, dtype=Q.dtype, device=Q.device)
        os_ = _heads(O, "O", self.n_seqs, self.head_dim, device)
        if O.shape != Q.shape:
            raise SpError(SP_ERR_SHAPE, "O must have the shape of Q")
        if O.dtype != Q.dtype:
            raise SpError(SP_ERR_DTYPE, "Q and O must have the same dtype")
        n_q, n_heads = Q.shape[1], Q.shape[2]
        if lse is not None:
            if lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape != Q.shape[:3]:
                raise SpError(SP_ERR_SHAPE, "lse must be contiguous float32 [n_seqs, n_q, heads]")
            _on_device(lse, "lse", device)
        ai = ao = None
        ld = max_len
        if acc_out is not None:
            ao, ld = _acc(acc_out, "acc_out", self.n_seqs, self.n_kv_heads, max_len, device)
            if acc_in is not None:
                ai, ld_in = _acc(acc_in, "acc_in", self.n_seqs, self.n_kv_heads, max_len, device)
                if ld_in != ld:
                    raise SpError(SP_ERR_SHAPE, "acc_in and acc_out must have the same shape")
        need = self.sp_cache_attention_workspace(n_q, n_heads, max_len, ao is not None)
        wptr, wbytes, keep = _workspace(need, workspace, Q, device, stream)
        _check(lib.sp_cache_attention(self._c, Q.data_ptr(), qs, _dtype_of(Q), n_q, n_heads,
                                      _int32(lens, "lens", (self.n_seqs,), device), max_len,
                                      self.head_dim ** -0.5 if scale is None else scale,
                                      O.data_ptr(), os_, _ptr(lse), ai, ao, ld, wptr, wbytes,
                                      _raw_stream(stream, device)))
        return O

    def sp_cache_evict(self, lens, max_len: int, acc, budget: int, recent: int, dst: "KvCache",
                       acc_out=None, kept_out=None, lens_out=None, stream=None):
        """Keeps budget tokens of every (sequence, kv head): the last `recent` and those with the
        largest acc; lays them into dst's blocks.  Returns (kept_out, acc_out, lens_out)."""
        device = self._here()
        a, ld = _acc(acc, "acc", self.n_seqs, self.n_kv_heads, max_len, device)
        dst._here("dst")
        if dst.n_seqs != self.n_seqs:
            raise SpError(SP_ERR_SHAPE, "dst must have the same sequences")
        shape = (self.n_seqs, self.n_kv_heads, budget)
        if kept_out is None:
            kept_out = _result(stream, torch.empty, shape, dtype=torch.int32, device=acc.device)
        if acc_out is None:
            acc_out = _result(stream, torch.empty, shape, dtype=torch.float32, device=acc.device)
        if lens_out is None:
            lens_out = _result(stream, torch.empty, self.n_seqs, dtype=torch.int32, device=acc.device)
        ao, ld_out = _acc(acc_out, "acc_out", self.n_seqs, self.n_kv_heads, budget, device)
        n = _int32(lens, "lens", (self.n_seqs,), device)
        no = _int32(lens_out, "lens_out", (self.n_seqs,), device)
        if (n == no and n) or (a == ao and a):
            raise SpError(SP_ERR_INVALID_ARG, "lens_out and acc_out are memory apart from lens and acc")
        _check(lib.sp_cache_evict(self._c, n, max_len, a, ld, budget, recent, dst._c,
                                  _int32(kept_out, "kept_out", shape, device), ao, ld_out, no,
                                  _raw_stream(stream, device)))
        return kept_out, acc_out, lens_out


    # ------------------------------------------------ several answers of one prompt

    def _counted(self) -> int:
        """The current device, for calls that need the counts."""
        device = self._here()
        if self.refs is None:
            raise SpError(SP_ERR_INVALID_ARG, "the cache has no refs")
        return device

    def _need(self, call: str, *sizes) -> int:
        """A call's workspace, remembered by its sizes."""
        key = (call,) + sizes
        found = self._workspaces.get(key)
        if found is None:
            need = ctypes.c_int64()
            _check(getattr(lib, call)(self._c, *sizes, ctypes.byref(need)))
            if len(self._workspaces) > 4096:
                self._workspaces.clear()
            found = self._workspaces[key] = need.value
        return found

    def sp_cache_fork(self, dst, src=None, workspace=None, stream=None):
        """Rows dst of the table (int32 [n]) become copies of the rows src, or empty where src is
        None or -1; refs follow."""
        device = self._counted()
        if dst.dim() != 1:
            raise SpError(SP_ERR_SHAPE, "dst must be one-dimensional")
        n = dst.shape[0]
        need = self._need("sp_cache_fork_workspace", n)
        wptr, wbytes, keep = _workspace(need, workspace, self.table, device, stream)
        _check(lib.sp_cache_fork(self._c, self.refs.data_ptr(), _int32(dst, "dst", (n,), device),
                                 _int32(src, "src", (n,), device), n, wptr, wbytes,
                                 _raw_stream(stream, device)))

    def sp_cache_reserve(self, start, n_new: int, count=None, status=None, workspace=None, stream=None):
        """Makes the places start[b] and following, n_new (or count[b]) of them, ready for
        sp_cache_append: free blocks, and own copies of shared ones.  Returns status (int32 [2]):
        how many blocks were missing (then nothing has changed), how many are free."""
        device = self._counted()
        if status is None:
            status = _result(stream, torch.empty, 2, dtype=torch.int32, device=self.table.device)
        shape = (self.n_seqs,)
        need = self._need("sp_cache_reserve_workspace", n_new)
        wptr, wbytes, keep = _workspace(need, workspace, self.table, device, stream)
        _check(lib.sp_cache_reserve(self._c, self.refs.data_ptr(), _int32(start, "start", shape, device),
                                    _int32(count, "count", shape, device), n_new,
                                    _int32(status, "status", (2,), device), wptr, wbytes,
                                    _raw_stream(stream, device)))
        return status

    def sp_cache_compact(self, live=None, table_out=None, refs_out=None, workspace=None, stream=None):
        """Moves the live blocks, n of them, into the blocks 0 .. n - 1.  The table and the refs
        that go with it replace the cache's own unless table_out and refs_out (int32, of their
        shapes) are given.  Returns live (int32 [1]), which holds n."""
        device = self._counted()
        if live is None:
            live = _result(stream, torch.empty, 1, dtype=torch.int32, device=self.table.device)
        table_out = self.table if table_out is None else table_out
        refs_out = self.refs if refs_out is None else refs_out
        shape = self.table.shape
        if (table_out.dtype != torch.int32 or table_out.shape != shape
                or (shape[1] > 1 and table_out.stride(1) != 1)):
            raise SpError(SP_ERR_INVALID_ARG, "table_out must be int32 %s" % list(shape))
        _on_device(table_out, "table_out", device)
        ld = table_out.stride(0) if shape[0] > 1 else max(table_out.stride(0), shape[1])
        need = self._need("sp_cache_compact_workspace")
        wptr, wbytes, keep = _workspace(need, workspace, self.table, device, stream)
        _check(lib.sp_cache_compact(self._c, self.refs.data_ptr(), table_out.data_ptr(), ld,
                                    _int32(refs_out, "refs_out", self.refs.shape, device),
                                    _int32(live, "live", (1,), device), wptr, wbytes,
                                    _raw_stream(stream, device)))
        return live

    def sp_cache_attention_shared(self, Q, lens, max_len: int, group_start, prefix, max_prefix: int,
                                  max_group: int, scale: float | None = None, O=None, lse=None,
                                  workspace=None, stream=None):
        """sp_cache_attention where the sequences group_start[g] .. group_start[g + 1] - 1 (int32
        [groups + 1]) share the whole blocks among their first prefix[g] tokens (int32 [groups]),
        which are read once, through the group's first row of the table.  max_prefix and max_group
        bound the prefixes and the sequences of a group.  Returns O."""
        device = self._here()
        if O is None:
            O = _result(stream, torch.empty, Q.shape, dtype=Q.dtype, device=Q.device)
        n_q, n_heads, qs, os_ = _query_layout(Q.shape, Q.stride(), O.shape, O.stride(), self.n_seqs, self.head_dim)
        if O.dtype is not Q.dtype:
            raise SpError(SP_ERR_DTYPE, "Q and O must have the same dtype")
        if not device == Q.get_device() == O.get_device():
            raise SpError(SP_ERR_INVALID_ARG, "Q and O must be CUDA tensors of the current device")
        qptr, optr = Q.data_ptr(), O.data_ptr()
        if optr == qptr and optr:
            raise SpError(SP_ERR_INVALID_ARG, "O is memory apart from Q")
        if lse is not None:
            if lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape != Q.shape[:3]:
                raise SpError(SP_ERR_SHAPE, "lse must be contiguous float32 [n_seqs, n_q, heads]")
            _on_device(lse, "lse", device)
        if prefix.dim() != 1:
            raise SpError(SP_ERR_SHAPE, "prefix must be one-dimensional")
        groups = prefix.shape[0]
        need = self._need("sp_cache_attention_shared_workspace", n_q, n_heads, max_len, groups, max_prefix, max_group)
        wptr, wbytes, keep = _workspace(need, workspace, Q, device, stream)
        _check(lib.sp_cache_attention_shared(
            self._c, qptr, qs, _dtype_of(Q), n_q, n_heads, _int32(lens, "lens", (self.n_seqs,), device),
            max_len, _int32(group_start, "group_start", (groups + 1,), device), groups,
            _int32(prefix, "prefix", (groups,), device), max_prefix, max_group,
            self.head_dim ** -0.5 if scale is None else scale, optr, os_, _ptr(lse), wptr, wbytes,
            _raw_stream(stream, device)))
        return O


@functools.lru_cache(maxsize=4096)
def _rotary_layout(q, qs, k, ks, qo, qos, ko, kos):
    """What a call's shapes and strides come to, checked once: sizes and the four sp_strides."""
    for shape, stride, what in ((q, qs, "Q"), (k, ks, "K"), (qo, qos, "Q_out"), (ko, kos, "K_out")):
        if len(shape) != 4 or shape[0] != q[0] or shape[3] != q[3] or stride[3] != 1:
            raise SpError(SP_ERR_SHAPE, "%s must be [n_seqs, tokens, heads, head size] with consecutive "
                                        "values, of the sequences and the head size of Q" % what)
    if q[1] != k[1]:
        raise SpError(SP_ERR_SHAPE, "Q and K must have the same tokens")
    if qo != q or ko != k:
        raise SpError(SP_ERR_SHAPE, "Q_out and K_out must have the shapes of Q and K")
    return q[0], q[1], q[2], k[2], q[3], _strides(*qs[:3]), _strides(*ks[:3]), _strides(*qos[:3]), _strides(*kos[:3])


def sp_qk_norm_rotary(Q, K, start, freq, q_weight=None, k_weight=None, eps: float = 1e-6,
                      pairs: bool = False, Q_out=None, K_out=None, stream=None):
    """Norms the heads of Q and K [n_seqs, tokens, heads, head size] (where a weight [head size] is
    given) and turns their first 2 * len(freq) values by (start[b] + i) * freq: neighbours together
    if pairs, else the two halves.  Q_out and K_out may be Q and K.  Returns (Q_out, K_out)."""
    device = _current_device()
    if Q_out is None:
        Q_out = _result(stream, torch.empty, Q.shape, dtype=Q.dtype, device=Q.device)
    if K_out is None:
        K_out = _result(stream, torch.empty, K.shape, dtype=K.dtype, device=K.device)
    q_strides, k_strides = Q.stride(), K.stride()
    qo_strides, ko_strides = Q_out.stride(), K_out.stride()
    n_seqs, tokens, heads, kv_heads, dim, qs, ks, qo, ko = _rotary_layout(
        Q.shape, q_strides, K.shape, k_strides, Q_out.shape, qo_strides, K_out.shape, ko_strides)
    dtype = Q.dtype
    if not (K.dtype is dtype and Q_out.dtype is dtype and K_out.dtype is dtype):
        raise SpError(SP_ERR_DTYPE, "Q, K and their outputs must have the same dtype")
    if not device == Q.get_device() == K.get_device() == Q_out.get_device() == K_out.get_device() == freq.get_device():
        raise SpError(SP_ERR_INVALID_ARG, "Q, K, their outputs and freq must be CUDA tensors of the current device")
    qp, kp, qop, kop = Q.data_ptr(), K.data_ptr(), Q_out.data_ptr(), K_out.data_ptr()
    if (qp == qop and q_strides != qo_strides and qp) or (kp == kop and k_strides != ko_strides and kp):
        raise SpError(SP_ERR_INVALID_ARG, "an output in its input's place has its strides")
    wq = wk = None
    if q_weight is not None:
        wq = _head_weight(q_weight, "q_weight", dtype, dim, device)
    if k_weight is not None:
        wk = _head_weight(k_weight, "k_weight", dtype, dim, device)
    if freq.dtype is not torch.float32 or freq.dim() != 1 or not freq.is_contiguous():
        raise SpError(SP_ERR_INVALID_ARG, "freq must be contiguous float32 [rotary / 2]")
    _check(lib.sp_qk_norm_rotary(qp, qs, heads, kp, ks, kv_heads, _dtype_of(Q), n_seqs, tokens, dim, wq, wk,
                                 eps, _int32(start, "start", (n_seqs,), device), freq.data_ptr(),
                                 2 * freq.shape[0], 1 if pairs else 0, qop, qo, kop, ko,
                                 _raw_stream(stream, device)))
    return Q_out, K_out


def _head_weight(w, what, dtype, dim, device) -> int:
    if w.dtype is not dtype or w.shape != (dim,) or not w.is_contiguous() or w.get_device() != device:
        raise SpError(SP_ERR_SHAPE, "%s must be contiguous [%d] of the type and device of Q" % (what, dim))
    return w.data_ptr()


def sp_wait_status(clear: bool = False) -> int:
    """How many bounded waits of the serving kernels ran out (0 unless something is broken)."""
    n = ctypes.c_int()
    _check(lib.sp_wait_status(ctypes.byref(n), 1 if clear else 0))
    return n.value


def new_counters(device=None) -> torch.Tensor:
    """Zeroed device counter block for the selection calls (int64 view of the uint64 pair)."""
    return torch.zeros(SP_NUM_COUNTERS, dtype=torch.int64, device=device or "cuda")
