"""Thin Python binding of libsparoa (include/sparoa.h): argument marshalling only.

Every function here forwards to the C ABI of the same name; tensors are torch
CUDA tensors (device memory and streams come from PyTorch), and the calls run
on the current torch stream.  There is no fallback: if ``libsparoa.so`` is
missing or fails to load, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsparoa.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libsparoa.so is not built ({LIB_PATH}); run __graft_entry__.build()")
_lib = ctypes.CDLL(LIB_PATH)

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_OOM, ERR_CUDA, ERR_TIMEOUT = range(6)
BF16, F32 = 0, 1
PATH_NONE, PATH_DENSE, PATH_SKIP, PATH_DEPTHWISE = 0, 1, 2, 3
ACT_NONE, ACT_RELU, ACT_RELU6, ACT_GELU = 0, 1, 2, 3
OP_CONV2D, OP_FC, OP_MAXPOOL, OP_AVGPOOL, OP_BN_ACT = 1, 2, 3, 4, 5
OP_LAYERNORM, OP_ATTENTION, OP_TOKENS, OP_SELECT = 6, 7, 8, 9
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_BASE, ROPE_SCALE_PARTS = 0, 1, 2, 3

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32


class Thresholds(ctypes.Structure):
    _fields_ = [("s_thr", ctypes.c_double), ("c_thr", ctypes.c_double),
                ("intensity_mode", _I32), ("force_path", _I32)]


class Stats(ctypes.Structure):
    _fields_ = [("numel", ctypes.c_uint64), ("nnz", ctypes.c_uint64), ("sparsity", ctypes.c_double),
                ("flops", ctypes.c_uint64), ("macs_eq2", ctypes.c_uint64),
                ("input_bytes", ctypes.c_uint64), ("flops_per_byte", ctypes.c_double),
                ("B", _I32), ("C_in", _I32), ("H", _I32), ("W", _I32), ("path", _I32),
                ("reserved", _I32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_ if k != "reserved"}


class Occupancy(ctypes.Structure):
    _fields_ = [("nnz", _P), ("col_nnz", _P), ("tile_nnz", _P), ("row_bm", _P), ("blk_mask", _P),
                ("R", _I64), ("C", _I64), ("bytes", ctypes.c_uint64)]


class Epilogue(ctypes.Structure):
    _fields_ = [("bias", _P), ("bn", _P), ("bn_eps", ctypes.c_float), ("act", _I32),
                ("residual", _P)]


class Op(ctypes.Structure):
    _fields_ = [("kind", _I32), ("input", _I32), ("residual", _I32), ("c_in", _I32), ("c_out", _I32),
                ("kh", _I32), ("kw", _I32), ("stride", _I32), ("pad", _I32), ("groups", _I32),
                ("act", _I32), ("reserved", _I32), ("weight", _P), ("weight_kn", _P), ("bias", _P),
                ("bn", _P), ("bn_eps", ctypes.c_float), ("reserved2", ctypes.c_float),
                ("thr", Thresholds)]


class NormSpec(ctypes.Structure):
    _fields_ = [("kind", _I32), ("eps", ctypes.c_float), ("weight", _P), ("bias", _P)]


class KvCacheDesc(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("pages", _I64), ("page_size", _I32), ("kv_heads", _I32),
                ("head_dim", _I32), ("reserved", _I32)]


class PagedBatchDesc(ctypes.Structure):
    _fields_ = [("q_start", _P), ("kv_len", _P), ("table", _P), ("table_stride", _I64), ("batch", _I32),
                ("max_pages", _I32), ("max_q", _I32), ("reserved", _I32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("rot", _I32), ("layout", _I32), ("turns", _P), ("scale", ctypes.c_float), ("reserved", _I32)]


class ScoreRulesDesc(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("reserved", _I32), ("slopes", _P), ("prefix", _P), ("tree", _P)]


class W4Desc(ctypes.Structure):
    _fields_ = [("packed", _P), ("N", _I64), ("K", _I64), ("group", _I32), ("zeros", _I32)]


class LogitRulesDesc(ctypes.Structure):
    _fields_ = [("seen_start", _P), ("seen", _P), ("n_seen", _I64), ("penalties", _P), ("bias", _P), ("ld_bias", _I64),
                ("allowed", _P), ("ld_allowed", _I64)]


class Record(ctypes.Structure):
    _fields_ = [("stats", Stats), ("output", _P), ("out_shape", _I64 * 4),
                ("out_occ", ctypes.POINTER(Occupancy))]


def _sig(name, args):
    f = getattr(_lib, name)
    f.restype = ctypes.c_int
    f.argtypes = args
    return f


_sig("sparoa_create", [ctypes.POINTER(_P), ctypes.c_int, _P])
_sig("sparoa_destroy", [_P])
_sig("sparoa_set_stream", [_P, _P])
_sig("sparoa_set_overlap", [_P, _I32])
_sig("sparoa_graph_workspace", [_P, _P, _I32, _I64, _I64, _I64, _I64, ctypes.POINTER(ctypes.c_uint64)])
_sig("sparoa_gemm_split", [_P, _P, _I64, _I64, _P, _P, _I64, _P, ctypes.c_double, _P, _I32, _P, _P])
_sig("sparoa_sync", [_P])
_sig("sparoa_last_path", [_P, ctypes.POINTER(_I32)])
_sig("sparoa_set_wait_limit", [_P, ctypes.c_int64])
_sig("sparoa_set_fault", [_P, ctypes.c_int32])
_lib.sparoa_status_str.restype = ctypes.c_char_p
_lib.sparoa_status_str.argtypes = [ctypes.c_int]
_lib.sparoa_last_error.restype = ctypes.c_char_p
_lib.sparoa_last_error.argtypes = [_P]
_lib.sparoa_occupancy_bytes.restype = ctypes.c_uint64
_lib.sparoa_occupancy_bytes.argtypes = [_I64, _I64]
_sig("sparoa_occupancy_init", [_P, ctypes.c_uint64, _I64, _I64, ctypes.POINTER(Occupancy)])
_sig("sparoa_op_stats", [_P, _P, _I64, _I64, _I64, _I64, ctypes.POINTER(Op),
                         ctypes.POINTER(Occupancy), ctypes.POINTER(Stats)])
_sig("sparoa_gemm", [_P, _P, _I64, _I64, _P, _P, _I64, ctypes.POINTER(Epilogue),
                     ctypes.POINTER(Thresholds), _P, _I32, ctypes.POINTER(Occupancy),
                     ctypes.POINTER(Occupancy), ctypes.POINTER(Stats)])
_sig("sparoa_conv2d", [_P, _P, _I64, _I64, _I64, _I64, _P, _I64, _I32, _I32, _I32, _I32, _I32,
                       ctypes.POINTER(Epilogue), ctypes.POINTER(Thresholds), _P,
                       ctypes.POINTER(Occupancy), ctypes.POINTER(Occupancy), ctypes.POINTER(Stats)])
_sig("sparoa_maxpool2d", [_P, _P, _I64, _I64, _I64, _I64, _I32, _I32, _I32, _P,
                          ctypes.POINTER(Occupancy)])
_sig("sparoa_avgpool_global", [_P, _P, _I64, _I64, _I64, _I64, _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_bn_act", [_P, _P, _I64, _I64, ctypes.POINTER(Epilogue), _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_layernorm", [_P, _P, _I64, _I64, _P, ctypes.c_float, _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_attention", [_P, _P, _I64, _I64, _I32, _I32, _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_add_norm", [_P, _P, _P, _I64, _I64, _I32, ctypes.POINTER(NormSpec), _P, _I64, ctypes.c_float,
                         ctypes.POINTER(NormSpec), _P, _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_rope_turns", [_I32, ctypes.c_double, _I32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                           ctypes.c_double, _P])
_sig("sparoa_rope_append", [_P, _P, _I64, _I64, _I32, ctypes.POINTER(RopeDesc), _P, ctypes.POINTER(KvCacheDesc),
                            ctypes.POINTER(PagedBatchDesc), _P, _I64])
_sig("sparoa_paged_attention", [_P, _P, _I64, _I64, _I32, ctypes.c_float, _I32, _I32, ctypes.POINTER(KvCacheDesc),
                                ctypes.POINTER(PagedBatchDesc), _P, _P, ctypes.POINTER(Occupancy)])
_sig("sparoa_ruled_attention", [_P, _P, _I64, _I64, _I32, ctypes.c_float, _I32, _I32, ctypes.POINTER(ScoreRulesDesc),
                                ctypes.POINTER(KvCacheDesc), ctypes.POINTER(PagedBatchDesc), _P, _P, ctypes.POINTER(Occupancy)])
_lib.sparoa_w4_bytes.restype = ctypes.c_uint64
_lib.sparoa_w4_bytes.argtypes = [_I64, _I64, _I32, _I32]
_sig("sparoa_w4_pack", [_P, _P, _P, _P, _I64, _I64, _I32, _P])
_sig("sparoa_gemm_w4", [_P, _P, _I64, ctypes.POINTER(W4Desc), ctypes.POINTER(Epilogue), _P, _I32, ctypes.POINTER(Occupancy)])
_sig("sparoa_shape_logits", [_P, _P, _I64, _I64, _I64, _I32, ctypes.POINTER(LogitRulesDesc), _P, _I64, _P, _P])
_sig("sparoa_tree_accept", [_P, _P, _P, _P, _I64, ctypes.POINTER(KvCacheDesc), _I32, ctypes.POINTER(PagedBatchDesc), _P, _P,
                            _P, _P])
_sig("sparoa_run_graph", [_P, ctypes.POINTER(Op), _I32, _P, _I64, _I64, _I64, _I64, _P,
                          ctypes.c_uint64, ctypes.POINTER(Record)])
_sig("sparoa_gemm_noalloc", [_P, _P, _I64, _I64, _P, _P, _I64, ctypes.POINTER(Epilogue),
                             ctypes.POINTER(Thresholds), _P, _I32, ctypes.POINTER(Stats)])

EXPORTED = ["sparoa_create", "sparoa_destroy", "sparoa_set_stream", "sparoa_set_overlap", "sparoa_sync",
            "sparoa_last_path",
            "sparoa_set_wait_limit", "sparoa_set_fault",
            "sparoa_status_str", "sparoa_last_error", "sparoa_occupancy_bytes",
            "sparoa_occupancy_init", "sparoa_op_stats", "sparoa_gemm", "sparoa_conv2d",
            "sparoa_maxpool2d", "sparoa_avgpool_global", "sparoa_bn_act", "sparoa_run_graph",
            "sparoa_graph_workspace", "sparoa_gemm_split", "sparoa_layernorm", "sparoa_attention",
            "sparoa_add_norm", "sparoa_rope_turns", "sparoa_rope_append", "sparoa_paged_attention",
            "sparoa_ruled_attention", "sparoa_w4_bytes", "sparoa_w4_pack", "sparoa_gemm_w4", "sparoa_shape_logits", "sparoa_tree_accept",
            "sparoa_gemm_noalloc"]


class SparoaError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{_lib.sparoa_status_str(status).decode()}: {msg}")
        self.status = status


def _ptr(t):
    """Device address for a c_void_p argument or field (an int converts itself)."""
    return None if t is None else t.data_ptr()


# The raw handle of a device's current stream, without the Stream object that
# torch.cuda.current_stream builds around it.  Host time of a call on the Grace
# cores: 10.6 -> 4.5 us (BN + activation, one launch), 7.6 -> 5.6 us (GEMM, one
# launch); a chain of statistics, BN + ReLU and average pool 31.1 -> 20.1 us, which
# the GPU needs 21 us for.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)
_set_stream = _lib.sparoa_set_stream
_byref = ctypes.byref


def _rows(shape):
    """Product of all dimensions but the last."""
    r = 1
    for n in shape[:-1]:
        r *= n
    return r


def thresholds(s_thr=0.5, c_thr=32.0, intensity_mode=0, force_path=0) -> Thresholds:
    return Thresholds(float(s_thr), float(c_thr), int(intensity_mode), int(force_path))


class Context:
    """A libsparoa context on one device; calls follow the current torch stream."""

    def __init__(self, device: int = 0):
        self.device = device
        h = ctypes.c_void_p()
        with torch.cuda.device(device):
            st = _lib.sparoa_create(ctypes.byref(h), device,
                                    ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream))
        if st != OK:
            raise SparoaError(st, "sparoa_create")
        self.h = h
        self._stream = None  # the stream that the context was last set to

    def _check(self, st):
        if st != OK:
            raise SparoaError(st, _lib.sparoa_last_error(self.h).decode())

    def _bind(self):
        s = _raw_stream(self.device)
        if s != self._stream:  # (0.4 us of host time a call otherwise)
            st = _set_stream(self.h, s)
            if st != OK:
                self._check(st)
            self._stream = s

    def close(self):
        if getattr(self, "h", None):
            _lib.sparoa_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sync(self):
        self._check(_lib.sparoa_sync(self.h))

    def last_path(self) -> int:
        """The path the last sparoa_gemm / sparoa_conv2d call took (synchronises)."""
        p = _I32(0)
        self._check(_lib.sparoa_last_path(self.h, ctypes.byref(p)))
        return int(p.value)

    def set_overlap(self, enable: bool):
        """Programmatic dependent launch between consecutive kernels (default on)."""
        self._check(_lib.sparoa_set_overlap(self.h, 1 if enable else 0))

    def set_wait_limit(self, cycles: int):
        """SM cycles before a kernel's bounded wait gives up (0 = default)."""
        self._check(_lib.sparoa_set_wait_limit(self.h, int(cycles)))

    def set_fault(self, code: int):
        """Error-path tests: 1 = withhold the first accumulator signal
        (timeout), 2 = fail the next workspace allocation, 0 = off."""
        self._check(_lib.sparoa_set_fault(self.h, int(code)))


class OccupancyBuffer:
    """Device occupancy block of a [R, C] tensor (caller-owned torch storage)."""

    def __init__(self, R: int, C: int, device="cuda"):
        nbytes = int(_lib.sparoa_occupancy_bytes(R, C))
        self.buf = torch.zeros(max(nbytes, 16), dtype=torch.uint8, device=device)
        self.occ = Occupancy()
        st = _lib.sparoa_occupancy_init(ctypes.c_void_p(self.buf.data_ptr()), nbytes, R, C,
                                        ctypes.byref(self.occ))
        if st != OK:
            raise SparoaError(st, "sparoa_occupancy_init")
        self.R, self.C = R, C

    def to_host(self) -> dict:
        """Copy the block back: nnz, col_nnz, tile_nnz, row_bm, blk_mask (numpy)."""
        R, C = self.R, self.C
        T = (C + 63) // 64
        W64 = (T + 63) // 64
        RB = (R + 127) // 128
        C32 = (C + 31) // 32
        raw = self.buf.cpu().numpy()
        base = self.occ.nnz

        def view(ptr, dtype, n):
            off = ptr - base
            return raw[off:off + n * np.dtype(dtype).itemsize].view(dtype).copy()

        return {"nnz": int(view(self.occ.nnz, np.uint64, 1)[0]),
                "col_nnz": view(self.occ.col_nnz, np.uint32, C),
                "tile_nnz": view(self.occ.tile_nnz, np.uint32, T),
                "row_bm": view(self.occ.row_bm, np.uint64, R * W64).reshape(R, W64),
                "blk_mask": view(self.occ.blk_mask, np.uint32, RB * C32).reshape(RB, C32)}


def _occ(o):
    return None if o is None else _byref(o.occ)


def _epi(bias=None, bn=None, eps=1e-5, act=ACT_NONE, residual=None):
    return Epilogue(_ptr(bias), _ptr(bn), float(eps), int(act), _ptr(residual))


def sparoa_op_stats(ctx: Context, x, shape, consumer: Op | None = None, occ=None, host=True):
    """Eq. 1 statistics of x (NHWC shape (N, H, W, C) or (M, K))."""
    N, H, W, C = (shape[0], 1, 1, shape[1]) if len(shape) == 2 else shape
    ctx._bind()
    st = Stats() if host else None
    ctx._check(_lib.sparoa_op_stats(ctx.h, _ptr(x), N, H, W, C,
                                    _byref(consumer) if consumer is not None else None,
                                    _occ(occ), _byref(st) if host else None))
    return st


def sparoa_gemm(ctx: Context, x, W, y, W_kn=None, bias=None, bn=None, eps=1e-5, act=ACT_NONE,
                residual=None, thr: Thresholds | None = None, x_occ=None, y_occ=None, host=False):
    """y[M, N] = epilogue(x[M, K] W[N, K]^T) with threshold dispatch."""
    M, K = x.shape
    N = W.shape[0]
    ctx._bind()
    ep = _epi(bias, bn, eps, act, residual)
    st = Stats() if host else None
    ydt = F32 if y.dtype == torch.float32 else BF16
    ctx._check(_lib.sparoa_gemm(ctx.h, _ptr(x), M, K, _ptr(W), _ptr(W_kn), N, _byref(ep),
                                _byref(thr) if thr is not None else None, _ptr(y), ydt,
                                _occ(x_occ), _occ(y_occ), _byref(st) if host else None))
    return st


def sparoa_gemm_split(ctx: Context, x, W, y, xi, W_kn=None, bias=None, bn=None, eps=1e-5,
                      act=ACT_NONE, residual=None, x_occ=None, y_occ=None):
    """y = epilogue(x W^T) with rows [0, xi*M) (whole 128-row blocks) on the
    zero-skip kernel and the rest on the dense kernel, on two streams."""
    M, K = x.shape
    N = W.shape[0]
    ctx._bind()
    ep = _epi(bias, bn, eps, act, residual)
    ydt = F32 if y.dtype == torch.float32 else BF16
    ctx._check(_lib.sparoa_gemm_split(ctx.h, _ptr(x), M, K, _ptr(W), _ptr(W_kn), N, _byref(ep),
                                      float(xi), _ptr(y), ydt, _occ(x_occ), _occ(y_occ)))


def sparoa_conv2d(ctx: Context, x, w, y, stride=1, pad=0, groups=1, bias=None, bn=None, eps=1e-5,
                  act=ACT_NONE, residual=None, thr: Thresholds | None = None, x_occ=None,
                  y_occ=None, host=False):
    """NHWC conv: x [N, H, W, C_in], w [C_out, kh, kw, C_in/groups], y [N, Ho, Wo, C_out]."""
    N, H, Wd, Cin = x.shape
    Cout, kh, kw, _ = w.shape
    ctx._bind()
    ep = _epi(bias, bn, eps, act, residual)
    st = Stats() if host else None
    ctx._check(_lib.sparoa_conv2d(ctx.h, _ptr(x), N, H, Wd, Cin, _ptr(w), Cout, kh, kw, stride, pad,
                                  groups, _byref(ep),
                                  _byref(thr) if thr is not None else None, _ptr(y),
                                  _occ(x_occ), _occ(y_occ), _byref(st) if host else None))
    return st


def sparoa_maxpool2d(ctx: Context, x, y, k=3, stride=2, pad=1, y_occ=None):
    N, H, W, C = x.shape
    ctx._bind()
    ctx._check(_lib.sparoa_maxpool2d(ctx.h, _ptr(x), N, H, W, C, k, stride, pad, _ptr(y), _occ(y_occ)))


def sparoa_avgpool_global(ctx: Context, x, y, y_occ=None):
    N, H, W, C = x.shape
    ctx._bind()
    ctx._check(_lib.sparoa_avgpool_global(ctx.h, _ptr(x), N, H, W, C, _ptr(y), _occ(y_occ)))


def sparoa_bn_act(ctx: Context, x, y, bias=None, bn=None, eps=1e-5, act=ACT_NONE, residual=None,
                  y_occ=None):
    R = _rows(x.shape)
    C = x.shape[-1]
    ctx._bind()
    ep = _epi(bias, bn, eps, act, residual)
    ctx._check(_lib.sparoa_bn_act(ctx.h, _ptr(x), R, C, _byref(ep), _ptr(y), _occ(y_occ)))


def sparoa_layernorm(ctx: Context, x, y, gamma_beta=None, eps=1e-6, y_occ=None):
    """y = LN(x) over the last dimension; gamma_beta fp32 [2, C] or None."""
    R = _rows(x.shape)
    C = x.shape[-1]
    ctx._bind()
    ctx._check(_lib.sparoa_layernorm(ctx.h, _ptr(x), R, C, _ptr(gamma_beta), float(eps), _ptr(y),
                                     _occ(y_occ)))


def sparoa_attention(ctx: Context, qkv, y, heads, y_occ=None):
    """Multi-head self-attention: qkv [N, T, 3 D] (q | k | v per token), y [N, T, D]."""
    N, T, C3 = qkv.shape
    D = C3 // 3
    ctx._bind()
    ctx._check(_lib.sparoa_attention(ctx.h, _ptr(qkv), N, T, int(heads), D // int(heads), _ptr(y),
                                     _occ(y_occ)))


# ---------------------------------------------------------------------------
# decoder operators: residual norm, rotary positions into a paged cache, attention over it
# ---------------------------------------------------------------------------
def _refuse(what):
    raise SparoaError(ERR_INVALID_ARG, what)


def _want(cond, what):
    if not cond:
        _refuse(what)


def _want_rows(t, dtypes, what):
    """t is a CUDA tensor of one of `dtypes` with contiguous storage."""
    if not (t.is_cuda and t.dtype in dtypes and t.is_contiguous()):
        _refuse(f"{what}: contiguous CUDA tensor of {dtypes} wanted")


_bf16, _f32, _i32 = torch.bfloat16, torch.float32, torch.int32
_BF16S = (torch.bfloat16,)
_FP32S = (torch.float32,)
_I32S = (torch.int32,)


class Norm:
    """A norm of sparoa_add_norm; keeps its parameters alive."""

    def __init__(self, kind, weight=None, bias=None, eps=1e-6):
        for t in (weight, bias):
            if t is not None:
                _want_rows(t, _FP32S, "norm parameter")
        self.weight, self.bias = weight, bias
        sizes = {t.numel() for t in (weight, bias) if t is not None}
        _want(len(sizes) < 2, "norm parameters of different lengths")
        self.C = sizes.pop() if sizes else 0
        self.desc = NormSpec({"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}[kind], float(eps),
                             _ptr(weight), _ptr(bias))
        self.ref = _byref(self.desc)


def norm(kind, weight=None, bias=None, eps=1e-6) -> Norm:
    """kind "none", "rms" or "layer"; weight and bias fp32 [C] or None."""
    return Norm(kind, weight, bias, eps)


def sparoa_add_norm(ctx: Context, x, h, r=None, y=None, post: Norm | None = None, gate=None, rows_per_gate=0,
                    scale=1.0, pre: Norm | None = None, y_occ=None):
    """r = x + scale gate N_post(h), y = N_pre(r) over the last dimension; x and r bf16 or
    fp32, h and y bf16; any of x, h (not both) and r, y may be None."""
    lead = h if x is None else x
    if lead is None:
        _refuse("add_norm: x or h")
    C, n = lead.shape[-1], lead.numel()
    R = n // C if C else 0
    stream = r if x is None else x
    res = _f32 if stream is not None and stream.dtype is _f32 else _bf16
    if not ((x is None or (x.dtype is res and x.is_cuda and x.is_contiguous())) and
            (h is None or (h.dtype is _bf16 and h.is_cuda and h.is_contiguous() and h.numel() == n)) and
            (r is None or (r.dtype is res and r.is_cuda and r.is_contiguous() and r.numel() == n)) and
            (y is None or (y.dtype is _bf16 and y.is_cuda and y.is_contiguous() and y.numel() == n))):
        _refuse("add_norm: contiguous CUDA tensors of one size wanted: x and r of one type, h and y bf16")
    if (post is not None and post.C not in (0, C)) or (pre is not None and pre.C not in (0, C)):
        _refuse("add_norm: norm parameters of another length")
    if gate is not None:
        _want_rows(gate, _FP32S, "add_norm gate")
        if rows_per_gate < 0 or gate.numel() < (C if not rows_per_gate else -(-R // rows_per_gate) * C):
            _refuse("add_norm: gate rows")
    ctx._bind()
    st = _add_norm(ctx.h, None if x is None else x.data_ptr(), None if h is None else h.data_ptr(), R, C,
                   F32 if res is _f32 else BF16, None if post is None else post.ref, _ptr(gate), rows_per_gate, scale,
                   None if pre is None else pre.ref, None if r is None else r.data_ptr(),
                   None if y is None else y.data_ptr(), _occ(y_occ))
    if st:
        ctx._check(st)


class KVCache:
    """Key and value pools [pages, kv_heads, page_size, head_dim] (bf16, contiguous)."""

    def __init__(self, k, v):
        _want(k.dim() == 4 and k.shape == v.shape, "KVCache: pools [pages, kv_heads, page_size, head_dim]")
        for t in (k, v):
            _want_rows(t, _BF16S, "KVCache")
        self.k, self.v = k, v
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.desc = KvCacheDesc(_ptr(k), _ptr(v), self.pages, self.page_size, self.kv_heads, self.head_dim, 0)
        self.ref = _byref(self.desc)
        self.scale = self.head_dim ** -0.5

    @staticmethod
    def empty(pages, kv_heads, page_size, head_dim, device="cuda"):
        k, v = (torch.empty(pages, kv_heads, page_size, head_dim, dtype=torch.bfloat16, device=device) for _ in range(2))
        return KVCache(k, v)


class PagedBatch:
    """New tokens of a batch of sequences: q_start int32 [batch + 1], kv_len int32 [batch],
    table int32 [batch, max_pages] (rows may be strided), max_q the largest number of new tokens."""

    def __init__(self, q_start, kv_len, table, max_q):
        for t in (q_start, kv_len):
            _want_rows(t, _I32S, "PagedBatch")
        _want(table.is_cuda and table.dtype == torch.int32 and table.dim() == 2, "PagedBatch: table int32 [batch, pages]")
        B = kv_len.numel()
        _want(table.shape[0] == B and q_start.numel() == B + 1, "PagedBatch: lists of different batches")
        _want(table.shape[1] <= 1 or table.stride(1) == 1, "PagedBatch: strided table entries")
        self.q_start, self.kv_len, self.table, self.max_q = q_start, kv_len, table, int(max_q)
        self.desc = PagedBatchDesc(_ptr(q_start), _ptr(kv_len), _ptr(table),
                                   table.stride(0) if B > 1 else max(table.stride(0), table.shape[1]),
                                   B, table.shape[1], self.max_q, 0)
        self.ref = _byref(self.desc)


def sparoa_rope_turns(rot, base=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0) -> np.ndarray:
    """Turns per position of each rotated pair, in units of 2^-64 (uint64 [rot / 2], host)."""
    kinds = {"none": ROPE_SCALE_NONE, "linear": ROPE_SCALE_LINEAR, "base": ROPE_SCALE_BASE, "parts": ROPE_SCALE_PARTS}
    out = np.zeros(max(int(rot), 0) // 2, dtype=np.uint64)
    st = _lib.sparoa_rope_turns(int(rot), float(base), kinds[scaling], float(factor), float(context), float(low),
                                float(high), out.ctypes.data if out.size else None)
    if st != OK:
        raise SparoaError(st, "sparoa_rope_turns")
    return out


class Rope:
    """Rotary positions: `rot` leading values of a head, layout "half" or "interleaved",
    frequencies as sparoa_rope_turns, cos and sin times `scale`."""

    def __init__(self, rot, layout="half", base=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0,
                 scale=1.0, device="cuda"):
        turns = sparoa_rope_turns(rot, base, scaling, factor, context, low, high)
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.desc = RopeDesc(int(rot), {"half": ROPE_HALF, "interleaved": ROPE_INTERLEAVED}[layout],
                             _ptr(self.turns) if rot else None, float(scale), 0)
        self.ref = _byref(self.desc)


def _token_rows(t, T, D, what):
    """(row length, values of a row) of t [T, width] or [T, heads, D], bf16: rows may be
    strided, the values of a row are adjacent."""
    shape = t.shape
    if not (t.dtype is _bf16 and t.is_cuda and 2 <= len(shape) <= 3 and shape[0] == T):
        _refuse(f"{what}: bf16 rows of {T} tokens wanted")
    if len(shape) == 3 and shape[2] != D:
        _refuse(f"{what}: heads of {shape[2]} values over a cache of {D}")
    width = shape[1] if len(shape) == 2 else shape[1] * shape[2]
    if t.is_contiguous():
        return width, width
    st = t.stride()
    if (shape[-1] > 1 and st[-1] != 1) or (len(shape) == 3 and shape[1] > 1 and st[1] != shape[2]):
        _refuse(f"{what}: adjacent values in a row wanted")
    return (st[0] if T > 1 else max(st[0], width)), width


def sparoa_rope_append(ctx: Context, qkv, q_out, cache: KVCache, batch: PagedBatch, rope: Rope, positions=None):
    """Rotate the new tokens' queries (to q_out [T, heads, head_dim]) and keys (to the cache, with the
    values) from qkv [T, (heads + 2 kv_heads) head_dim]; rows may be strided."""
    T = qkv.shape[0]
    D = cache.head_dim
    ld, have = _token_rows(qkv, T, D, "rope_append qkv")
    ldq, width = _token_rows(q_out, T, D, "rope_append q_out")
    if width % D or have != width + 2 * cache.kv_heads * D:
        _refuse("rope_append: qkv rows hold heads, key heads and value heads; q_out rows the heads")
    if positions is not None:
        _want_rows(positions, _I32S, "rope_append positions")
        _want(positions.numel() == T, "rope_append: a position per token")
    ctx._bind()
    st = _rope_append(ctx.h, qkv.data_ptr(), ld, T, width // D, rope.ref, _ptr(positions), cache.ref, batch.ref,
                      q_out.data_ptr(), ldq)
    if st:
        ctx._check(st)


def _attention_rows(q, y, cache, lse, what):
    """Checks of q [T, heads, head_dim] and its results; (row length, T, heads)."""
    T, D = q.shape[0], cache.head_dim
    ld, width = _token_rows(q, T, D, what)
    if width % D or not (y.dtype is _bf16 and y.is_cuda and y.is_contiguous() and y.numel() == T * width):
        _refuse(f"{what}: q rows of whole heads, y of q's size")
    if lse is not None:
        _want_rows(lse, _FP32S, f"{what} lse")
        _want(lse.numel() == T * (width // D), f"{what}: lse")
    return ld, T, width // D


def sparoa_paged_attention(ctx: Context, q, y, cache: KVCache, batch: PagedBatch, scale=None, causal=True, window=0,
                           lse=None, y_occ=None):
    """y = softmax(scale q K^T) V of the new tokens over their cached sequences; q [T, heads, head_dim]
    (rows may be strided), y the same (contiguous), lse fp32 [T, heads] or None."""
    ld, T, heads = _attention_rows(q, y, cache, lse, "paged_attention")
    ctx._bind()
    st = _paged_attention(ctx.h, q.data_ptr(), ld, T, heads, cache.scale if scale is None else scale,
                          1 if causal else 0, window, cache.ref, batch.ref, y.data_ptr(), _ptr(lse), _occ(y_occ))
    if st:
        ctx._check(st)


class ScoreRules:
    """Rules of sparoa_ruled_attention; keeps its tensors alive.  cap: scores s become cap tanh(s / cap); slopes
    fp32 [heads]: less slope |distance|; prefix int32 [batch]: keys that every new token sees, within its window;
    tree int64 [T]: bits of each new token's ancestors among its sequence's new tokens."""

    def __init__(self, cap=0.0, slopes=None, prefix=None, tree=None):
        for t, types in ((slopes, _FP32S), (prefix, _I32S), (tree, (torch.int64,))):
            if t is not None:
                _want_rows(t, types, "ScoreRules")
        self.slopes, self.prefix, self.tree = slopes, prefix, tree
        self.desc = ScoreRulesDesc(float(cap), 0, _ptr(slopes), _ptr(prefix), _ptr(tree))
        self.ref = _byref(self.desc)


def sparoa_ruled_attention(ctx: Context, q, y, cache: KVCache, batch: PagedBatch, rules: ScoreRules, scale=None, causal=True,
                           window=0, lse=None, y_occ=None):
    """sparoa_paged_attention with score rules: a cap, a bias by distance, a prefix, a tree of drafted tokens."""
    ld, T, heads = _attention_rows(q, y, cache, lse, "ruled_attention")
    for t, n, what in ((rules.slopes, heads, "a slope per head"), (rules.prefix, batch.kv_len.numel(), "a prefix per sequence"),
                       (rules.tree, T, "ancestors of every new token")):
        if t is not None and t.numel() != n:
            _refuse(f"ruled_attention: {what} wanted")
    ctx._bind()
    st = _ruled_attention(ctx.h, q.data_ptr(), ld, T, heads, cache.scale if scale is None else scale, 1 if causal else 0, window,
                          rules.ref, cache.ref, batch.ref, y.data_ptr(), _ptr(lse), _occ(y_occ))
    if st:
        ctx._check(st)


_add_norm, _rope_append = _lib.sparoa_add_norm, _lib.sparoa_rope_append
_paged_attention, _ruled_attention = _lib.sparoa_paged_attention, _lib.sparoa_ruled_attention


# ---------------------------------------------------------------------------
# a step that checks drafted tokens: 4-bit products, logits to tokens, trees accepted
# ---------------------------------------------------------------------------
_U8S = (torch.uint8,)


def _w4_sizes(codes, scales, zeros):
    """(N, K, group, packed bytes) of 4-bit weights as W4 takes them."""
    _want_rows(codes, _U8S, "W4 codes")
    _want_rows(scales, _BF16S, "W4 scales")
    _want(codes.dim() == 2 and scales.dim() == 2 and codes.shape[0] == scales.shape[0], "W4: codes and scales of N rows")
    N, K, groups = codes.shape[0], 2 * codes.shape[1], scales.shape[1]
    _want(groups > 0 and K % groups == 0, "W4: a scale for every group of columns")
    if zeros is not None:
        _want_rows(zeros, _U8S, "W4 zeros")
        _want(zeros.shape == scales.shape, "W4: a zero for every scale")
    for t in (scales, zeros):
        _want(t is None or t.device == codes.device, "W4: tensors on one device")
    nbytes = int(_lib.sparoa_w4_bytes(N, K, K // groups, 0 if zeros is None else 1))
    _want(nbytes > 0, f"W4: [{N}, {K}] in groups of {K // groups}: N a multiple of 8, groups of 32, 64 or 128")
    return N, K, K // groups, nbytes


class W4:
    """Weights [N, K] of 4 bits: codes uint8 [N, K / 2] (column 2 i in the low half of byte i), scales bf16
    [N, K / group], zeros uint8 [N, K / group] or None (8).  Laid out for sparoa_gemm_w4 when it is made, on
    the current torch stream; holds a copy of its own."""

    def __init__(self, ctx: Context, codes, scales, zeros=None):
        self.N, self.K, self.group, nbytes = _w4_sizes(codes, scales, zeros)
        self.packed = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
        sparoa_w4_pack(ctx, codes, scales, zeros, self.packed)
        self.desc = W4Desc(_ptr(self.packed), self.N, self.K, self.group, 0 if zeros is None else 1)
        self.ref = _byref(self.desc)

    @staticmethod
    def quantise(ctx: Context, weight, group=128, zeros=False) -> "W4":
        """4-bit weights nearest to weight [N, K], by the range of each group (w4_quantise)."""
        return W4(ctx, *w4_quantise(weight, group, zeros))


def w4_quantise(weight, group=128, zeros=False):
    """(codes, scales, zeros or None) of weight [N, K], as W4 takes them."""
    N, K = weight.shape
    w = weight.float().view(N, K // group, group)
    lo, hi = w.amin(-1), w.amax(-1)
    if zeros:
        lo, hi = lo.clamp_max(0.0), hi.clamp_min(0.0)
        scales = ((hi - lo) / 15.0).to(torch.bfloat16)
    else:
        scales = torch.maximum(lo / -8.0, hi / 7.0).to(torch.bfloat16)
    step = scales.float()
    step = torch.where(step > 0, step, 1.0)
    zero = (-lo / step).round().clamp(0, 15) if zeros else torch.full_like(step, 8.0)
    c = ((w / step[..., None]).round() + zero[..., None]).clamp(0, 15).to(torch.uint8).view(N, K)
    return (c[:, 0::2] | c[:, 1::2] << 4).contiguous(), scales.contiguous(), zero.to(torch.uint8).contiguous() if zeros else None


def sparoa_w4_pack(ctx: Context, codes, scales, zeros, packed):
    """Lay out 4-bit weights (see W4) into packed, uint8 of sparoa_w4_bytes."""
    N, K, group, nbytes = _w4_sizes(codes, scales, zeros)
    _want_rows(packed, _U8S, "w4_pack packed")
    _want(packed.numel() == nbytes and packed.device == codes.device, f"w4_pack: packed of {nbytes} bytes beside the codes")
    ctx._bind()
    ctx._check(_lib.sparoa_w4_pack(ctx.h, _ptr(codes), _ptr(scales), _ptr(zeros), N, K, group, _ptr(packed)))


def sparoa_gemm_w4(ctx: Context, x, w: W4, y, bias=None, bn=None, eps=1e-5, act=ACT_NONE, residual=None, y_occ=None):
    """y[M, N] = epilogue(x[M, K] W^T) with 4-bit weights; x bf16, y bf16 or fp32."""
    M = x.numel() // w.K
    if not (x.is_cuda and x.dtype is _bf16 and x.is_contiguous() and x.shape[-1] == w.K):
        _refuse(f"gemm_w4: contiguous bf16 rows of {w.K} wanted")
    if not (y.is_cuda and y.dtype in (_bf16, _f32) and y.is_contiguous() and y.numel() == M * w.N):
        _refuse(f"gemm_w4: contiguous bf16 or fp32 y of [{M}, {w.N}] wanted")
    if bias is not None and not (bias.is_cuda and bias.dtype is _f32 and bias.is_contiguous() and bias.numel() == w.N):
        _refuse("gemm_w4: bias fp32 [N]")
    if bn is not None and not (bn.is_cuda and bn.dtype is _f32 and bn.is_contiguous() and bn.numel() == 4 * w.N):
        _refuse("gemm_w4: bn fp32 [4, N]")
    if residual is not None and not (residual.is_cuda and residual.dtype is _bf16 and residual.is_contiguous() and
                                     residual.numel() == M * w.N):
        _refuse("gemm_w4: residual bf16 of y's size")
    plain = act == ACT_NONE and bias is None and bn is None and residual is None
    ctx._bind()
    st = _gemm_w4(ctx.h, x.data_ptr(), M, w.ref, None if plain else _byref(_epi(bias, bn, eps, act, residual)), y.data_ptr(),
                  F32 if y.dtype is _f32 else BF16, _occ(y_occ))
    if st:
        ctx._check(st)


class LogitRules:
    """Changes of sparoa_shape_logits to logits [R, V]; keeps its tensors alive.  seen_start int32 [R + 1] and
    seen int32: the tokens that a row has seen; penalties fp32 [R, 4] (repetition, presence, frequency,
    temperature); bias fp32 [V], [1, V] or [R, V]; allowed int32 [R, words >= V / 32], bit v % 32 of word v / 32."""

    def __init__(self, seen_start=None, seen=None, penalties=None, bias=None, allowed=None):
        _want((seen_start is None) == (seen is None), "LogitRules: seen_start and seen go together")
        for t, types in ((seen_start, _I32S), (seen, _I32S), (penalties, _FP32S), (bias, _FP32S), (allowed, _I32S)):
            if t is not None:
                _want_rows(t, types, "LogitRules")
        _want(penalties is None or (penalties.dim() == 2 and penalties.shape[1] == 4), "LogitRules: penalties [R, 4]")
        _want(allowed is None or allowed.dim() == 2, "LogitRules: allowed [R, words]")
        _want(bias is None or bias.dim() in (1, 2), "LogitRules: bias [V] or [R, V]")
        self.keep = (seen_start, seen, penalties, bias, allowed)
        self.bias_rows = 1 if bias is None or bias.dim() == 1 else bias.shape[0]
        self.V = None if bias is None else bias.shape[-1]
        # rows that the rules are for, where they say
        rows = {n for n in (None if seen_start is None else seen_start.numel() - 1, None if penalties is None else penalties.shape[0],
                            None if allowed is None else allowed.shape[0], self.bias_rows if self.bias_rows != 1 else None)
                if n is not None}
        _want(len(rows) <= 1, "LogitRules: lists, penalties, bias and masks of as many rows")
        self.R = rows.pop() if rows else None
        self.words = None if allowed is None else allowed.shape[1]
        self.desc = LogitRulesDesc(_ptr(seen_start), _ptr(seen), 0 if seen is None else seen.numel(), _ptr(penalties), _ptr(bias),
                                   self.V if self.bias_rows != 1 else 0, _ptr(allowed), self.words or 0)
        self.ref = _byref(self.desc)


def _logit_rows(t, R, V, what):
    """Row length of t [R, V], whose rows may be strided."""
    if t.dim() != 2 or t.shape[0] != R or t.shape[1] != V or not t.is_cuda or (V > 1 and t.stride(1) != 1):
        _refuse(f"{what}: CUDA rows of {V} adjacent values wanted")
    return t.stride(0) if R > 1 else max(t.stride(0), V)


def sparoa_shape_logits(ctx: Context, logits, rules: LogitRules | None = None, y=None, best=None, lse=None):
    """The rules over logits [R, V] (bf16 or fp32): y fp32 [R, V] (may be the logits), best int32 [R], lse fp32
    [R], each of them or None."""
    if logits.dim() != 2 or logits.dtype not in (_bf16, _f32):
        _refuse("shape_logits: bf16 or fp32 logits [R, V]")
    R, V = logits.shape
    ld = _logit_rows(logits, R, V, "shape_logits logits")
    ld_y = 0
    if y is not None:
        if y.dtype is not _f32:
            _refuse("shape_logits: y fp32")
        ld_y = _logit_rows(y, R, V, "shape_logits y")
    if best is not None and not (best.dtype is _i32 and best.is_cuda and best.is_contiguous() and best.numel() == R):
        _refuse("shape_logits: best int32, a value per row")
    if lse is not None and not (lse.dtype is _f32 and lse.is_cuda and lse.is_contiguous() and lse.numel() == R):
        _refuse("shape_logits: lse fp32, a value per row")
    # (one row of bias is for all)
    if rules is not None and (rules.R not in (None, R) or rules.V not in (None, V) or (rules.words is not None and rules.words * 32 < V)):
        _refuse("shape_logits: rules of other rows or tokens")
    ctx._bind()
    st = _shape_logits(ctx.h, logits.data_ptr(), ld, R, V, F32 if logits.dtype is _f32 else BF16, None if rules is None else rules.ref,
                       _ptr(y), ld_y, _ptr(best), _ptr(lse))
    if st:
        ctx._check(st)


def sparoa_tree_accept(ctx: Context, tokens, best, tree, caches, batch: PagedBatch, path, count, following, new_len):
    """The path through each sequence's tree that the model's choices confirm; its keys and values move to the
    places that follow one another in all caches.  tokens, best, path int32 [T], tree int64 [T] (ancestor
    bits), count, following and new_len int32 [batch]."""
    T, B = tokens.numel(), batch.desc.batch
    for t in (tokens, best, path, count, following, new_len):
        if not (t.dtype is _i32 and t.is_cuda and t.is_contiguous()):
            _refuse("tree_accept: contiguous CUDA int32 lists wanted")
    if not (best.numel() == T == path.numel() and count.numel() == B == following.numel() == new_len.numel()):
        _refuse("tree_accept: lists of T or batch entries wanted")
    if not (tree.dtype is torch.int64 and tree.is_cuda and tree.is_contiguous() and tree.numel() == T):
        _refuse("tree_accept: ancestors int64 [T] wanted")
    descs = (KvCacheDesc * len(caches))(*[c.desc for c in caches])
    ctx._bind()
    st = _tree_accept(ctx.h, tokens.data_ptr(), best.data_ptr(), tree.data_ptr(), T, descs, len(caches), batch.ref,
                      path.data_ptr(), count.data_ptr(), following.data_ptr(), new_len.data_ptr())
    if st:
        ctx._check(st)


_gemm_w4, _shape_logits, _tree_accept = _lib.sparoa_gemm_w4, _lib.sparoa_shape_logits, _lib.sparoa_tree_accept


def sparoa_gemm_noalloc(x, W, y, W_kn=None, bias=None, bn=None, eps=1e-5, act=ACT_NONE,
                        residual=None, thr: Thresholds | None = None, host=False):
    """sparoa_gemm for callers that cannot allocate: no context, the input's
    occupancy lives in the library's static device array (see sparoa.h).
    Runs on the current torch stream of the current device."""
    M, K = x.shape
    N = W.shape[0]
    ep = _epi(bias, bn, eps, act, residual)
    st = Stats() if host else None
    ydt = F32 if y.dtype == torch.float32 else BF16
    rc = _lib.sparoa_gemm_noalloc(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream),
                                  _ptr(x), M, K, _ptr(W), _ptr(W_kn), N, _byref(ep),
                                  _byref(thr) if thr is not None else None, _ptr(y), ydt,
                                  _byref(st) if host else None)
    if rc != OK:
        raise SparoaError(rc, "sparoa_gemm_noalloc")
    return st


# ---------------------------------------------------------------------------
# graphs
# ---------------------------------------------------------------------------
_KIND = {"layernorm": OP_LAYERNORM, "attention": OP_ATTENTION, "tokens": OP_TOKENS, "select": OP_SELECT,
         "conv": OP_CONV2D, "fc": OP_FC, "maxpool": OP_MAXPOOL, "avgpool": OP_AVGPOOL,
         "bn_act": OP_BN_ACT}


def bits_to_device(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bf16 bit patterns (numpy) -> torch bf16 tensor on the device."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    return t.to(device)


def device_to_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Graph:
    """Operator list uploaded to the device, ready for sparoa_run_graph."""

    def __init__(self, ops: list, device="cuda"):
        self.keep = []
        arr = (Op * len(ops))()
        for i, d in enumerate(ops):
            o = arr[i]
            o.kind = _KIND[d["kind"]]
            o.input = d.get("input", i)
            r = d.get("residual", -1)
            o.residual = -1 if r is None else r
            o.act = d.get("act", ACT_NONE)
            o.groups = d.get("groups", 1)
            if d["kind"] in ("conv", "fc"):
                o.c_in, o.c_out = d["cin"], d["cout"]
                w = bits_to_device(d["w"], device)
                self.keep.append(w)
                o.weight = w.data_ptr()
                if d.get("w_kn") is not None:
                    wk = bits_to_device(d["w_kn"], device)
                    self.keep.append(wk)
                    o.weight_kn = wk.data_ptr()
            if d["kind"] == "conv":
                o.kh = o.kw = d["k"]
                o.stride, o.pad = d["stride"], d["pad"]
            elif d["kind"] == "maxpool":
                o.kh = o.kw = d["k"]
                o.stride, o.pad = d["stride"], d["pad"]
            elif d["kind"] == "layernorm":
                if d.get("gamma_beta") is not None:
                    t = torch.from_numpy(np.ascontiguousarray(d["gamma_beta"], dtype=np.float32)).to(device)
                    self.keep.append(t)
                    o.bn = t.data_ptr()
                o.bn_eps = d.get("eps", 1e-6)
            elif d["kind"] == "attention":
                o.groups = d["heads"]
            elif d["kind"] == "tokens":
                c = bits_to_device(d["cls"], device)
                pos = torch.from_numpy(np.ascontiguousarray(d["pos"], dtype=np.float32)).to(device)
                self.keep += [c, pos]
                o.weight = c.data_ptr()
                o.bias = pos.data_ptr()
            elif d["kind"] == "select":
                o.pad = d.get("index", 0)
            for name in ("bias", "bn"):
                if d.get(name) is not None:
                    t = torch.from_numpy(np.ascontiguousarray(d[name], dtype=np.float32)).to(device)
                    self.keep.append(t)
                    setattr(o, name, t.data_ptr())
            o.bn_eps = d.get("eps", 1e-5)
            thr = d.get("thr", {}) or {}
            o.thr = Thresholds(thr.get("s_thr", 0.5), thr.get("c_thr", 32.0),
                               thr.get("intensity_mode", 0), thr.get("force_path", 0))
        self.ops = arr
        self.n = len(ops)


def sparoa_graph_workspace(ctx: Context, graph: Graph, x_shape) -> int:
    """Bytes of device workspace sparoa_run_graph needs for this input shape."""
    N, H, W, C = (int(v) for v in x_shape)
    out = ctypes.c_uint64(0)
    ctx._check(_lib.sparoa_graph_workspace(ctx.h, graph.ops, graph.n, N, H, W, C, ctypes.byref(out)))
    return int(out.value)


def sparoa_run_graph(ctx: Context, graph: Graph, x, y=None, records=False):
    """Run the graph on x (bf16 NHWC); returns the list of Record (records=True) or None."""
    N, H, W, C = x.shape
    ctx._bind()
    recs = (Record * graph.n)() if records else None
    ctx._check(_lib.sparoa_run_graph(ctx.h, graph.ops, graph.n, _ptr(x), N, H, W, C, _ptr(y),
                                     0 if y is None else y.numel() * y.element_size(), recs))
    return list(recs) if records else None


class _DevView:
    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr,
                                         "data": (int(ptr), False), "version": 2}


def view_device(ptr: int, shape, dtype=torch.bfloat16) -> torch.Tensor:
    """A torch view (no copy) of device memory owned by the library, e.g. a
    graph record's output; valid only as long as the library keeps it."""
    if dtype == torch.bfloat16:
        t = torch.as_tensor(_DevView(ptr, shape, "<i2"), device="cuda")
        return t.view(torch.bfloat16)
    typestr = {torch.float32: "<f4", torch.int32: "<i4", torch.uint8: "|u1"}[dtype]
    return torch.as_tensor(_DevView(ptr, shape, typestr), device="cuda")


def record_occupancy(rec: Record) -> dict:
    """Copy a graph record's output occupancy to the host (same layout as
    OccupancyBuffer.to_host)."""
    o = rec.out_occ.contents
    R, C = o.R, o.C
    raw = view_device(o.nnz, (int(o.bytes),), torch.uint8).cpu().numpy()
    base = o.nnz
    T = (C + 63) // 64
    W64 = (T + 63) // 64
    RB = (R + 127) // 128
    C32 = (C + 31) // 32

    def view(ptr, dt, n):
        off = ptr - base
        return raw[off:off + n * np.dtype(dt).itemsize].view(dt).copy()

    return {"nnz": int(view(o.nnz, np.uint64, 1)[0]), "col_nnz": view(o.col_nnz, np.uint32, C),
            "tile_nnz": view(o.tile_nnz, np.uint32, T),
            "row_bm": view(o.row_bm, np.uint64, R * W64).reshape(R, W64),
            "blk_mask": view(o.blk_mask, np.uint32, RB * C32).reshape(RB, C32)}
