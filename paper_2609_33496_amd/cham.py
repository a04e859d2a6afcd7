"""Thin Python binding of the HIP library's C ABI (``include/chameleon.h``).

Argument marshalling only: torch tensors supply device memory and the current HIP stream;
every step of the computation runs in the library's kernels.  There is no fallback: if the
shared library is missing or a call fails, an exception is raised.

Functions keep the C names without the ``cham_`` prefix:
``select_weight_formats``, ``act_stats_reset``, ``act_stats_accumulate``,
``build_act_lut``, ``quantize_act``, ``quantize_act_lut``, ``mixed_linear``;
around 8-bit linear layers ``rms_norm_quantize``, ``gated_quantize`` (each with either of the
C functions for its output format), ``block_quantize_weights``, ``block_linear``;
attention: ``norm_rotate``, ``cache_write``, ``cache_read``, ``attention``, ``cache_attention``.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libchameleon.so")

# status codes
OK, EINVAL, ESHAPE, EFORMAT, EHIP, EWORKSPACE = 0, -1, -2, -3, -4, -5
# weight formats (palette order) and masks
W_INT8_SYM, W_INT8_ASYM, W_MXINT8, W_INT4_SYM, W_INT4_ASYM, W_NF4, W_FP4, W_MXINT4, W_MXFP4 = range(9)
W_NAMES = ["INT8-sym", "INT8-asym", "MXINT8", "INT4-sym", "INT4-asym", "NF4", "FP4", "MXINT4", "MXFP4"]
MASK_W4 = 0x1F0
MASK_W8 = 0x007
# activation formats (LUT codes)
A_INT8_ASYM, A_FP8_E4M3, A_FP8_E5M2, A_MXFP8, A_MXINT8 = range(5)
A_NAMES = ["INT8-asym", "FP8-E4M3", "FP8-E5M2", "MXFP8-E4M3", "MXINT8"]
# workspace ops
OP_SELECT, OP_STATS, OP_QUANT_ACT, OP_LINEAR, OP_GSELECT, OP_COLSQ = range(6)
GROUP_SIZES = (32, 64, 128, 192, 288)
GMASK_ALL = 0x1F
MASK_DIT_W4 = 0x070  # {INT4-asym, NF4, FP4}
SCHED_SCALED_LINEAR, SCHED_LINEAR = 0, 1

_P = ctypes.c_void_p


class _WQ(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("palette_mask", ctypes.c_uint32),
                ("code_bits", ctypes.c_int32), ("fmt", _P), ("codes", _P), ("scale", _P), ("zero", _P),
                ("nf4_absmax", _P), ("e8m0", _P), ("perm", _P), ("group_off", _P), ("err", _P), ("packed", _P)]


class _Stats(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("B", ctypes.c_int32), ("nS", _P), ("lohi", _P)]


class _Sched(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("beta0", ctypes.c_double), ("beta1", ctypes.c_double),
                ("kind", ctypes.c_int32), ("kappa_lo", ctypes.c_double), ("kappa_hi", ctypes.c_double),
                ("snr_lo", ctypes.c_double), ("snr_hi", ctypes.c_double), ("snr_gate_on", ctypes.c_int32)]


class _LUT(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("B", ctypes.c_int32), ("T", ctypes.c_int32), ("F", _P), ("S", _P),
                ("Z", _P)]


class _GWQ(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("palette_mask", ctypes.c_uint32),
                ("group_mask", ctypes.c_uint32), ("code_bits", ctypes.c_int32), ("choice", _P), ("fmt", _P),
                ("codes", _P), ("gscale", _P), ("gzero", _P), ("e8m0", _P), ("err", _P), ("packed", _P)]


class _AQ(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int64), ("fmt", ctypes.c_int32), ("nsamples", ctypes.c_int32),
                ("codes", _P), ("e8m0", _P), ("scale", _P), ("zero", _P)]


class _BQ(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int64), ("pow2", ctypes.c_int32), ("codes", _P), ("scale", _P)]


class _BW(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("pow2", ctypes.c_int32), ("codes", _P), ("scale", _P)]


class _Norm(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int64), ("x", _P), ("ldx", ctypes.c_int64), ("r", _P),
                ("ldr", ctypes.c_int64), ("h", _P), ("ldh", ctypes.c_int64), ("g", _P), ("x_type", ctypes.c_int32),
                ("r_type", ctypes.c_int32), ("g_type", ctypes.c_int32), ("eps", ctypes.c_float)]


class _Gate(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int64), ("x", _P), ("ldx", ctypes.c_int64), ("u", _P),
                ("ldu", ctypes.c_int64), ("type", ctypes.c_int32), ("act", ctypes.c_int32)]


class _Heads(ctypes.Structure):
    _fields_ = [("p", _P), ("token", ctypes.c_int64), ("head", ctypes.c_int64), ("H", ctypes.c_int32), ("type", ctypes.c_int32)]


class _Rotate(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("D", ctypes.c_int32), ("R", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("norm", ctypes.c_int32), ("eps", ctypes.c_float), ("amp", ctypes.c_float), ("qg", _P), ("kg", _P),
                ("qg_type", ctypes.c_int32), ("kg_type", ctypes.c_int32), ("pos", _P), ("freq", _P)]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("H", ctypes.c_int32), ("D", ctypes.c_int32), ("page", ctypes.c_int32),
                ("type", ctypes.c_int32), ("k", _P), ("v", _P), ("ks", _P), ("vs", _P)]


class _Attn(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("T", ctypes.c_int64), ("D", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float), ("pad", ctypes.c_int32), ("cu_q", _P), ("q", _Heads), ("o", _Heads)]


_lib = None


def lib():
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library {LIB_PATH} is not built; run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    L.cham_status_string.argtypes = [ctypes.c_int]
    L.cham_status_string.restype = ctypes.c_char_p
    L.cham_version.restype = ctypes.c_int
    L.cham_select_weight_formats.argtypes = [_P, ctypes.POINTER(_WQ), _P]
    L.cham_select_weight_formats_batch.argtypes = [ctypes.POINTER(_P), ctypes.POINTER(_WQ), i32, _P]
    L.cham_pack_weights_batch.argtypes = [ctypes.POINTER(_WQ), i32, _P]
    L.cham_act_stats_reset.argtypes = [ctypes.POINTER(_Stats), _P]
    L.cham_act_stats_accumulate.argtypes = [_P, i64, i32, i32, ctypes.POINTER(_Stats), _P, sz, _P]
    L.cham_act_stats_accumulate_batch.argtypes = [ctypes.POINTER(_P), ctypes.POINTER(i64), ctypes.POINTER(i32),
                                                  ctypes.POINTER(i32), i32, ctypes.POINTER(_Stats), _P, sz, _P]
    L.cham_schedule_default.argtypes = [ctypes.POINTER(_Sched)]
    L.cham_schedule_default.restype = None
    L.cham_build_act_lut.argtypes = [ctypes.POINTER(_Stats), ctypes.POINTER(_Sched), _P, ctypes.POINTER(_LUT), _P,
                                     _P]
    L.cham_bucket.argtypes = [i32, i32, i32]
    L.cham_bucket.restype = i32
    L.cham_quantize_act.argtypes = [_P, i32, i32, _P, _P, ctypes.POINTER(_AQ), _P, sz, _P]
    L.cham_quantize_act_lut.argtypes = [_P, ctypes.POINTER(_LUT), _P, i32, i32, i32, ctypes.POINTER(_AQ), _P, sz,
                                        _P]
    L.cham_quantize_act_noalloc.argtypes = [_P, i32, i32, _P, _P, ctypes.POINTER(_AQ), _P]
    L.cham_quantize_act_lut_accumulate_batch.argtypes = [ctypes.POINTER(_P), ctypes.POINTER(i32), i32, i32,
                                                         ctypes.POINTER(_LUT), _P, ctypes.POINTER(_AQ),
                                                         ctypes.POINTER(_Stats), _P, sz, _P]
    L.cham_mixed_linear.argtypes = [ctypes.POINTER(_AQ), ctypes.POINTER(_WQ), _P, _P, sz, _P]
    L.cham_mixed_linear_grouped.argtypes = [ctypes.POINTER(_AQ), ctypes.POINTER(_GWQ), _P, _P, sz, _P]
    L.cham_mixed_linear_workspace_query.argtypes = [ctypes.POINTER(_AQ), ctypes.POINTER(_WQ), ctypes.POINTER(sz)]
    L.cham_mixed_linear_grouped_workspace_query.argtypes = [ctypes.POINTER(_AQ), ctypes.POINTER(_GWQ),
                                                            ctypes.POINTER(sz)]
    L.cham_conv3x3_mixed.argtypes = [ctypes.POINTER(_AQ), i32, i32, i32, ctypes.POINTER(_WQ), _P, _P, sz, _P]
    L.cham_conv3x3_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    L.cham_conv3x3_workspace_bytes.restype = sz
    L.cham_select_group_formats.argtypes = [_P, _P, ctypes.POINTER(_GWQ), _P, sz, _P]
    L.cham_act_colsq_accumulate.argtypes = [_P, i64, i64, _P, _P, sz, _P]
    L.cham_workspace_bytes.argtypes = [i32, i64, i64, i64]
    L.cham_workspace_bytes.restype = sz
    L.cham_packed_bytes.argtypes = [i64, i64]
    L.cham_packed_bytes.restype = sz
    L.cham_linear_plan.argtypes = [i64, i64, i64, i32, ctypes.POINTER(ctypes.c_int32), i32]
    L.cham_rms_norm_quantize_block.argtypes = [ctypes.POINTER(_Norm), ctypes.POINTER(_BQ), _P]
    L.cham_rms_norm_quantize.argtypes = [ctypes.POINTER(_Norm), i32, ctypes.POINTER(_AQ), _P]
    L.cham_gated_quantize_block.argtypes = [ctypes.POINTER(_Gate), ctypes.POINTER(_BQ), _P]
    L.cham_gated_quantize.argtypes = [ctypes.POINTER(_Gate), i32, ctypes.POINTER(_AQ), _P]
    L.cham_block_quantize_weights.argtypes = [_P, i32, i64, ctypes.POINTER(_BW), _P]
    L.cham_block_linear.argtypes = [ctypes.POINTER(_BQ), ctypes.POINTER(_BW), _P, i32, i64, _P]
    L.cham_block_linear_plan.argtypes = [i64, i64, i64, i32, ctypes.POINTER(i32), i32]
    heads = ctypes.POINTER(_Heads)
    L.cham_norm_rotate.argtypes = [ctypes.POINTER(_Rotate), heads, heads, heads, heads, _P]
    L.cham_cache_write.argtypes = [ctypes.POINTER(_Cache), _P, ctypes.POINTER(_Rotate), heads, heads, heads, heads, _P]
    L.cham_cache_read.argtypes = [ctypes.POINTER(_Cache), _P, i64, _P, i64, i64, heads, heads, _P]
    L.cham_attention.argtypes = [ctypes.POINTER(_Attn), heads, heads, i64, _P, _P, sz, _P]
    L.cham_cache_attention.argtypes = [ctypes.POINTER(_Attn), ctypes.POINTER(_Cache), _P, i64, _P, _P, sz, _P]
    L.cham_attention_workspace_bytes.argtypes = [ctypes.POINTER(_Attn), i32]
    L.cham_attention_workspace_bytes.restype = sz
    for name in ("cham_norm_rotate", "cham_cache_write", "cham_cache_read", "cham_attention", "cham_cache_attention",
                 "cham_select_weight_formats", "cham_select_weight_formats_batch", "cham_pack_weights_batch",
                 "cham_act_stats_reset", "cham_act_stats_accumulate",
                 "cham_act_stats_accumulate_batch",
                 "cham_build_act_lut", "cham_quantize_act", "cham_quantize_act_lut", "cham_quantize_act_noalloc",
                 "cham_quantize_act_lut_accumulate_batch",
                 "cham_mixed_linear", "cham_mixed_linear_grouped", "cham_select_group_formats", "cham_conv3x3_mixed",
                 "cham_act_colsq_accumulate",
                 "cham_linear_plan", "cham_rms_norm_quantize_block", "cham_rms_norm_quantize",
                 "cham_gated_quantize_block", "cham_gated_quantize", "cham_block_quantize_weights",
                 "cham_block_linear", "cham_block_linear_plan"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


class ChamError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().cham_status_string(status).decode()} (status {status})")


def _check(rc: int, where: str):
    if rc != OK:
        raise ChamError(rc, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dev_tensor(t: torch.Tensor, dtype, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def workspace_bytes(op: int, M: int, N: int, K: int) -> int:
    return int(lib().cham_workspace_bytes(op, M, N, K))


def linear_plan(M: int, N: int, K: int, code_bits: int) -> dict:
    """The launch plan mixed_linear takes for these sizes (host only)."""
    out = (ctypes.c_int32 * 10)()
    _check(lib().cham_linear_plan(M, N, K, code_bits, out, 10), "cham_linear_plan")
    launches = [{"rows": (out[2 + 4 * i], out[3 + 4 * i]), "tile": (out[4 + 4 * i], out[5 + 4 * i])}
                for i in range(out[0])]
    return {"splits": out[1], "launches": launches}


def _exact_workspace(ws, device, query, a, w):
    """The caller's workspace, else one of the exact size the query reports for these
    operands (None when it is 0)."""
    if ws is not None:
        return ws, ws.numel()
    nb = ctypes.c_size_t(0)
    _check(query(ctypes.byref(a), ctypes.byref(w), ctypes.byref(nb)), "workspace query")
    if nb.value == 0:
        return None, 0
    return torch.empty(nb.value, dtype=torch.uint8, device=device), nb.value


def linear_workspace_query(xq: "AQ", wq: "WQ") -> int:
    """Exact workspace bytes mixed_linear needs for these operands (host only)."""
    a, w = xq.struct(), wq.struct()
    nb = ctypes.c_size_t(0)
    _check(lib().cham_mixed_linear_workspace_query(ctypes.byref(a), ctypes.byref(w), ctypes.byref(nb)),
           "cham_mixed_linear_workspace_query")
    return nb.value


def _workspace(op, M, N, K, device, ws):
    nb = workspace_bytes(op, M, N, K)
    if ws is not None:
        return ws, ws.numel()
    if nb == 0:
        return None, 0
    return torch.empty(nb, dtype=torch.uint8, device=device), nb


# -------------------------------------------------------------------------------------------
# weight search
# -------------------------------------------------------------------------------------------
def code_bits(mask: int) -> int:
    return 8 if mask & 0x7 else 4


@dataclass
class WQ:
    """Packed per-channel weights (device tensors, see cham_wq)."""
    N: int
    K: int
    mask: int
    code_bits: int
    fmt: torch.Tensor
    codes: torch.Tensor
    scale: torch.Tensor
    zero: torch.Tensor
    nf4_absmax: Optional[torch.Tensor]
    e8m0: Optional[torch.Tensor]
    perm: Optional[torch.Tensor]
    group_off: Optional[torch.Tensor]
    err: Optional[torch.Tensor]
    packed: Optional[torch.Tensor] = None  # GEMM-ready layout written by the search (cham_wq.packed)

    def struct(self) -> _WQ:
        return _WQ(self.N, self.K, self.mask, self.code_bits, _ptr(self.fmt), _ptr(self.codes), _ptr(self.scale),
                   _ptr(self.zero), _ptr(self.nf4_absmax), _ptr(self.e8m0), _ptr(self.perm), _ptr(self.group_off),
                   _ptr(self.err), _ptr(self.packed))


def packed_bytes(N: int, K: int) -> int:
    return int(lib().cham_packed_bytes(N, K))


def alloc_wq(N: int, K: int, mask: int, device="cuda", want_perm=True, want_err=False, want_packed=False) -> WQ:
    cb = code_bits(mask)
    u8, f32, i32 = torch.uint8, torch.float32, torch.int32
    nf4 = bool(mask >> W_NF4 & 1)
    mx = bool(mask & ((1 << W_MXINT8) | (1 << W_MXINT4) | (1 << W_MXFP4)))
    return WQ(N, K, mask, cb,
              fmt=torch.empty(N, dtype=u8, device=device),
              codes=torch.empty((N, K * cb // 8), dtype=u8, device=device),
              scale=torch.empty(N, dtype=f32, device=device),
              zero=torch.empty(N, dtype=torch.float32, device=device),
              nf4_absmax=torch.empty((N, K // 64), dtype=f32, device=device) if nf4 else None,
              e8m0=torch.empty((N, K // 32), dtype=u8, device=device) if mx else None,
              perm=torch.empty(N, dtype=i32, device=device) if want_perm else None,
              group_off=torch.empty(10, dtype=i32, device=device) if want_perm else None,
              err=torch.empty((N, 9), dtype=torch.float64, device=device) if want_err else None,
              packed=torch.empty(packed_bytes(N, K), dtype=u8, device=device) if want_packed else None)


def select_weight_formats(W: torch.Tensor, mask: int = MASK_W4, out: Optional[WQ] = None, want_perm=True,
                          want_err=False, want_packed=False, stream=None) -> WQ:
    """Per-output-channel format search of W [N, K] (fp32, device); with want_packed the
    search also writes the GEMM-ready layout that mixed_linear then uses."""
    _dev_tensor(W, torch.float32, "W")
    N, K = W.shape
    if out is None:
        out = alloc_wq(N, K, mask, W.device, want_perm, want_err, want_packed)
    st = out.struct()
    _check(lib().cham_select_weight_formats(_ptr(W), ctypes.byref(st), _stream(stream)), "select_weight_formats")
    out.code_bits = st.code_bits
    return out


class SearchBatch:
    """Prepared C arguments of a batched search over several layers (host arrays of the
    weight pointers and descriptors), reusable across calls."""

    def __init__(self, Ws, outs):
        assert len(Ws) == len(outs) and len(Ws) > 0
        for W in Ws:
            _dev_tensor(W, torch.float32, "W")
        self.Ws, self.outs = list(Ws), list(outs)
        self.ptrs = (_P * len(Ws))(*[W.data_ptr() for W in Ws])
        self.structs = (_WQ * len(outs))(*[o.struct() for o in outs])

    def run(self, stream=None):
        _check(lib().cham_select_weight_formats_batch(self.ptrs, self.structs, len(self.Ws), _stream(stream)),
               "select_weight_formats_batch")
        for o, st in zip(self.outs, self.structs):
            o.code_bits = st.code_bits


class PackBatch:
    """Prepared C arguments of the packing step on its own for several searched weights
    (their descriptors, each with a packed buffer), reusable across calls."""

    def __init__(self, wqs, packed):
        assert len(wqs) == len(packed) and len(wqs) > 0
        self.wqs = list(wqs)
        structs = []
        for w, buf in zip(wqs, packed):
            st = w.struct()
            st.packed = _ptr(buf)
            st.perm = st.group_off = st.err = None
            structs.append(st)
        self.packed = list(packed)
        self.structs = (_WQ * len(structs))(*structs)

    def run(self, stream=None):
        _check(lib().cham_pack_weights_batch(self.structs, len(self.wqs), _stream(stream)), "pack_weights_batch")


def pack_weights_batch(wqs, stream=None):
    """Write the packed layout of searched weights (each wq.packed set) on its own."""
    PackBatch(wqs, [w.packed for w in wqs]).run(stream)


def select_weight_formats_batch(Ws, mask: int = MASK_W4, outs=None, want_perm=True, want_err=False,
                                want_packed=False, stream=None):
    """Format search of several layers' weights (each [N_i, K_i] fp32, device) in one call."""
    if outs is None:
        outs = [alloc_wq(W.shape[0], W.shape[1], mask, W.device, want_perm, want_err, want_packed) for W in Ws]
    SearchBatch(Ws, outs).run(stream)
    return outs


# -------------------------------------------------------------------------------------------
# statistics and LUT
# -------------------------------------------------------------------------------------------
@dataclass
class Stats:
    L: int
    B: int
    nS: torch.Tensor    # [L*B, 5] f64
    lohi: torch.Tensor  # [L*B, 2] f32

    def struct(self):
        return _Stats(self.L, self.B, _ptr(self.nS), _ptr(self.lohi))


def alloc_stats(L: int, B: int, device="cuda") -> Stats:
    return Stats(L, B, torch.empty((L * B, 5), dtype=torch.float64, device=device),
                 torch.empty((L * B, 2), dtype=torch.float32, device=device))


def act_stats_reset(st: Stats, stream=None):
    s = st.struct()
    _check(lib().cham_act_stats_reset(ctypes.byref(s), _stream(stream)), "act_stats_reset")


class StatsBatch:
    """Prepared C arguments of a batched statistics accumulation (several layer inputs),
    reusable across calls with the same tensors."""

    def __init__(self, Xs, layers, buckets, st: Stats, ws=None):
        n = len(Xs)
        assert n > 0 and len(layers) == n and len(buckets) == n
        for X in Xs:
            _dev_tensor(X, torch.float32, "X")
        self.Xs, self.st = list(Xs), st
        self.ptrs = (_P * n)(*[X.data_ptr() for X in Xs])
        self.numel = (ctypes.c_int64 * n)(*[X.numel() for X in Xs])
        self.layer = (ctypes.c_int32 * n)(*layers)
        self.bucket = (ctypes.c_int32 * n)(*buckets)
        nb = sum(workspace_bytes(OP_STATS, X.numel(), 0, 0) for X in Xs)
        self.ws = ws if ws is not None else torch.empty(max(nb, 256), dtype=torch.uint8, device=Xs[0].device)
        self.ws_bytes = self.ws.numel()
        self.s = st.struct()

    def run(self, stream=None):
        _check(lib().cham_act_stats_accumulate_batch(self.ptrs, self.numel, self.layer, self.bucket, len(self.Xs),
                                                     ctypes.byref(self.s), _ptr(self.ws), self.ws_bytes,
                                                     _stream(stream)), "act_stats_accumulate_batch")


def act_stats_accumulate_batch(Xs, layers, buckets, st: Stats, stream=None):
    StatsBatch(Xs, layers, buckets, st).run(stream)


def act_stats_accumulate(X: torch.Tensor, layer: int, bucket: int, st: Stats, ws=None, stream=None):
    _dev_tensor(X, torch.float32, "X")
    n = X.numel()
    ws, nb = _workspace(OP_STATS, n, 0, 0, X.device, ws)
    s = st.struct()
    _check(lib().cham_act_stats_accumulate(_ptr(X), n, layer, bucket, ctypes.byref(s), _ptr(ws), nb,
                                           _stream(stream)), "act_stats_accumulate")


@dataclass
class Schedule:
    T: int = 1000
    beta0: float = 0.00085
    beta1: float = 0.012
    kind: int = SCHED_SCALED_LINEAR
    kappa_lo: float = 3.0
    kappa_hi: float = 5.0
    snr_lo: float = 0.2
    snr_hi: float = 2.0
    snr_gate_on: int = 1

    def struct(self):
        return _Sched(self.T, self.beta0, self.beta1, self.kind, self.kappa_lo, self.kappa_hi, self.snr_lo,
                      self.snr_hi, self.snr_gate_on)


@dataclass
class LUT:
    L: int
    B: int
    T: int
    F: torch.Tensor       # [L*B] u8 (device)
    S: torch.Tensor       # [L*B] f32
    Z: torch.Tensor       # [L*B] f32
    kappa: Optional[torch.Tensor] = None
    F_host: Optional[torch.Tensor] = None  # host mirror of F

    def struct(self):
        return _LUT(self.L, self.B, self.T, _ptr(self.F), _ptr(self.S), _ptr(self.Z))

    def mirror(self):
        """Copy F to the host once (after calibration); the per-step lookup then needs no sync."""
        self.F_host = self.F.cpu().contiguous()
        return self


def build_act_lut(st: Stats, sched: Optional[Schedule] = None, is_shortcut: Optional[torch.Tensor] = None,
                  want_kappa=True, out: Optional[LUT] = None, stream=None) -> LUT:
    sched = sched or Schedule()
    dev = st.nS.device
    n = st.L * st.B
    if out is None:
        out = LUT(st.L, st.B, sched.T, torch.empty(n, dtype=torch.uint8, device=dev),
                  torch.empty(n, dtype=torch.float32, device=dev), torch.empty(n, dtype=torch.float32, device=dev),
                  torch.empty(n, dtype=torch.float64, device=dev) if want_kappa else None)
    if is_shortcut is not None:
        _dev_tensor(is_shortcut, torch.uint8, "is_shortcut")
    s, sc, l = st.struct(), sched.struct(), out.struct()
    _check(lib().cham_build_act_lut(ctypes.byref(s), ctypes.byref(sc), _ptr(is_shortcut), ctypes.byref(l),
                                    _ptr(out.kappa), _stream(stream)), "build_act_lut")
    out.T = l.T
    return out


def bucket(t: int, T: int, B: int) -> int:
    return int(lib().cham_bucket(t, T, B))


# -------------------------------------------------------------------------------------------
# activation quantization
# -------------------------------------------------------------------------------------------
@dataclass
class AQ:
    M: int
    K: int
    fmt: int
    codes: torch.Tensor              # [M, K] u8
    e8m0: Optional[torch.Tensor]     # [M, K/32] u8
    scale: torch.Tensor              # [nsamples] f32
    zero: torch.Tensor               # [nsamples] f32
    nsamples: int = 1                # samples of M / nsamples consecutive rows

    def struct(self):
        return _AQ(self.M, self.K, self.fmt, self.nsamples, _ptr(self.codes), _ptr(self.e8m0), _ptr(self.scale),
                   _ptr(self.zero))


def alloc_aq(M: int, K: int, device="cuda", with_e8m0=True, nsamples: int = 1) -> AQ:
    return AQ(M, K, -1, torch.empty((M, K), dtype=torch.uint8, device=device),
              torch.empty((M, K // 32), dtype=torch.uint8, device=device) if with_e8m0 else None,
              torch.empty(nsamples, dtype=torch.float32, device=device),
              torch.empty(nsamples, dtype=torch.float32, device=device), nsamples)


def quantize_act(X: torch.Tensor, fmt: int, dynamic: bool = True, s: Optional[torch.Tensor] = None,
                 z: Optional[torch.Tensor] = None, out: Optional[AQ] = None, ws=None, stream=None,
                 nsamples: int = 1) -> AQ:
    """Quantize X [M, K]; static mode reads the scale/zero from device tensors s, z; dynamic
    mode takes each of the nsamples row blocks' own range (per-sample scaling)."""
    _dev_tensor(X, torch.float32, "X")
    M, K = X.shape
    if out is None:
        out = alloc_aq(M, K, X.device, nsamples=nsamples)
    ws, nb = _workspace(OP_QUANT_ACT, M, 0, K, X.device, ws)
    a = out.struct()
    _check(lib().cham_quantize_act(_ptr(X), fmt, int(dynamic), _ptr(s), _ptr(z), ctypes.byref(a), _ptr(ws), nb,
                                   _stream(stream)), "quantize_act")
    out.fmt = a.fmt
    return out


def quantize_act_noalloc(X: torch.Tensor, fmt: int, dynamic: bool, s: Optional[torch.Tensor], z: Optional[torch.Tensor],
                         out: AQ, stream=None) -> AQ:
    """cham_quantize_act_noalloc: the caller passes the output buffers; no workspace."""
    _dev_tensor(X, torch.float32, "X")
    a = out.struct()
    _check(lib().cham_quantize_act_noalloc(_ptr(X), fmt, int(dynamic), _ptr(s), _ptr(z), ctypes.byref(a),
                                           _stream(stream)), "quantize_act_noalloc")
    out.fmt = a.fmt
    return out


def quantize_act_lut(X: torch.Tensor, lut: LUT, layer: int, t: int, dynamic: bool = False,
                     out: Optional[AQ] = None, ws=None, stream=None, nsamples: int = 1) -> AQ:
    _dev_tensor(X, torch.float32, "X")
    if lut.F_host is None:
        lut.mirror()
    M, K = X.shape
    if out is None:
        out = alloc_aq(M, K, X.device, nsamples=nsamples)
    ws, nb = _workspace(OP_QUANT_ACT, M, 0, K, X.device, ws)
    a, l = out.struct(), lut.struct()
    _check(lib().cham_quantize_act_lut(_ptr(X), ctypes.byref(l), ctypes.c_void_p(lut.F_host.data_ptr()), layer, t,
                                       int(dynamic), ctypes.byref(a), _ptr(ws), nb, _stream(stream)),
           "quantize_act_lut")
    out.fmt = a.fmt
    return out


class QuantStatsBatch:
    """Prepared C arguments of a fused quantize-and-accumulate call: inputs Xs[i] of
    layers[i] quantized into outs[i] with the LUT's static scales at timestep t while their
    moments are added into st (reusable across calls with the same tensors)."""

    def __init__(self, Xs, layers, outs, lut: "LUT", st: Stats, ws=None):
        n = len(Xs)
        assert n > 0 and len(layers) == n and len(outs) == n
        for X, o in zip(Xs, outs):
            _dev_tensor(X, torch.float32, "X")
            assert X.shape == (o.M, o.K), "X and its AQ differ in shape"
        if lut.F_host is None:
            lut.mirror()
        self.Xs, self.outs, self.lut, self.st = list(Xs), list(outs), lut, st
        self.ptrs = (_P * n)(*[X.data_ptr() for X in Xs])
        self.layer = (ctypes.c_int32 * n)(*layers)
        self.aq = (_AQ * n)(*[o.struct() for o in outs])
        nb = sum(workspace_bytes(OP_STATS, X.numel(), 0, 0) for X in Xs)
        self.ws = ws if ws is not None else torch.empty(max(nb, 256), dtype=torch.uint8, device=Xs[0].device)
        self.ws_bytes = self.ws.numel()
        self.s = st.struct()
        self.l = lut.struct()

    def run(self, t: int, stream=None):
        _check(lib().cham_quantize_act_lut_accumulate_batch(
            self.ptrs, self.layer, len(self.Xs), t, ctypes.byref(self.l), ctypes.c_void_p(self.lut.F_host.data_ptr()),
            self.aq, ctypes.byref(self.s), _ptr(self.ws), self.ws_bytes, _stream(stream)),
            "quantize_act_lut_accumulate_batch")
        for o, a in zip(self.outs, self.aq):
            o.fmt = a.fmt


def quantize_act_lut_accumulate_batch(Xs, layers, t: int, lut: "LUT", st: Stats, outs=None, stream=None):
    """Quantize each Xs[i] as quantize_act_lut(Xs[i], lut, layers[i], t) does (static scales)
    and add its moments into st at (layers[i], bucket of t), in one pass; returns the AQs."""
    if outs is None:
        outs = [alloc_aq(X.shape[0], X.shape[1], X.device) for X in Xs]
    QuantStatsBatch(Xs, layers, outs, lut, st).run(t, stream)
    return outs


# -------------------------------------------------------------------------------------------
# DiT joint (group size, format) search (Sec. 4.6 (i))
# -------------------------------------------------------------------------------------------
@dataclass
class GWQ:
    """Group-scaled weights of one format (device tensors, see cham_gwq)."""
    N: int
    K: int
    mask: int
    gmask: int
    code_bits: int
    choice: torch.Tensor             # [2] i32: group size, format
    fmt: torch.Tensor
    codes: torch.Tensor
    gscale: torch.Tensor             # [N, K/32]
    gzero: torch.Tensor              # [N, K/32]
    e8m0: Optional[torch.Tensor]
    err: Optional[torch.Tensor]      # [45] f64
    packed: Optional[torch.Tensor] = None

    def struct(self) -> _GWQ:
        return _GWQ(self.N, self.K, self.mask, self.gmask, self.code_bits, _ptr(self.choice), _ptr(self.fmt),
                    _ptr(self.codes), _ptr(self.gscale), _ptr(self.gzero), _ptr(self.e8m0), _ptr(self.err),
                    _ptr(self.packed))


def alloc_gwq(N: int, K: int, mask: int, gmask: int = GMASK_ALL, device="cuda", want_err=True,
              want_packed=False) -> GWQ:
    cb = code_bits(mask)
    mx = bool(mask & ((1 << W_MXINT8) | (1 << W_MXINT4) | (1 << W_MXFP4)))
    f32 = torch.float32
    return GWQ(N, K, mask, gmask, cb, torch.zeros(2, dtype=torch.int32, device=device),
               torch.empty(N, dtype=torch.uint8, device=device),
               torch.empty((N, K * cb // 8), dtype=torch.uint8, device=device),
               torch.empty((N, K // 32), dtype=f32, device=device), torch.empty((N, K // 32), dtype=f32, device=device),
               torch.empty((N, K // 32), dtype=torch.uint8, device=device) if mx else None,
               torch.empty(45, dtype=torch.float64, device=device) if want_err else None,
               torch.empty(packed_bytes(N, K), dtype=torch.uint8, device=device) if want_packed else None)


def select_group_formats(W: torch.Tensor, energy: torch.Tensor, mask: int = MASK_DIT_W4, gmask: int = GMASK_ALL,
                         out: Optional[GWQ] = None, want_packed=False, ws=None, stream=None) -> GWQ:
    _dev_tensor(W, torch.float32, "W")
    _dev_tensor(energy, torch.float32, "energy")
    N, K = W.shape
    if out is None:
        out = alloc_gwq(N, K, mask, gmask, W.device, want_packed=want_packed)
    ws, nb = _workspace(OP_GSELECT, 0, N, K, W.device, ws)
    g = out.struct()
    _check(lib().cham_select_group_formats(_ptr(W), _ptr(energy), ctypes.byref(g), _ptr(ws), nb, _stream(stream)),
           "select_group_formats")
    out.code_bits = g.code_bits
    return out


def act_colsq_accumulate(X: torch.Tensor, colsq: torch.Tensor, ws=None, stream=None):
    """colsq[k] += sum_m X[m, k]^2 (binary64, fixed order)."""
    _dev_tensor(X, torch.float32, "X")
    _dev_tensor(colsq, torch.float64, "colsq")
    M, K = X.shape
    ws, nb = _workspace(OP_COLSQ, M, 0, K, X.device, ws)
    _check(lib().cham_act_colsq_accumulate(_ptr(X), M, K, _ptr(colsq), _ptr(ws), nb, _stream(stream)),
           "act_colsq_accumulate")


def mixed_linear_grouped(xq: "AQ", gq: GWQ, Y: Optional[torch.Tensor] = None, ws=None, stream=None) -> torch.Tensor:
    if Y is None:
        Y = torch.empty((xq.M, gq.N), dtype=torch.float32, device=xq.codes.device)
    _dev_tensor(Y, torch.float32, "Y")
    a, g = xq.struct(), gq.struct()
    ws, nb = _exact_workspace(ws, Y.device, lib().cham_mixed_linear_grouped_workspace_query, a, g)
    _check(lib().cham_mixed_linear_grouped(ctypes.byref(a), ctypes.byref(g), _ptr(Y), _ptr(ws), nb, _stream(stream)),
           "mixed_linear_grouped")
    return Y


# -------------------------------------------------------------------------------------------
# mixed-format linear layer
# -------------------------------------------------------------------------------------------
def mixed_linear(xq: AQ, wq: WQ, Y: Optional[torch.Tensor] = None, ws=None, stream=None) -> torch.Tensor:
    if Y is None:
        Y = torch.empty((xq.M, wq.N), dtype=torch.float32, device=xq.codes.device)
    _dev_tensor(Y, torch.float32, "Y")
    a, w = xq.struct(), wq.struct()
    ws, nb = _exact_workspace(ws, Y.device, lib().cham_mixed_linear_workspace_query, a, w)
    _check(lib().cham_mixed_linear(ctypes.byref(a), ctypes.byref(w), _ptr(Y), _ptr(ws), nb, _stream(stream)),
           "mixed_linear")
    return Y


def conv3x3_mixed(xq: AQ, B: int, H: int, W: int, wq: WQ, Y: Optional[torch.Tensor] = None, ws=None,
                  stream=None) -> torch.Tensor:
    """3x3 convolution (stride 1, zero padding 1) of channels-last activation codes xq
    (M = B H W rows, K = C) with weights wq [Co][9 C]; returns Y [B H W, Co]."""
    if Y is None:
        Y = torch.empty((xq.M, wq.N), dtype=torch.float32, device=xq.codes.device)
    _dev_tensor(Y, torch.float32, "Y")
    if ws is None:
        nb = int(lib().cham_conv3x3_workspace_bytes(B, H, W, xq.K, wq.N))
        ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=Y.device)
    a, w = xq.struct(), wq.struct()
    _check(lib().cham_conv3x3_mixed(ctypes.byref(a), B, H, W, ctypes.byref(w), _ptr(Y), _ptr(ws), ws.numel(),
                                    _stream(stream)), "conv3x3_mixed")
    return Y



# -------------------------------------------------------------------------------------------
# operators around 8-bit linear layers
# -------------------------------------------------------------------------------------------
BLOCK = 128
#: format of an operator's output besides the activation formats A_*: E4M3 codes with one scale
#: per row and 128 elements (a BQ, which block_linear reads)
A_BLOCK128 = 16
ACT_NONE, ACT_SILU, ACT_GELU, ACT_GELU_TANH = range(4)
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_EXACT = 256  # CHAM_T_EXACT


@dataclass
class BQ:
    """Activations in the block format (device tensors, see cham_bq).  scale: float32, or uint8
    where the scales are powers of two (exponent bytes)."""
    M: int
    K: int
    codes: torch.Tensor              # [M, K] u8
    scale: torch.Tensor              # [ceil(K / 128), M]

    def struct(self) -> _BQ:
        M, K, codes, scale = self.M, self.K, self.codes, self.scale
        return _BQ(M, K, _scales(scale, _cdiv(K, BLOCK), M, codes, M, K), codes.data_ptr(), scale.data_ptr())


@dataclass
class BW:
    """Weights in the block format (device tensors, see cham_bw)."""
    N: int
    K: int
    codes: torch.Tensor              # [N, K] u8
    scale: torch.Tensor              # [ceil(N / 128), ceil(K / 128)]

    def struct(self) -> _BW:
        N, K, codes, scale = self.N, self.K, self.codes, self.scale
        return _BW(N, K, _scales(scale, _cdiv(N, BLOCK), _cdiv(K, BLOCK), codes, N, K), codes.data_ptr(), scale.data_ptr())


def _cdiv(a: int, b: int) -> int:
    return -(-a // b)


def _scales(scale, rows, cols, codes, n, k) -> int:
    """Check a block-format pair of tensors; whether its scales are powers of two."""
    at = codes.get_device()  # negative on the host; cheaper than a comparison of device objects
    if at < 0 or codes.dtype is not torch.uint8 or codes.shape != (n, k) or not codes.is_contiguous():
        raise ValueError(f"codes must be a contiguous device uint8 [{n}, {k}]")
    pow2 = scale.dtype is torch.uint8
    if (not pow2 and scale.dtype is not torch.float32) or scale.shape != (rows, cols) or not scale.is_contiguous():
        raise ValueError(f"scale must be a contiguous float32 or uint8 [{rows}, {cols}]")
    if scale.get_device() != at:
        raise ValueError("codes and scale must be on one device")
    return int(pow2)


def _scale_type(pow2):
    return torch.uint8 if pow2 else torch.float32


def alloc_bq(M: int, K: int, device="cuda", pow2: bool = False) -> BQ:
    return BQ(M, K, torch.empty((M, K), dtype=torch.uint8, device=device),
              torch.empty((_cdiv(K, BLOCK), M), dtype=_scale_type(pow2), device=device))


def alloc_bw(N: int, K: int, device="cuda", pow2: bool = False) -> BW:
    return BW(N, K, torch.empty((N, K), dtype=torch.uint8, device=device),
              torch.empty((_cdiv(N, BLOCK), _cdiv(K, BLOCK)), dtype=_scale_type(pow2), device=device))


def _matrix(t: torch.Tensor, name: str, shape=None, device=None) -> int:
    """Check a [rows, columns] device tensor with unit column stride; its element type."""
    ty = _TYPES.get(t.dtype)
    if ty is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    if t.shape != shape if shape is not None else t.dim() != 2:
        raise ValueError(f"{name} must be a matrix" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    if t.get_device() != device.index if device is not None else not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor" + (f" on {device}" if device is not None else ""))
    if not t.is_contiguous() and t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"{name} must have unit stride along its columns")
    return ty


def _ld(t: torch.Tensor, rows: int, cols: int) -> int:
    """Row stride in elements; a single row's stride says nothing, so it counts as packed."""
    return t.stride(0) if rows > 1 else cols


# the current device and its current stream's handle, without the stream object that
# torch.cuda.current_stream makes (2 us of the host's time in front of a 3 us launch)
_device_now = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _on_device(dev, stream, call, *args):
    """call(*args, stream handle) with the tensors' device current."""
    if stream is None and dev.index == _device_now():
        return call(*args, _stream_now(dev.index))
    if stream is not None and stream.device != dev:
        raise ValueError(f"stream is on {stream.device}, the tensors on {dev}")
    with torch.cuda.device(dev):
        return call(*args, _stream_now(dev.index) if stream is None else stream.cuda_stream)


def _empty(rows, cols, dtype, dev, stream):
    """Memory of the launch stream's pool: that of another stream's may still be in use there."""
    if stream is None:
        return torch.empty(rows, cols, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(rows, cols, dtype=dtype, device=dev)


def _row_out(out, fmt, M, K, dev, pow2, stream):
    """The output of a row pass (the caller's, else a new one) and its C descriptor."""
    if fmt == A_BLOCK128:
        if out is None:
            out = BQ(M, K, _empty(M, K, torch.uint8, dev, stream), _empty(_cdiv(K, BLOCK), M, _scale_type(pow2), dev, stream))
            return out, _BQ(M, K, int(bool(pow2)), out.codes.data_ptr(), out.scale.data_ptr())
        if not isinstance(out, BQ) or (out.M, out.K) != (M, K) or out.codes.device != dev:
            raise ValueError(f"out must be a BQ of shape ({M}, {K}) on {dev}")
        if (out.scale.dtype is torch.uint8) != bool(pow2):
            raise ValueError("out's scales are not of the kind pow2 asks for")
        return out, out.struct()
    mx = fmt in (A_MXFP8, A_MXINT8)
    if out is None:
        out = AQ(M, K, fmt, _empty(M, K, torch.uint8, dev, stream), _empty(M, K // 32, torch.uint8, dev, stream) if mx else None,
                 *_empty(2, M, torch.float32, dev, stream).unbind(0), M)
        return out, out.struct()
    if not isinstance(out, AQ) or (out.M, out.K) != (M, K) or out.codes.device != dev:
        raise ValueError(f"out must be an AQ of shape ({M}, {K}) on {dev}")
    if out.codes.shape != (M, K) or out.codes.dtype is not torch.uint8 or not out.codes.is_contiguous():
        raise ValueError(f"out.codes must be a contiguous uint8 [{M}, {K}]")
    for t in (out.scale, out.zero):
        if t.shape != (M,) or t.dtype is not torch.float32 or not t.is_contiguous() or t.device != dev:
            raise ValueError(f"out.scale and out.zero must be contiguous float32 [{M}] (one scale per token)")
    if mx and (out.e8m0 is None or out.e8m0.shape != (M, K // 32) or out.e8m0.dtype is not torch.uint8 or
               not out.e8m0.is_contiguous() or out.e8m0.device != dev):
        raise ValueError(f"out.e8m0 must be a contiguous uint8 [{M}, {K // 32}]")
    return out, out.struct()


def rms_norm_quantize(X: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6, *,
                      residual: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None,
                      fmt: int = A_BLOCK128, pow2: bool = False, out=None, stream=None):
    """h = X + residual, y = h / sqrt(mean(h^2) + eps) * weight, in 8 bits: (BQ, h) for
    A_BLOCK128 (pow2: scales that are powers of two), else (AQ, h) with one scale per token.
    h has the residual's type (None without a residual); pass residual_out=residual to update
    it in place.  X, residual and residual_out [M, K] may have strided rows."""
    xt = _matrix(X, "X")
    M, K = X.shape
    dev = X.device
    rt = r_ptr = ldr = h_ptr = ldh = gt = g_ptr = 0
    if residual is not None:
        rt = _matrix(residual, "residual", X.shape, dev)
        r_ptr, ldr = residual.data_ptr(), _ld(residual, M, K)
        if residual_out is None:
            residual_out = _empty(M, K, residual.dtype, dev, stream)
            ldh = K
        elif _matrix(residual_out, "residual_out", X.shape, dev) != rt:
            raise ValueError("residual_out must have the residual's type")
        else:
            ldh = _ld(residual_out, M, K)
        h_ptr = residual_out.data_ptr()
    elif residual_out is not None:
        raise ValueError("residual_out needs a residual")
    if weight is not None:
        gt = _TYPES.get(weight.dtype, -1)
        if gt < 0 or weight.shape != (K,) or weight.device != dev or not weight.is_contiguous():
            raise ValueError(f"weight must be a contiguous float32, float16 or bfloat16 [{K}] on {dev}")
        g_ptr = weight.data_ptr()
    out, st = _row_out(out, fmt, M, K, dev, pow2, stream)
    n = _Norm(M, K, X.data_ptr(), _ld(X, M, K), r_ptr, ldr, h_ptr, ldh, g_ptr, xt, rt, gt, eps)
    if fmt == A_BLOCK128:
        rc = _on_device(dev, stream, lib().cham_rms_norm_quantize_block, ctypes.byref(n), ctypes.byref(st))
    else:
        rc = _on_device(dev, stream, lib().cham_rms_norm_quantize, ctypes.byref(n), fmt, ctypes.byref(st))
    _check(rc, "rms_norm_quantize")
    if fmt != A_BLOCK128:
        out.fmt, out.nsamples = fmt, M
    return out, residual_out


def gated_quantize(X: torch.Tensor, up: Optional[torch.Tensor] = None, act: int = ACT_SILU, *, fmt: int = A_BLOCK128,
                   pow2: bool = False, out=None, stream=None):
    """y = act(X) * up (up=None: act(X)) in 8 bits: a BQ for A_BLOCK128, else an AQ with one
    scale per token.  X and up [M, K] may have strided rows (the halves of one matrix)."""
    xt = _matrix(X, "X")
    M, K = X.shape
    dev = X.device
    u_ptr = ldu = 0
    if up is not None:
        if _matrix(up, "up", X.shape, dev) != xt:
            raise ValueError("X and up must have one type")
        u_ptr, ldu = up.data_ptr(), _ld(up, M, K)
    out, st = _row_out(out, fmt, M, K, dev, pow2, stream)
    g = _Gate(M, K, X.data_ptr(), _ld(X, M, K), u_ptr, ldu, xt, act)
    if fmt == A_BLOCK128:
        rc = _on_device(dev, stream, lib().cham_gated_quantize_block, ctypes.byref(g), ctypes.byref(st))
    else:
        rc = _on_device(dev, stream, lib().cham_gated_quantize, ctypes.byref(g), fmt, ctypes.byref(st))
    _check(rc, "gated_quantize")
    if fmt != A_BLOCK128:
        out.fmt, out.nsamples = fmt, M
    return out


def block_quantize_weights(W: torch.Tensor, pow2: bool = False, out: Optional[BW] = None, stream=None) -> BW:
    """W [N, K] (rows may be strided) in the block format: a scale for each 128 x 128 block."""
    ty = _matrix(W, "W")
    N, K = W.shape
    dev = W.device
    if out is None:
        out = BW(N, K, _empty(N, K, torch.uint8, dev, stream),
                 _empty(_cdiv(N, BLOCK), _cdiv(K, BLOCK), _scale_type(pow2), dev, stream))
        st = _BW(N, K, int(bool(pow2)), out.codes.data_ptr(), out.scale.data_ptr())
    elif (out.N, out.K) != (N, K) or out.codes.device != dev or (out.scale.dtype is torch.uint8) != bool(pow2):
        raise ValueError("out does not fit W and pow2")
    else:
        st = out.struct()
    rc = _on_device(dev, stream, lib().cham_block_quantize_weights, W.data_ptr(), ty, _ld(W, N, K), ctypes.byref(st))
    _check(rc, "block_quantize_weights")
    return out


def block_linear(xb: BQ, wb: BW, Y: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
                 stream=None, exact: bool = False) -> torch.Tensor:
    """Y [M, N] = activations times weights^T, both in the block format; Y (rows may be strided)
    decides the type where it is given, else dtype.  exact: a 16-bit Y from exact products too, as
    a float32 one always is, instead of the 8-bit matrix instructions' (see cham_block_linear)."""
    dev = xb.codes.device
    a, w = xb.struct(), wb.struct()
    if wb.codes.get_device() != dev.index:
        raise ValueError(f"the weights must be on {dev}")
    if Y is None:
        ty, ld = _TYPES.get(dtype), wb.N
        if ty is None:
            raise ValueError("dtype must be float32, float16 or bfloat16")
        Y = _empty(xb.M, ld, dtype, dev, stream)
    else:
        ty, ld = _matrix(Y, "Y", (xb.M, wb.N), dev), _ld(Y, xb.M, wb.N)
    if exact:
        ty |= _EXACT
    rc = _on_device(dev, stream, lib().cham_block_linear, ctypes.byref(a), ctypes.byref(w), Y.data_ptr(), ty, ld)
    _check(rc, "block_linear")
    return Y


def block_linear_plan(M: int, N: int, K: int, dtype: torch.dtype = torch.bfloat16, exact: bool = False) -> tuple:
    """(tile rows, tile channels, k groups) block_linear takes for these sizes (host only)."""
    out = (ctypes.c_int32 * 3)()
    _check(lib().cham_block_linear_plan(M, N, K, _TYPES[dtype] | (_EXACT if exact else 0), out, 3), "block_linear_plan")
    return tuple(out)


# -------------------------------------------------------------------------------------------
# attention
# -------------------------------------------------------------------------------------------
ROT_HALF, ROT_PAIRS = range(2)
_E4M3 = 3  # CHAM_T_E4M3
_CACHE_TYPES = {torch.float16: 1, torch.bfloat16: 2, torch.float8_e4m3fn: _E4M3}
_NO_HEADS = _Heads()


def _heads(t: torch.Tensor, name: str, T: int, D: int, dev, ty: int, H: int = -1) -> _Heads:
    """Check rows of heads [T, H, D] of type ty on dev, any strides along tokens and heads."""
    if t.get_device() != dev.index:  # negative on the host
        raise ValueError(f"{name} must be a device tensor on {dev}")
    if _TYPES.get(t.dtype) != ty:
        raise ValueError(f"{name} is of type {t.dtype}, which does not fit the others")
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name} must be of shape (tokens, heads, D), got {tuple(shape)}")
    n, h, d = shape
    if n != T or d != D or (H >= 0 and h != H):
        raise ValueError(f"{name} must be of shape ({T}, {H if H >= 0 else 'heads'}, {D}), got {tuple(shape)}")
    token, head, one = t.stride()
    if one != 1 and D > 1:
        raise ValueError(f"{name} must have unit stride along a head's elements")
    return _Heads(t.data_ptr(), token, head, h, ty)


def _float_type(t: torch.Tensor, name: str) -> int:
    ty = _TYPES.get(t.dtype)
    if ty is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    return ty


def _vector(t: torch.Tensor, name: str, n: int, dtype, dev) -> int:
    """Check a contiguous device vector; its address."""
    if t.get_device() != dev.index or t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} [{n}] on {dev}")
    return t.data_ptr()


def _empty_heads(T, H, D, dtype, dev, stream):
    if stream is None:
        return torch.empty(T, H, D, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(T, H, D, dtype=dtype, device=dev)


class Cache:
    """Pages of keys and values (device tensors, see cham_cache): k, v [pages, heads, page, D] in
    float16, bfloat16 or float8_e4m3fn, the last with float32 scales k_scale, v_scale [pages, heads, page]."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "pages", "H", "page", "D", "device", "_struct")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        ty, at, shape = _CACHE_TYPES.get(k.dtype), k.get_device(), k.shape
        if ty is None or v.dtype is not k.dtype:
            raise ValueError("k and v must both be float16, bfloat16 or float8_e4m3fn")
        if len(shape) != 4 or v.shape != shape:
            raise ValueError("k and v must be of one shape [pages, heads, page, D]")
        if at < 0 or v.get_device() != at or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("k and v must be contiguous device tensors on one device")
        ks = vs = None
        if ty == _E4M3:
            for t in (k_scale, v_scale):
                if (t is None or t.dtype is not torch.float32 or t.shape != shape[:3] or t.get_device() != at or
                        not t.is_contiguous()):
                    raise ValueError(f"an 8-bit cache needs contiguous float32 scales of shape {tuple(shape[:3])} beside it")
            ks, vs = k_scale.data_ptr(), v_scale.data_ptr()
        elif k_scale is not None or v_scale is not None:
            raise ValueError("a 16-bit cache has no scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.H, self.page, self.D = shape
        self.device = k.device
        self._struct = _Cache(shape[0], shape[1], shape[3], shape[2], ty, k.data_ptr(), v.data_ptr(), ks, vs)


def alloc_cache(pages: int, H: int, page: int, D: int, dtype: torch.dtype = torch.float8_e4m3fn, device="cuda") -> Cache:
    """A cache of `pages` pages of `page` tokens (a power of two, 16 and more) and H heads; its
    memory is not initialized."""
    k = torch.empty((2, pages, H, page, D), dtype=dtype, device=device)
    if dtype is not torch.float8_e4m3fn:
        return Cache(k[0], k[1])
    s = torch.empty((2, pages, H, page), dtype=torch.float32, device=device)
    return Cache(k[0], k[1], s[0], s[1])


def _rotate(T, D, dev, q_weight, k_weight, eps, norm, positions, freq, layout, amp) -> _Rotate:
    w = [0, 0, 0, 0]
    for i, (t, name) in enumerate(((q_weight, "q_weight"), (k_weight, "k_weight"))):
        if t is not None:
            if not norm:
                raise ValueError(f"{name} is a weight of the norm, which norm=False leaves out")
            w[2 + i] = _float_type(t, name)
            w[i] = _vector(t, name, D, t.dtype, dev)
    R = pos = fr = 0
    if (positions is None) != (freq is None):
        raise ValueError("a rotation needs positions and freq")
    if freq is not None:
        R = 2 * freq.numel()
        pos, fr = _vector(positions, "positions", T, torch.int32, dev), _vector(freq, "freq", R // 2, torch.float64, dev)
    return _Rotate(T, D, R, layout, int(bool(norm)), eps, amp, w[0] or None, w[1] or None, w[2], w[3], pos or None, fr or None)


def norm_rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], *, q_weight: Optional[torch.Tensor] = None,
                k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, norm: bool = True,
                positions: Optional[torch.Tensor] = None, freq: Optional[torch.Tensor] = None, layout: int = ROT_HALF,
                amp: float = 1.0, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """(q', k'): each head x / sqrt(mean(x^2) + eps) * weight (norm=False: as it is), then its first
    2 len(freq) elements turned by positions[t] * freq[i] and scaled by amp; layout ROT_HALF turns
    element i with i + len(freq), ROT_PAIRS 2i with 2i + 1.  q [T, Hq, D] and k [T, Hk, D] (slices of one
    matrix, or None) of one type; positions int32 [T], freq float64 [at most D / 2].  q_out=q and
    k_out=k work in place."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k must be given")
    if x.dim() != 3:
        raise ValueError("q and k must be of shape (tokens, heads, D)")
    T, _, D = x.shape
    dev, ty = x.device, _float_type(x, "q and k")
    r = _rotate(T, D, dev, q_weight, k_weight, eps, norm, positions, freq, layout, amp)
    st = []
    outs = [q_out, k_out]
    for i, (t, name) in enumerate(((q, "q"), (k, "k"))):
        if t is None:
            if outs[i] is not None:
                raise ValueError(f"{name}_out without {name}")
            st += [_Heads(None, 0, 0, 0, ty)] * 2
            continue
        s = _heads(t, name, T, D, dev, ty)
        if outs[i] is None:
            H = s.H
            outs[i] = o = _empty_heads(T, H, D, t.dtype, dev, stream)
            st += [s, _Heads(o.data_ptr(), H * D, D, H, ty)]
        else:
            st += [s, _heads(outs[i], name + "_out", T, D, dev, ty, s.H)]
    rc = _on_device(dev, stream, lib().cham_norm_rotate, r, st[0], st[1], st[2], st[3])
    _check(rc, "norm_rotate")
    return outs


def cache_write(cache: Cache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None, *,
                q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                norm: bool = True, positions: Optional[torch.Tensor] = None, freq: Optional[torch.Tensor] = None,
                layout: int = ROT_HALF, amp: float = 1.0, q_out: Optional[torch.Tensor] = None, stream=None):
    """Keys (normed and turned as norm_rotate does) and values (as they are) of token t written to slot
    slots[t] = page index * page + place of the cache; a slot outside it (-1) takes none, and no two
    tokens may have one slot.  Returns q normed and turned in the same pass (None without q)."""
    if k.dim() != 3:
        raise ValueError("k must be of shape (tokens, heads, D)")
    T, H, D = k.shape
    dev, ty = k.device, _float_type(k, "k")
    if cache.device != dev or (H, D) != (cache.H, cache.D):
        raise ValueError(f"the cache holds {cache.H} heads of {cache.D} on {cache.device}")
    r = _rotate(T, D, dev, q_weight, k_weight, eps, norm, positions, freq, layout, amp)
    ks, vs = _heads(k, "k", T, D, dev, ty), _heads(v, "v", T, D, dev, ty, H)
    at = _vector(slots, "slots", T, torch.int32, dev)
    qs = os = None
    if q is not None:
        qs = _heads(q, "q", T, D, dev, ty)
        if q_out is None:
            q_out = _empty_heads(T, qs.H, D, q.dtype, dev, stream)
        os = _heads(q_out, "q_out", T, D, dev, ty, qs.H)
    elif q_out is not None:
        raise ValueError("q_out without q")
    elif q_weight is not None:
        raise ValueError("q_weight without q")
    _check(_on_device(dev, stream, lib().cham_cache_write, cache._struct, at, r, ks, vs, qs, os), "cache_write")
    return q_out


def _table(table: torch.Tensor, B: int, dev) -> int:
    if table.dim() != 2 or table.shape[0] != B or table.dtype is not torch.int32 or table.get_device() != dev.index or \
            not table.is_contiguous():
        raise ValueError(f"table must be a contiguous int32 [{B}, pages of a sequence] on {dev}")
    return table.data_ptr()


def cache_read(cache: Cache, table: torch.Tensor, cu: torch.Tensor, total: int, *, dtype: torch.dtype = torch.bfloat16,
               k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None, stream=None):
    """(k, v) [total, heads, D]: rows cu[b] .. cu[b + 1] hold the tokens of sequence b, whose pages
    are table[b] (int32 [B, pages], cu int32 [B + 1] on the device).  Rows from cu[B] on are left as they are
    (of new tensors: undefined); tokens without a page come back as zeros."""
    dev, D, H = cache.device, cache.D, cache.H
    if (k_out is None) != (v_out is None):
        raise ValueError("k_out and v_out go together")
    if k_out is None:
        ty = _TYPES.get(dtype)
        if ty is None:
            raise ValueError("dtype must be float32, float16 or bfloat16")
        if total < 0:
            raise ValueError("total must not be negative")
        k_out, v_out = _empty_heads(total, H, D, dtype, dev, stream), _empty_heads(total, H, D, dtype, dev, stream)
    else:
        ty = _float_type(k_out, "k_out")
    ko, vo = _heads(k_out, "k_out", total, D, dev, ty, H), _heads(v_out, "v_out", total, D, dev, ty, H)
    if cu.dim() != 1 or cu.shape[0] < 1:
        raise ValueError("cu must hold a start for each sequence and the end")
    B = cu.shape[0] - 1
    c, t = _vector(cu, "cu", B + 1, torch.int32, dev), _table(table, B, dev)
    _check(_on_device(dev, stream, lib().cham_cache_read, cache._struct, t, table.shape[1], c, B, total, ko, vo), "cache_read")
    return k_out, v_out


_NO_WS, _NO_WS_ONE = 256, 1024  # CHAM_ATTN_NO_WS, CHAM_ATTN_NO_WS_ONE


def _attn(q, B, cu_q, causal, scale, out, Hk, need_ws, ws, stream):
    """The descriptor, output and workspace of an attention call."""
    if q.dim() != 3:
        raise ValueError("q must be of shape (tokens, heads, D)")
    T, Hq, D = q.shape
    dev, ty = q.device, _float_type(q, "q")
    if ty == 0:
        raise ValueError("q must be float16 or bfloat16")
    if Hk < 1 or Hq % Hk != 0:
        raise ValueError(f"{Hq} query heads cannot share {Hk} key heads")
    qs = _heads(q, "q", T, D, dev, ty)
    if out is None:
        out = _empty_heads(T, Hq, D, q.dtype, dev, stream)
        os = _Heads(out.data_ptr(), Hq * D, D, Hq, ty)
    else:
        os = _heads(out, "out", T, D, dev, ty, Hq)
    cu = None if cu_q is None else _vector(cu_q, "cu_q", B + 1, torch.int32, dev)
    a = _Attn(B, T, D, int(bool(causal)), D ** -0.5 if scale is None else scale, 0, cu, qs, os)
    if ws is None:
        if not need_ws:
            return a, out, dev, None, 0
        ws = _empty(1, attention_workspace_bytes(D, dev), torch.uint8, dev, stream)
    elif ws.get_device() != dev.index or ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    return a, out, dev, ws.data_ptr(), ws.numel()


_attn_ws = {}


def attention_workspace_bytes(D: int, device="cuda") -> int:
    """Workspace bytes of attention and cache_attention for heads of D on a device."""
    dev = device if isinstance(device, torch.device) else torch.device(device)
    key = (D, dev.index if dev.index is not None else _device_now())
    n = _attn_ws.get(key)
    if n is None:
        h = _Heads(None, 0, 0, 1, 2)
        with torch.cuda.device(key[1]):
            n = lib().cham_attention_workspace_bytes(_Attn(0, 0, D, 0, 1.0, 0, None, h, h), 1)
        _attn_ws[key] = n
    return n


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, batch: Optional[int] = None,
              cu_q: Optional[torch.Tensor] = None, cu_k: Optional[torch.Tensor] = None, causal: bool = False,
              scale: Optional[float] = None, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """softmax(scale q k^T) v of packed sequences: q [Tq, Hq, D], k and v [Tk, Hk, D], float16 or bfloat16,
    Hq a multiple of Hk; scale: D^-0.5 if None.  Sequences: `batch` (1 if None) of equal lengths, or rows
    cu_q[b] .. cu_q[b + 1] of q with cu_k[b] .. cu_k[b + 1] of k (int32 [B + 1] on the device; cu_k: cu_q if None).
    causal is aligned at the sequences' ends: the last query sees every key.  A query that sees none
    gets zeros; rows from cu_q[B] on are left as they are (of a new tensor: undefined)."""
    if cu_q is None:
        if cu_k is not None:
            raise ValueError("cu_k needs cu_q")
        B = 1 if batch is None else batch
        if B < 1 or q.shape[0] % B or k.shape[0] % B:
            raise ValueError(f"{q.shape[0]} queries and {k.shape[0]} keys are not {B} sequences of equal lengths")
    else:
        if batch is not None:
            raise ValueError("give batch or cu_q")
        if cu_q.dim() != 1 or cu_q.shape[0] < 1:
            raise ValueError("cu_q must hold a start for each sequence and the end")
        B = cu_q.shape[0] - 1
        if cu_k is None:
            cu_k = cu_q
    if k.dim() != 3:
        raise ValueError("k and v must be of shape (tokens, heads, D)")
    Tk = k.shape[0]
    a, out, dev, space, nb = _attn(q, B, cu_q, causal, scale, out, k.shape[1], Tk > _NO_WS, ws, stream)
    ty = a.q.type
    ks, vs = _heads(k, "k", Tk, a.D, dev, ty), _heads(v, "v", Tk, a.D, dev, ty, k.shape[1])
    cu = None if cu_k is None else _vector(cu_k, "cu_k", B + 1, torch.int32, dev)
    _check(_on_device(dev, stream, lib().cham_attention, a, ks, vs, Tk, cu, space, nb), "attention")
    return out


def cache_attention(q: torch.Tensor, cache: Cache, table: torch.Tensor, lens: torch.Tensor,
                    cu_q: Optional[torch.Tensor] = None, *, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of each sequence's newest tokens over its tokens in the cache, causal: q [T, Hq, D] holds
    one token of each sequence (cu_q None) or rows cu_q[b] .. cu_q[b + 1] for sequence b; lens[b] (int32 [B]
    on the device) counts its tokens with these, which cache_write has written before; table int32
    [B, pages of a sequence].  The cache is of q's type or in 8 bits."""
    if lens.dim() != 1:
        raise ValueError("lens must hold a length for each sequence")
    B = lens.shape[0]
    if cu_q is None and q.shape[0] != B:
        raise ValueError(f"without cu_q, q must hold one token of each of {B} sequences")
    t, width = _table(table, B, q.device), table.shape[1]
    need_ws = width * cache.page > (_NO_WS_ONE if cu_q is None else _NO_WS)
    a, out, dev, space, nb = _attn(q, B, cu_q, True, scale, out, cache.H, need_ws, ws, stream)
    if cache.device != dev or cache.D != a.D:
        raise ValueError(f"the cache holds heads of {cache.D} on {cache.device}")
    n = _vector(lens, "lens", B, torch.int32, dev)
    _check(_on_device(dev, stream, lib().cham_cache_attention, a, cache._struct, t, width, n, space, nb), "cache_attention")
    return out
