"""ctypes binding of libcafeq.so: argument marshalling only.

Every function takes torch CUDA tensors (used purely as device memory), builds the
C descriptors of include/cafeq.h and enqueues the call on torch's current stream.
There is no fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import struct
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("CAFEQ_LIBRARY", os.path.join(_HERE, "libcafeq.so"))

AXIS_COL, AXIS_ROW = 0, 1
Q_SYM, Q_MINMAX = 0, 1   # the symmetric absmax grid; the min/max grid of the paper's Eq. (1)
SIDE_T, SIDE_TINV = 0, 1
F32, BF16, I8 = 0, 1, 2   # I8: activations of infer_packed only
CALL_RTN, CALL_PROXY, CALL_DUAL, CALL_ADAPTIVE = 0, 1, 2, 3

EXPORTS = (
    "cafeq_strerror", "cafeq_version", "cafeq_workspace_bytes", "cafeq_block_inverse",
    "cafeq_rtn_quantize", "cafeq_apply_transform", "cafeq_proxy_loss_fwd_bwd",
    "cafeq_dual_proxy_loss_fwd_bwd", "cafeq_adaptive_round_step",
    "cafeq_orth_penalty", "cafeq_sgd_update", "cafeq_adam_update", "cafeq_optimize_single",
    "cafeq_optimize_pair", "cafeq_pqe", "cafeq_rtn_quantize_minmax", "cafeq_hadamard_rtn", "cafeq_hadamard_workspace_bytes",
    "cafeq_infer_single", "cafeq_infer_workspace_bytes", "cafeq_set_launch_timing", "cafeq_rtn_quantize_static", "cafeq_prepared_bytes", "cafeq_prepare_weights",
    "cafeq_stream_read_probe", "cafeq_norm_quantize", "cafeq_norm_workspace_bytes", "cafeq_packed_bytes", "cafeq_pack_nibbles",
    "cafeq_infer_packed", "cafeq_infer_packed_workspace_bytes",
    "cafeq_rotate_heads", "cafeq_cache_append", "cafeq_cache_values", "cafeq_cache_attend", "cafeq_cache_attend_workspace_bytes",
    "cafeq_cache_reserve", "cafeq_cache_reorder", "cafeq_cache_compact", "cafeq_cache_pages_workspace_bytes",
)


class CafeqError(RuntimeError):
    pass


class Mat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("prepared", ctypes.c_void_p)]


class Xform(ctypes.Structure):
    _fields_ = [("T", ctypes.c_void_p), ("Tinv", ctypes.c_void_p), ("k", ctypes.c_int32),
                ("nb", ctypes.c_int32), ("rep", ctypes.c_int32)]


class QuantCfg(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("group", ctypes.c_int32), ("axis", ctypes.c_int32),
                ("mode", ctypes.c_int32)]


class LaunchTiming(ctypes.Structure):
    _fields_ = [("start", ctypes.POINTER(ctypes.c_void_p)), ("stop", ctypes.POINTER(ctypes.c_void_p)),
                ("capacity", ctypes.c_int32), ("count", ctypes.c_int32), ("every", ctypes.c_int32),
                ("seen", ctypes.c_int32), ("kind", ctypes.c_int32)]


class OptCfg(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("lr", ctypes.c_float), ("lambda_orth", ctypes.c_float),
                ("normalize", ctypes.c_int32), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double)]


class Activations(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("sum", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("ldr", ctypes.c_int64), ("lds", ctypes.c_int64), ("dtype", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("gain", ctypes.c_void_p), ("gain_offset", ctypes.c_float), ("eps", ctypes.c_float)]


class Heads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("hsx", ctypes.c_int64), ("ldo", ctypes.c_int64),
                ("hso", ctypes.c_int64), ("heads", ctypes.c_int32), ("gain", ctypes.c_void_p)]


class Rotation(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("d", ctypes.c_int32), ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("eps", ctypes.c_float), ("gain_offset", ctypes.c_float), ("amplitude", ctypes.c_float)]


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("kscale", ctypes.c_void_p), ("vscale", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("pages", ctypes.c_int64), ("sequences", ctypes.c_int32), ("width", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("d", ctypes.c_int32), ("block", ctypes.c_int32), ("missing", ctypes.c_void_p)]


class Attention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("n", ctypes.c_int64), ("ldq", ctypes.c_int64),
                ("hsq", ctypes.c_int64), ("ldo", ctypes.c_int64), ("hso", ctypes.c_int64), ("longest", ctypes.c_int64), ("starts", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float), ("softcap", ctypes.c_float)]


_pack_attention = struct.Struct("@PPPqqqqqqPiiiiff").pack      # an Attention's bytes, in a quarter of the time


def _load():
    if not os.path.exists(LIB_PATH):
        raise CafeqError("libcafeq.so has not been built (run `python __graft_entry__.py`): " + LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    missing = [n for n in EXPORTS if not hasattr(lib, n)]
    if missing:
        raise CafeqError("libcafeq.so lacks exports: %s" % missing)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.cafeq_strerror.restype = ctypes.c_char_p
    lib.cafeq_strerror.argtypes = [i32]
    lib.cafeq_version.restype = i32
    lib.cafeq_workspace_bytes.restype = ctypes.c_size_t
    lib.cafeq_workspace_bytes.argtypes = [i32, ctypes.POINTER(Mat), ctypes.POINTER(Mat),
                                          ctypes.POINTER(Xform), ctypes.POINTER(QuantCfg)]
    lib.cafeq_block_inverse.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.cafeq_rtn_quantize.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(QuantCfg), vp, vp, vp, vp, vp]
    lib.cafeq_prepared_bytes.restype = ctypes.c_size_t
    lib.cafeq_prepared_bytes.argtypes = [ctypes.POINTER(Mat), i32]
    lib.cafeq_prepare_weights.argtypes = [ctypes.POINTER(Mat), i32, vp, vp]
    lib.cafeq_rtn_quantize_static.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(QuantCfg), vp, vp, vp, vp]
    lib.cafeq_apply_transform.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(Xform), i32, i32, vp, vp, vp]
    lib.cafeq_proxy_loss_fwd_bwd.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(Xform),
                                             ctypes.POINTER(QuantCfg), vp, vp, vp, vp, vp, vp]
    lib.cafeq_dual_proxy_loss_fwd_bwd.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(Mat),
                                                  ctypes.POINTER(Xform), ctypes.POINTER(QuantCfg),
                                                  ctypes.c_float, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.cafeq_adaptive_round_step.argtypes = [vp, vp, i64, i64, i64, i64, ctypes.POINTER(QuantCfg),
                                              i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    f32 = ctypes.c_float
    lib.cafeq_orth_penalty.argtypes = [vp, i32, i32, f32, vp, vp, vp, vp]
    lib.cafeq_sgd_update.argtypes = [vp, vp, f32, vp, i64, vp]
    f64 = ctypes.c_double
    lib.cafeq_adam_update.argtypes = [vp, vp, vp, vp, i32, f64, f64, f64, f64, i64, vp]
    lib.cafeq_optimize_single.argtypes = [ctypes.POINTER(Mat), vp, vp, i32, i32, i32, ctypes.POINTER(QuantCfg),
                                          ctypes.POINTER(OptCfg), vp, vp, vp, vp]
    lib.cafeq_optimize_pair.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(Mat), vp, vp, i32, i32, i32,
                                        ctypes.POINTER(QuantCfg), f32, ctypes.POINTER(OptCfg), vp, vp, vp, vp, vp]
    lib.cafeq_rtn_quantize_minmax.argtypes = [ctypes.POINTER(Mat), ctypes.POINTER(QuantCfg), vp, vp, vp, vp, vp, vp]
    lib.cafeq_hadamard_workspace_bytes.restype = ctypes.c_size_t
    lib.cafeq_hadamard_workspace_bytes.argtypes = [i64, i64, i32]
    lib.cafeq_infer_workspace_bytes.restype = ctypes.c_size_t
    lib.cafeq_infer_workspace_bytes.argtypes = [i32, i64]
    lib.cafeq_infer_single.argtypes = [vp, i32, i64, ctypes.POINTER(Xform), vp, vp, i64, i64, i32, vp, i64, vp, vp]
    lib.cafeq_hadamard_rtn.argtypes = [ctypes.POINTER(Mat), vp, i32, ctypes.POINTER(QuantCfg), vp, vp, vp, vp, vp, vp]
    lib.cafeq_pqe.argtypes = [vp, vp, i64, i64, i64, i64, ctypes.POINTER(QuantCfg), i32, i32, i32, vp, vp, vp, vp,
                              vp, vp, vp]
    lib.cafeq_set_launch_timing.argtypes = [ctypes.POINTER(LaunchTiming)]
    lib.cafeq_stream_read_probe.argtypes = [vp, ctypes.c_size_t, vp, vp]
    lib.cafeq_norm_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(Xform), i64]
    lib.cafeq_norm_quantize.argtypes = [ctypes.POINTER(Activations), i64, i64, ctypes.POINTER(Xform), i64, vp, vp, vp, i32,
                                        i64, vp, vp]
    lib.cafeq_packed_bytes.argtypes = [i64, i64, i64]
    lib.cafeq_pack_nibbles.argtypes = [vp, vp, i64, i64, i64, vp, vp]
    lib.cafeq_infer_packed.argtypes = [vp, i32, i64, i64, vp, i64, vp, i64, i64, i64, vp, i32, i64, vp, vp]
    lib.cafeq_infer_packed_workspace_bytes.argtypes = [i32, i64, i64, i64, i64]
    cache = ctypes.POINTER(Cache)
    lib.cafeq_rotate_heads.argtypes = [ctypes.POINTER(Rotation), ctypes.POINTER(Heads), ctypes.POINTER(Heads), i64, vp, vp, vp]
    lib.cafeq_cache_append.argtypes = [cache, vp, vp, i32, i64, i64, i64, i64, i64, vp, i64, vp]
    lib.cafeq_cache_values.argtypes = [cache, vp, vp, i64, vp, vp, i32, vp]
    lib.cafeq_cache_attend.argtypes = [cache, vp, vp, vp]      # (an Attention, or its bytes)
    lib.cafeq_cache_attend_workspace_bytes.argtypes = [cache, vp]
    lib.cafeq_cache_reserve.argtypes = [cache, vp, i64, vp, vp, vp, vp]
    lib.cafeq_cache_reorder.argtypes = [cache, vp, vp, vp]
    lib.cafeq_cache_compact.argtypes = [cache, vp, vp, vp]
    lib.cafeq_cache_pages_workspace_bytes.argtypes = [cache]
    for n in EXPORTS[3:]:
        getattr(lib, n).restype = ctypes.c_size_t if n.endswith("_bytes") else i32
    return lib


lib = _load()


def _check(rc):
    if rc != 0:
        raise CafeqError("cafeq call failed: %s (%d)" % (lib.cafeq_strerror(rc).decode(), rc))


# The smallest calls wait for the host (256 x 256, blocks of 32: three launches, 19 us of the GPU): torch.cuda.current_stream(), which
# makes a Stream object, took 2.8 us a call, the handle alone takes 0.1; integers as pointers 0.05 us against 0.14 for ctypes objects.
def _stream():
    """Handle of the current device's current stream."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _prepared_ptr(m, prepared, axis):
    """Address of a prepared copy of m, transformed along `axis` (None: whichever it was made for), for its descriptor.
    A copy made from the same values in the other storage type has another layout and is not read: the call runs on the
    weights themselves.  A buffer too small for either is refused: the kernels would read past its end."""
    have = prepared.numel() * prepared.element_size()
    other = Mat(m.data, m.rows, m.cols, m.ld, BF16 if m.dtype == F32 else F32, 0)
    axes = (AXIS_COL, AXIS_ROW) if axis is None else (axis,)
    need = [int(lib.cafeq_prepared_bytes(ctypes.byref(m), a)) for a in axes]
    if have in need:
        return prepared.data_ptr()
    if have in [int(lib.cafeq_prepared_bytes(ctypes.byref(other), a)) for a in axes]:
        return 0
    if have < max(need):
        raise CafeqError("the prepared copy holds %d bytes, that of this matrix %d: made for another one?" % (have, max(need)))
    return prepared.data_ptr()


def mat(t, prepared=None, axis=None):
    """Descriptor of a 2-D CUDA tensor (float32 or bfloat16, unit column stride); `prepared`: the buffer
    prepare_weights() returned for it and the axis the call transforms, or None."""
    if t.dim() != 2 or t.stride(1) != 1 or not t.is_cuda:
        raise CafeqError("need a 2-D CUDA tensor with unit column stride")
    if t.dtype == torch.float32:
        dt = F32
    elif t.dtype == torch.bfloat16:
        dt = BF16
    else:
        raise CafeqError("dtype must be float32 or bfloat16")
    m = Mat(t.data_ptr(), t.shape[0], t.shape[1], t.stride(0), dt, 0)
    if prepared is not None:
        m.prepared = _prepared_ptr(m, prepared, axis)
    return m


def xform(T, Tinv, rep=1):
    for x in (T, Tinv):
        if x is not None and (x.dtype != torch.float32 or not x.is_contiguous() or x.dim() != 3):
            raise CafeqError("transform blocks must be contiguous float32 [nb][k][k]")
    return Xform(_ptr(T), _ptr(Tinv), T.shape[1], T.shape[0], rep)


_ws_cache = {}


def workspace(nbytes, device):
    """A cached scratch buffer (device memory owned by the binding, grown on demand)."""
    key = (device.type, device.index)
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < nbytes:
        buf = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
        _ws_cache[key] = buf
    return buf


def workspace_bytes(call_id, a, b=None, x=None, cfg=None):
    return int(lib.cafeq_workspace_bytes(call_id, ctypes.byref(a), ctypes.byref(b) if b else None,
                                         ctypes.byref(x) if x else None,
                                         ctypes.byref(cfg) if cfg else None))


def _scale_shape(rows, cols, group, axis):
    if axis == AXIS_COL:
        return (rows, cols // (group or cols))
    return (rows // (group or rows), cols)


def _minmax_shape(shape, mode):
    """Scale buffer of the fused calls: on the min/max grid the group minima follow the scales."""
    return shape if mode == Q_SYM else (2,) + tuple(shape)


def rtn_quantize(W, bits, group, axis=AXIS_COL, want_err=False):
    m = mat(W)
    cfg = QuantCfg(bits, group, axis, 0)
    R, C = W.shape
    codes = torch.empty((R, C), dtype=torch.int8, device=W.device)
    scales = torch.empty(_scale_shape(R, C, group, axis), dtype=torch.float32, device=W.device)
    err = torch.empty(1, dtype=torch.float32, device=W.device) if want_err else None
    ws = workspace(workspace_bytes(CALL_RTN, m, cfg=cfg), W.device) if want_err else None
    _check(lib.cafeq_rtn_quantize(ctypes.byref(m), ctypes.byref(cfg), _ptr(codes), _ptr(scales),
                                  _ptr(err), _ptr(ws), _stream()))
    return codes, scales, err


def prepare_weights(W, axis=AXIS_COL):
    """The prepared copy of W for transforms along `axis` (a uint8 tensor; see cafeq_prepare_weights)."""
    m = mat(W)
    nbytes = int(lib.cafeq_prepared_bytes(ctypes.byref(m), axis))
    if nbytes == 0:
        raise CafeqError("weights cannot be prepared for this axis (its length must be a multiple of 128)")
    buf = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    _check(lib.cafeq_prepare_weights(ctypes.byref(m), axis, _ptr(buf), _stream()))
    return buf


def rtn_quantize_static(W, codes, scales, err, bits, group, axis=AXIS_COL):
    """The quantizer with built-in scratch: the caller passes every output buffer; nothing is allocated."""
    m = mat(W)
    cfg = QuantCfg(bits, group, axis, 0)
    _check(lib.cafeq_rtn_quantize_static(ctypes.byref(m), ctypes.byref(cfg), _ptr(codes), _ptr(scales),
                                         _ptr(err), _stream()))


def block_inverse(T, want_rho=False):
    """Tinv (and optionally rho_row, rho_col) plus per-block status."""
    nb, k, _ = T.shape
    dev = T.device
    Tinv = torch.empty_like(T)
    rr = torch.empty(nb * k, dtype=torch.float32, device=dev) if want_rho else None
    rc_ = torch.empty(nb * k, dtype=torch.float32, device=dev) if want_rho else None
    status = torch.empty(nb, dtype=torch.int32, device=dev)
    x = Xform(_ptr(T), 0, k, nb, 1)
    ws = workspace(int(lib.cafeq_workspace_bytes(4, None, None, ctypes.byref(x), None)), dev)
    _check(lib.cafeq_block_inverse(_ptr(T), k, nb, _ptr(Tinv), _ptr(rr), _ptr(rc_), _ptr(status),
                                   _ptr(ws), _stream()))
    return (Tinv, rr, rc_, status) if want_rho else (Tinv, status)


def apply_transform(W, T, Tinv=None, axis=AXIS_COL, side=SIDE_T, rep=1):
    m = mat(W)
    x = xform(T, Tinv, rep)
    Z = torch.empty(W.shape, dtype=torch.float32, device=W.device)
    ws = workspace(int(lib.cafeq_workspace_bytes(5, None, None, ctypes.byref(x), None)), W.device)
    _check(lib.cafeq_apply_transform(ctypes.byref(m), ctypes.byref(x), axis, side, _ptr(Z), _ptr(ws), _stream()))
    return Z


def proxy_loss_fwd_bwd(W, T, Tinv, bits, group, axis=AXIS_COL, rep=1, want_grad=True, want_codes=False,
                       prepared=None, mode=Q_SYM):
    """Returns (losses[4], gradT or None, codes or None, scales or None).  With mode=Q_MINMAX the codes are
    unsigned bytes and `scales` is [2][...]: the scales, then the group minima."""
    m = mat(W, prepared, axis)
    x = xform(T, Tinv, rep)
    cfg = QuantCfg(bits, group, axis, mode)
    dev = W.device
    losses = torch.empty(4, dtype=torch.float32, device=dev)
    grad = torch.empty_like(T) if want_grad else None
    R, C = W.shape
    codes = torch.empty((R, C), dtype=torch.int8, device=dev) if want_codes else None
    scales = torch.empty(_minmax_shape(_scale_shape(R, C, group, axis), mode), dtype=torch.float32,
                         device=dev) if want_codes else None
    nbytes = workspace_bytes(CALL_PROXY, m, x=x, cfg=cfg)
    if nbytes == 0:
        raise CafeqError("unsupported proxy-loss configuration (workspace query returned 0)")
    ws = workspace(nbytes, dev)
    _check(lib.cafeq_proxy_loss_fwd_bwd(ctypes.byref(m), ctypes.byref(x), ctypes.byref(cfg), _ptr(losses),
                                        _ptr(grad), _ptr(codes), _ptr(scales), _ptr(ws), _stream()))
    if want_codes and mode == Q_MINMAX:
        codes = codes.view(torch.uint8)
    return losses, grad, codes, scales


def dual_proxy_loss_fwd_bwd(A, B, T, Tinv, bits, group, rep=1, lse_t=5.0, want_grad=True, want_codes=False,
                            prepared=(None, None), mode=Q_SYM):
    """Returns (losses[6], gradT or None, (codesU, scalesU, codesV, scalesV) or None); mode as in
    proxy_loss_fwd_bwd."""
    ma, mb = mat(A, prepared[0], AXIS_COL), mat(B, prepared[1], AXIS_ROW)
    x = xform(T, Tinv, rep)
    cfg = QuantCfg(bits, group, 0, mode)
    dev = A.device
    losses = torch.empty(6, dtype=torch.float32, device=dev)
    grad = torch.empty_like(T) if want_grad else None
    outs = None
    cu = su = cv = sv = None
    if want_codes:
        cu = torch.empty(A.shape, dtype=torch.int8, device=dev)
        su = torch.empty(_minmax_shape(_scale_shape(A.shape[0], A.shape[1], group, AXIS_COL), mode),
                         dtype=torch.float32, device=dev)
        cv = torch.empty(B.shape, dtype=torch.int8, device=dev)
        sv = torch.empty(_minmax_shape(_scale_shape(B.shape[0], B.shape[1], group, AXIS_ROW), mode),
                         dtype=torch.float32, device=dev)
        outs = (cu, su, cv, sv) if mode == Q_SYM else (cu.view(torch.uint8), su, cv.view(torch.uint8), sv)
    nbytes = workspace_bytes(CALL_DUAL, ma, mb, x, cfg)
    if nbytes == 0:
        raise CafeqError("unsupported dual configuration (workspace query returned 0)")
    ws = workspace(nbytes, dev)
    _check(lib.cafeq_dual_proxy_loss_fwd_bwd(ctypes.byref(ma), ctypes.byref(mb), ctypes.byref(x),
                                             ctypes.byref(cfg), ctypes.c_float(lse_t), _ptr(losses), _ptr(grad),
                                             _ptr(cu), _ptr(su), _ptr(cv), _ptr(sv), _ptr(ws), _stream()))
    return losses, grad, outs


def adaptive_round_step(U, V, codesU, scalesU, codesV, scalesV, bits, group, k, rep=1, half=0):
    """One iteration of Alg. 1; codes/scales are updated in place.  Returns status[2*nb]."""
    for t in (U, V):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise CafeqError("U and V must be contiguous float32")
    nb = U.shape[1] // k
    cfg = QuantCfg(bits, group, 0, 0)
    mu, mv = mat(U), mat(V)
    x = Xform(0, 0, k, nb, rep)
    status = torch.zeros(2 * nb, dtype=torch.int32, device=U.device)
    nbytes = workspace_bytes(CALL_ADAPTIVE, mu, mv, x, cfg)
    if nbytes == 0:
        raise CafeqError("unsupported adaptive-rounding configuration (workspace query returned 0)")
    ws = workspace(nbytes, U.device)
    _check(lib.cafeq_adaptive_round_step(_ptr(U), _ptr(V), U.shape[0], U.shape[1], V.shape[0], V.shape[1],
                                         ctypes.byref(cfg), k, nb, rep, half, _ptr(codesU), _ptr(scalesU),
                                         _ptr(codesV), _ptr(scalesV), _ptr(status), _ptr(ws), _stream()))
    return status


def stream_read_probe(buf, sink=None):
    """One launch of the library's plain streaming read over the tensor `buf` (cafeq_stream_read_probe)."""
    if sink is None:
        sink = torch.zeros(1, dtype=torch.int32, device=buf.device)
    _check(lib.cafeq_stream_read_probe(_ptr(buf), ctypes.c_size_t(buf.numel() * buf.element_size()), _ptr(sink),
                                       _stream()))
    return sink


class LaunchTimer:
    """Caller-owned events around the fused-kernel launches (cafeq_set_launch_timing): `capacity` pairs of
    torch events are created up front; the library only records them.  every > 1: only every `every`-th launch
    is timed (an event pair holds the stream up for several microseconds).  kind: 0 the loss pass (fused transform
    kernel), 1 the gradient pass over the weights."""

    def __init__(self, capacity, every=1, kind=0):
        self.ev = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(capacity)]
        for a, b in self.ev:          # torch creates the underlying event on first use
            a.record()
            b.record()
        torch.cuda.synchronize()
        self.start = (ctypes.c_void_p * capacity)(*[a.cuda_event for a, _ in self.ev])
        self.stop = (ctypes.c_void_p * capacity)(*[b.cuda_event for _, b in self.ev])
        self.table = LaunchTiming(self.start, self.stop, capacity, 0, every, 0, kind)

    def __enter__(self):
        self.table.count = 0
        self.table.seen = 0
        _check(lib.cafeq_set_launch_timing(ctypes.byref(self.table)))
        return self

    def __exit__(self, *exc):
        _check(lib.cafeq_set_launch_timing(None))

    def durations_ms(self):
        """Per-launch durations (the caller has synchronised the stream)."""
        return [self.ev[i][0].elapsed_time(self.ev[i][1]) for i in range(self.table.count)]


def orth_penalty(T, lam, grad=None):
    """(value[1], grad) with grad incremented in place when given."""
    nb, k, _ = T.shape
    x = Xform(_ptr(T), 0, k, nb, 1)
    ws = workspace(int(lib.cafeq_workspace_bytes(6, None, None, ctypes.byref(x), None)), T.device)
    value = torch.empty(1, dtype=torch.float32, device=T.device)
    _check(lib.cafeq_orth_penalty(_ptr(T), k, nb, lam, _ptr(value), _ptr(grad), _ptr(ws), _stream()))
    return value, grad


def sgd_update(T, grad, lr, denom=None):
    _check(lib.cafeq_sgd_update(_ptr(T), _ptr(grad), lr, _ptr(denom), T.numel(), _stream()))


def adam_update(T, grad, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8):
    _check(lib.cafeq_adam_update(_ptr(T), _ptr(grad), _ptr(m), _ptr(v), step, lr, beta1, beta2, eps, T.numel(),
                                 _stream()))


def optimize_single(W, T, bits, group, axis=AXIS_COL, rep=1, lr=1.0, steps=10, lambda_orth=0.0, normalize=True,
                    mode=Q_SYM):
    """Gradient descent on the surrogate, T updated in place.  Returns (Tinv, history[steps][8], status)."""
    m = mat(W)
    nb, k, _ = T.shape
    Tinv = torch.empty_like(T)
    x = Xform(_ptr(T), _ptr(Tinv), k, nb, rep)
    cfg = QuantCfg(bits, group, axis, mode)
    opt = OptCfg(steps, lr, lambda_orth, 1 if normalize else 0, 0.0, 0.0, 0.0)
    ws = workspace(int(lib.cafeq_workspace_bytes(7, ctypes.byref(m), None, ctypes.byref(x), ctypes.byref(cfg))), W.device)
    history = torch.empty((max(steps, 1), 8), dtype=torch.float32, device=W.device)
    status = torch.empty(nb, dtype=torch.int32, device=W.device)
    _check(lib.cafeq_optimize_single(ctypes.byref(m), _ptr(T), _ptr(Tinv), k, nb, rep, ctypes.byref(cfg),
                                     ctypes.byref(opt), _ptr(history), _ptr(status), _ptr(ws), _stream()))
    return Tinv, history[:steps], status


def optimize_pair(A, B, T, bits, group, rep=1, lse_t=5.0, lr=1e-2, steps=10, lambda_orth=0.0, beta1=0.1,
                  beta2=0.999, eps=1e-8, prepared=(None, None), mode=Q_SYM):
    """Adam on the LogSumExp surrogate, T updated in place.  Returns (Tinv, history[steps][8], status)."""
    ma, mb = mat(A, prepared[0], AXIS_COL), mat(B, prepared[1], AXIS_ROW)
    nb, k, _ = T.shape
    Tinv = torch.empty_like(T)
    x = Xform(_ptr(T), _ptr(Tinv), k, nb, rep)
    cfg = QuantCfg(bits, group, 0, mode)
    opt = OptCfg(steps, lr, lambda_orth, 0, beta1, beta2, eps)
    ws = workspace(int(lib.cafeq_workspace_bytes(8, ctypes.byref(ma), ctypes.byref(mb), ctypes.byref(x),
                                                 ctypes.byref(cfg))), A.device)
    moments = torch.empty(2 * T.numel(), dtype=torch.float32, device=A.device)
    history = torch.empty((max(steps, 1), 8), dtype=torch.float32, device=A.device)
    status = torch.empty(nb, dtype=torch.int32, device=A.device)
    _check(lib.cafeq_optimize_pair(ctypes.byref(ma), ctypes.byref(mb), _ptr(T), _ptr(Tinv), k, nb, rep,
                                   ctypes.byref(cfg), lse_t, ctypes.byref(opt), _ptr(moments), _ptr(history),
                                   _ptr(status), _ptr(ws), _stream()))
    return Tinv, history[:steps], status


def pqe(U, V, codesU, scalesU, codesV, scalesV, bits, group, k, rep=1):
    """out[2] (device): sum of squared paired quantization errors over heads, and of the squared products."""
    nb = U.shape[1] // k
    mu, mv = mat(U), mat(V)
    x = Xform(0, 0, k, nb, rep)
    cfg = QuantCfg(bits, group, 0, 0)
    ws = workspace(int(lib.cafeq_workspace_bytes(9, ctypes.byref(mu), ctypes.byref(mv), ctypes.byref(x),
                                                 ctypes.byref(cfg))), U.device)
    out = torch.empty(2, dtype=torch.float32, device=U.device)
    _check(lib.cafeq_pqe(_ptr(U), _ptr(V), U.shape[0], U.shape[1], V.shape[0], V.shape[1], ctypes.byref(cfg), k, nb,
                         rep, _ptr(codesU), _ptr(scalesU), _ptr(codesV), _ptr(scalesV), _ptr(out), _ptr(ws), _stream()))
    return out


def rtn_quantize_minmax(W, bits, group, axis=AXIS_COL, want_err=False):
    """Eq. (1) grid: (codes uint8, scales, mins, err or None)."""
    m = mat(W)
    cfg = QuantCfg(bits, group, axis, 1)
    R, C = W.shape
    codes = torch.empty((R, C), dtype=torch.uint8, device=W.device)
    shape = _scale_shape(R, C, group, axis)
    scales = torch.empty(shape, dtype=torch.float32, device=W.device)
    mins = torch.empty(shape, dtype=torch.float32, device=W.device)
    err = torch.empty(1, dtype=torch.float32, device=W.device) if want_err else None
    ws = workspace(workspace_bytes(CALL_RTN, m, cfg=cfg), W.device) if want_err else None
    _check(lib.cafeq_rtn_quantize_minmax(ctypes.byref(m), ctypes.byref(cfg), _ptr(codes), _ptr(scales), _ptr(mins),
                                         _ptr(err), _ptr(ws), _stream()))
    return codes, scales, mins, err


def hadamard_rtn(W, signs, block, bits, group, want_z=False, want_codes=False):
    """Randomized-Hadamard baseline: (losses[2] = (err_sq, w_sq), Z or None, codes or None, scales or None)."""
    m = mat(W)
    cfg = QuantCfg(bits, group, AXIS_COL, 0)
    R, C = W.shape
    dev = W.device
    Z = torch.empty((R, C), dtype=torch.float32, device=dev) if want_z else None
    codes = torch.empty((R, C), dtype=torch.int8, device=dev) if want_codes else None
    scales = torch.empty((R, C // group), dtype=torch.float32, device=dev) if want_codes else None
    losses = torch.empty(2, dtype=torch.float32, device=dev)
    ws = workspace(int(lib.cafeq_hadamard_workspace_bytes(R, C, block)), dev)
    _check(lib.cafeq_hadamard_rtn(ctypes.byref(m), _ptr(signs), block, ctypes.byref(cfg), _ptr(Z), _ptr(codes),
                                  _ptr(scales), _ptr(losses), _ptr(ws), _stream()))
    return losses, Z, codes, scales


def infer_single(X, Tinv, codes, scales, group, out=None):
    """Y[n][out] = (X . blockdiag(Tinv)^T) . dequant(codes, scales)^T; Tinv None = no transform."""
    n, d = X.shape
    O = codes.shape[0]
    Y = out if out is not None else torch.empty((n, O), dtype=torch.float32, device=X.device)
    if Tinv is not None:
        nb, k, _ = Tinv.shape
        xf = Xform(None, _ptr(Tinv), k, nb, 1)
        ws = workspace(int(lib.cafeq_infer_workspace_bytes(n, d)), X.device)
        xfp = ctypes.byref(xf)
    else:
        ws, xfp = None, None
    _check(lib.cafeq_infer_single(_ptr(X), n, X.stride(0), xfp, _ptr(codes), _ptr(scales), O, d, group, _ptr(Y),
                                  Y.stride(0), _ptr(ws), _stream()))
    return Y


_FLOATS = {torch.float32: F32, torch.bfloat16: BF16}
_ERR_WORKSPACE = -7

# The calls below are made once a projection and token: their checks read each property of a tensor once (a property takes 0.05 to 0.15 us;
# an allocation 1.2 by empty_like or empty_strided, 2 by empty; the launch 3.7).  A norm of one row with its sum: 17.2 -> 13.1 us of the host; a product with one token 11.8 -> 8.2.


def _rows(t, dev, what):
    """Leading dimension of a 2-D tensor with unit column stride on device number `dev`."""
    st = t.stride()
    if len(st) != 2 or t.get_device() != dev or (st[1] != 1 and t.shape[1] > 1):
        raise CafeqError("%s: need a 2-D tensor with unit column stride on the current CUDA device" % what)
    return st[0] if t.shape[0] > 1 else max(st[0], t.shape[1])


def _operand(t, dev, dtype, shape, what):
    """Address of an operand that has to be contiguous, of this type and shape, on device number `dev`."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise CafeqError("%s: need a contiguous tensor %s of %s on the current CUDA device" % (what, tuple(shape), dtype))
    return t.data_ptr()


class Normed(NamedTuple):
    """What norm_quantize returns; None for what was not asked for."""
    codes: Optional[torch.Tensor]
    scales: Optional[torch.Tensor]
    values: Optional[torch.Tensor]
    sum: Optional[torch.Tensor]


def norm_quantize(X, gain=None, residual=None, eps=1e-6, gain_offset=0.0, norm=True, Tinv=None, group=0, values=None,
                  sum_out=None):
    """cafeq_norm_quantize: residual addition, root-mean-square norm (norm=False: none), the transform's inverse blocks Tinv and
    8 bits with a scale per `group` columns (0: per row; None: no codes).  X, residual [n][d] float32 or bfloat16.
    values: None, or the type of a tensor that receives what the codes stand for (without codes: the result itself).
    The sum X + residual is returned where a residual is given, in sum_out if that is given too (which without Tinv may be X or
    residual)."""
    dtype, dev = X.dtype, torch._C._cuda_getDevice()
    kind = _FLOATS.get(dtype)
    if kind is None:
        raise CafeqError("X must be float32 or bfloat16")
    ldx = _rows(X, dev, "X")
    n, d = shape = X.shape
    px = X.data_ptr()
    res = ldr = total = lds = xf = None
    pgain = None if gain is None else _operand(gain, dev, torch.float32, (d,), "gain")
    if residual is not None:
        if residual.shape != shape or residual.dtype is not dtype:
            raise CafeqError("residual must have the shape and type of X")
        res, ldr = residual.data_ptr(), _rows(residual, dev, "residual")
        if sum_out is None:
            sum_out = torch.empty_like(X)
            total, lds = sum_out.data_ptr(), d
    if sum_out is not None and total is None:
        if sum_out.shape != shape or sum_out.dtype is not dtype:
            raise CafeqError("sum_out must have the shape and type of X")
        total, lds = sum_out.data_ptr(), _rows(sum_out, dev, "sum_out")
    codes = scales = pcodes = pscales = out = pout = None
    g = -1
    if group is not None:
        g = group
        if group < 0 or (group and d % group):
            raise CafeqError("group must divide the columns")
        ng = d // group if group else 1
        codes = torch.empty_like(X, dtype=torch.int8)
        scales = torch.empty_strided((n, ng), (ng, 1), dtype=torch.float32, device=X.device)
        pcodes, pscales = codes.data_ptr(), scales.data_ptr()
    vkind = F32
    if values is not None:
        vkind = _FLOATS.get(values)
        if vkind is None:
            raise CafeqError("values must be torch.float32 or torch.bfloat16")
        out = torch.empty_like(X, dtype=values)
        pout = out.data_ptr()
    elif group is None:
        raise CafeqError("neither codes nor values are asked for")
    if Tinv is not None:
        k = Tinv.shape[-1]
        xf = ctypes.byref(Xform(None, _operand(Tinv, dev, torch.float32, (d // k if k else 0, k, k), "Tinv"), k, d // k, 1))
    if n:
        a = Activations(px, res, total, ldx, ldr or 0, lds or 0, kind, 1 if norm else 0, pgain, gain_offset, eps)
        stream = torch._C._cuda_getCurrentRawStream(dev)
        rc = lib.cafeq_norm_quantize(ctypes.byref(a), n, d, xf, g if g > 0 else 0, pcodes, pscales, pout, vkind, d, None, stream)
        if rc == _ERR_WORKSPACE:
            # few rows need none and are what waits for the host; the buffer is of this call alone, so that streams share nothing
            ws = X.new_empty(lib.cafeq_norm_workspace_bytes(n, d, xf, g), dtype=torch.uint8)
            rc = lib.cafeq_norm_quantize(ctypes.byref(a), n, d, xf, g if g > 0 else 0, pcodes, pscales, pout, vkind, d, ws.data_ptr(), stream)
        if rc:
            _check(rc)
    return Normed(codes, scales, out, sum_out)


class PackedWeight(NamedTuple):
    """Weights packed by pack_nibbles: the buffer and what it was made from."""
    data: torch.Tensor
    rows: int
    cols: int
    group: int


@functools.lru_cache(maxsize=None)
def _packed_bytes(rows, cols, group):
    return int(lib.cafeq_packed_bytes(rows, cols, group))


def pack_nibbles(codes, scales, group):
    """Codes of up to 4 bits and their scales (AXIS_COL, as rtn_quantize returns them) packed for infer_packed.  Codes outside [-8, 7] are refused;
    seeing them takes a read of all codes and a wait, once a weight (none while a graph is captured, which must not wait)."""
    if codes.dim() != 2:
        raise CafeqError("codes must be a 2-D tensor")
    dev = torch._C._cuda_getDevice()
    rows, cols = codes.shape
    pcodes = _operand(codes, dev, torch.int8, (rows, cols), "codes")
    nbytes = _packed_bytes(rows, cols, group)
    if nbytes == 0:
        raise CafeqError("cannot pack codes of this shape (columns and group must be multiples of 32, the group a divisor)")
    pscales = _operand(scales, dev, torch.float32, _scale_shape(rows, cols, group, AXIS_COL), "scales")
    if not torch.cuda.is_current_stream_capturing():
        low, high = torch.stack(torch.aminmax(codes)).tolist()
        if low < -8 or high > 7:
            raise CafeqError("codes must lie in [-8, 7], these in [%d, %d]: more than 4 bits?" % (low, high))
    buf = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
    _check(lib.cafeq_pack_nibbles(pcodes, pscales, rows, cols, group, buf.data_ptr(), _stream()))
    return PackedWeight(buf, rows, cols, group)


_ACTIVATIONS = {torch.float32: F32, torch.bfloat16: BF16, torch.int8: I8}


def infer_packed(X, weight, xscales=None, xgroup=0, dtype=torch.float32, out=None):
    """Y[n][rows] = X . dequant(weight)^T (cafeq_infer_packed).  X float32 or bfloat16, or the int8 codes of norm_quantize with their
    scales and group; Y in `dtype` (float32 or bfloat16), or in `out`."""
    data, rows, cols, group = weight
    kind, dev = _ACTIVATIONS.get(X.dtype), torch._C._cuda_getDevice()
    if kind is None:
        raise CafeqError("X must be float32, bfloat16 or int8")
    ldx = _rows(X, dev, "X")
    n, d = X.shape
    if d != cols or data.get_device() != dev:
        raise CafeqError("X must have the columns (%d) and the device of the weight" % cols)
    if data.numel() != _packed_bytes(rows, cols, group) or not data.is_contiguous():   # (of another type than bytes: at least as large)
        raise CafeqError("weight: its buffer is not one that pack_nibbles made for %d x %d with groups of %d" % (rows, cols, group))
    ps = None
    if kind == I8:
        if xscales is None or xgroup < 0 or (xgroup and d % xgroup):
            raise CafeqError("int8 activations need their scales and a group that divides the columns")
        ps = _operand(xscales, dev, torch.float32, (n, d // xgroup if xgroup else 1), "xscales")
    elif xscales is not None:
        raise CafeqError("xscales go with int8 activations")
    if out is None:
        ykind, ldy = _FLOATS.get(dtype), rows
    else:
        if out.shape != (n, rows):
            raise CafeqError("out must be [%d][%d]" % (n, rows))
        ykind, ldy = _FLOATS.get(out.dtype), _rows(out, dev, "out")
    if ykind is None:
        raise CafeqError("Y must be float32 or bfloat16")
    if out is None:
        out = torch.empty_strided((n, rows), (rows, 1), dtype=dtype, device=X.device)
    if n:
        px, pw, py, stream = X.data_ptr(), data.data_ptr(), out.data_ptr(), torch._C._cuda_getCurrentRawStream(dev)
        rc = lib.cafeq_infer_packed(px, kind, n, ldx, ps, xgroup, pw, rows, d, group, py, ykind, ldy, None, stream)
        if rc == _ERR_WORKSPACE:
            # few tokens need none and are what waits for the host; the buffer is of this call alone, so that streams share nothing
            ws = X.new_empty(lib.cafeq_infer_packed_workspace_bytes(kind, n, rows, d, group), dtype=torch.uint8)
            rc = lib.cafeq_infer_packed(px, kind, n, ldx, ps, xgroup, pw, rows, d, group, py, ykind, ldy, ws.data_ptr(), stream)
        if rc:
            _check(rc)
    return out


def rotary_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained=8192, low=1.0, high=32.0, device=None):
    """(freq, amplitude) for rotate_heads: float64 [rot/2], base^(-2 i / rot) in radians a position, scaled for contexts `factor` times the
    `trained` one:
      none     as they are
      linear   all divided by factor (positions between the trained ones)
      base     base * factor^(rot / (rot - 2)): the highest frequency stays, the lowest is divided by factor
      parts    a frequency that turns more than `high` times over the trained context stays, one of less than `low` turns is divided by factor,
               linear in the turns between (arXiv 2309.00071, Sec. 3.2); amplitude 0.1 ln(factor) + 1 (its Sec. 3.4)"""
    if rot < 0 or rot % 2 or not base > 0 or not factor > 0:
        raise CafeqError("need an even number of turned channels, and base and factor above 0")
    if scaling not in ("none", "linear", "base", "parts"):
        raise CafeqError("scaling must be none, linear, base or parts")
    if scaling == "parts" and (not trained > 0 or not high > low):
        raise CafeqError("need a trained context above 0 and high above low")
    exponent = torch.arange(0, rot, 2, dtype=torch.float64, device=device) / max(rot, 1)
    if scaling == "base":
        base = base * factor ** (rot / max(1, rot - 2))
    freq = base ** -exponent
    if scaling == "linear":
        return freq / factor, 1.0
    if scaling != "parts":
        return freq, 1.0
    turns = trained * freq / (2 * math.pi)
    keep = ((turns - low) / (high - low)).clamp_(0.0, 1.0)
    return freq * keep + freq / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0


def _head_rows(t, dev, what):
    """(leading dimension, head stride) of a tensor [tokens][heads][d] with neighbouring channels on device number `dev`.  Strides that lead nowhere
    (one token, one head) may be anything: they are given as those of a dense tensor."""
    st = t.stride()
    if len(st) != 3 or t.get_device() != dev or (st[2] != 1 and t.shape[2] > 1):
        raise CafeqError("%s: need a tensor [tokens][heads][d] with unit channel stride on the current CUDA device" % what)
    n, h, d = t.shape
    hs = st[1] if h > 1 else d
    return (st[0] if n > 1 else h * hs), hs


def _part(x, out, gain, d, dev, what):
    if x is None:
        if out is not None or gain is not None:
            raise CafeqError("%s is not given" % what)
        return None, None
    if out is None:
        n, h = x.shape[:2]
        out = torch.empty_strided((n, h, d), (h * d, d, 1), dtype=x.dtype, device=x.device)
    elif out.shape != x.shape or out.dtype is not x.dtype:
        raise CafeqError("out_%s must have the shape and type of %s" % (what, what))
    ldx, hsx = _head_rows(x, dev, what)
    ldo, hso = _head_rows(out, dev, "out_" + what)
    g = None if gain is None else _operand(gain, dev, torch.float32, (d,), "gain_" + what)
    return Heads(x.data_ptr(), out.data_ptr(), ldx, hsx, ldo, hso, x.shape[1], g), out


def rotate_heads(q, k, positions, freq, interleaved=False, norm=False, gain_q=None, gain_k=None, eps=1e-6, gain_offset=0.0, amplitude=1.0, out_q=None,
                 out_k=None):
    """cafeq_rotate_heads: root-mean-square norm of each head (norm=True; with gains) and rotary positions of the first 2 len(freq) channels.
    q, k [n][heads][d] float32 or bfloat16 (either may be None), positions int32 [n], freq and amplitude as rotary_frequencies returns
    them.  out_q, out_k: None (new tensors), or where the results go, which may be q and k themselves.  Returns (out_q, out_k)."""
    x = q if q is not None else k
    if x is None or x.dim() != 3:
        raise CafeqError("need q or k, [n][heads][d]")
    dev, kind = torch._C._cuda_getDevice(), _FLOATS.get(x.dtype)
    if kind is None:
        raise CafeqError("q and k must be float32 or bfloat16")
    n, _, d = x.shape
    if k is not None and (k.dim() != 3 or k.dtype is not x.dtype or k.shape[0] != n or k.shape[2] != d):
        raise CafeqError("q and k must have the same type, tokens and channels")
    pp = _operand(positions, dev, torch.int32, (n,), "positions")
    pf = _operand(freq, dev, torch.float64, (freq.numel(),), "freq")
    hq, out_q = _part(q, out_q, gain_q, d, dev, "q")
    hk, out_k = _part(k, out_k, gain_k, d, dev, "k")
    cfg = Rotation(kind, d, 2 * freq.numel(), 1 if interleaved else 0, 1 if norm else 0, eps, gain_offset, amplitude)
    if n:
        rc = lib.cafeq_rotate_heads(ctypes.byref(cfg), ctypes.byref(hq) if hq is not None else None, ctypes.byref(hk) if hk is not None else None, n, pp, pf,
                                    torch._C._cuda_getCurrentRawStream(dev))
        if rc:
            _check(rc)
    return out_q, out_k


class KVCache:
    """A cache as cafeq.h describes it: codes and scales of keys and values, the page of each block of a sequence, tokens of a sequence, rows that
    hold a page, what the last cache_reserve lacked (int32 [1], made if not given).  Its tensors are checked at the first call and after one of them was replaced or moved; their contents may change at will."""
    __slots__ = ("k", "v", "kscale", "vscale", "table", "lengths", "refs", "missing", "_desc")
    _fields = __slots__[:8]

    def __init__(self, k, v, kscale, vscale, table, lengths, refs, missing=None):
        self.k, self.v, self.kscale, self.vscale, self.table, self.lengths, self.refs = k, v, kscale, vscale, table, lengths, refs
        self.missing = torch.zeros(1, dtype=torch.int32, device=refs.device) if missing is None else missing

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_desc", None)

    def _replace(self, **tensors):
        return KVCache(**{**{n: getattr(self, n) for n in self._fields}, **tensors})


def kv_cache(sequences, pages, heads, d, block=64, width=None, device=None):
    """An empty cache: room for `sequences` rows of `width` blocks (all pages, if not given) over a pool of `pages` pages of `block` tokens."""
    if block not in (16, 32, 64, 128) or d % 16 or not 16 <= d <= 256 or heads < 1 or pages < 1 or sequences < 0:
        raise CafeqError("need blocks of 16, 32, 64 or 128 tokens and d a multiple of 16 up to 256")
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device

    def make(shape, dtype, value=0):
        return torch.full(shape, value, dtype=dtype, device=device)

    return KVCache(make((pages, heads, block, d), torch.int8), make((pages, heads, d, block), torch.int8), make((pages, heads), torch.float32),
                   make((pages, heads), torch.float32), make((sequences, pages if width is None else width), torch.int32, -1),
                   make((sequences,), torch.int32), make((pages,), torch.int32))


def _cache(c, dev):
    """(descriptor, its reference for a call, device, scratch of the page calls, what the tensors were, scratch of attention by its sizes) of a KVCache on
    device number `dev`.  The checks of eight tensors (8 us) are made once, and again where one has another address, shape or order."""
    have = c._desc
    k, v, ks, vs, table, lengths, refs, missing = c.k, c.v, c.kscale, c.vscale, c.table, c.lengths, c.refs, c.missing
    at = (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), table.data_ptr(), lengths.data_ptr(), refs.data_ptr(), missing.data_ptr(), k.shape, v.shape,
          table.shape, ks.numel(), vs.numel(), lengths.numel(), refs.numel(), missing.numel(), k.is_contiguous(), v.is_contiguous(), ks.is_contiguous(),
          vs.is_contiguous(), table.is_contiguous(), lengths.is_contiguous(), refs.is_contiguous(), missing.is_contiguous())
    if have is not None and have[2] == dev and have[4] == at:
        return have
    if k.dim() != 4 or table.dim() != 2:
        raise CafeqError("cache: k must be [pages][heads][block][d], table [sequences][width]")
    pages, heads, block, d = k.shape
    rows, width = table.shape
    i8, i32, f32 = torch.int8, torch.int32, torch.float32
    desc = Cache(_operand(k, dev, i8, (pages, heads, block, d), "cache.k"), _operand(v, dev, i8, (pages, heads, d, block), "cache.v"),
                 _operand(ks, dev, f32, (pages, heads), "cache.kscale"), _operand(vs, dev, f32, (pages, heads), "cache.vscale"),
                 _operand(table, dev, i32, (rows, width), "cache.table"), _operand(lengths, dev, i32, (rows,), "cache.lengths"),
                 _operand(refs, dev, i32, (pages,), "cache.refs"), pages, rows, width, heads, d, block, _operand(missing, dev, i32, (1,), "cache.missing"))
    have = (desc, ctypes.byref(desc), dev, max(256, int(lib.cafeq_cache_pages_workspace_bytes(ctypes.byref(desc)))), at, {})
    object.__setattr__(c, "_desc", have)
    return have


def _starts(t, rows, dev, what="starts"):
    return _operand(t, dev, torch.int32, (rows + 1,), what)


def _bound(longest, n):
    """The bound on a sequence's rows as 64 bits hold it."""
    if longest is None:
        return n
    if longest < 0:
        raise CafeqError("longest must be 0 or more")
    return min(longest, n)


def cache_append(cache, k, v, starts, longest=None):
    """cafeq_cache_append: new keys and values [n][heads][d] into the pages of their sequences, in 8 bits.  starts int32 [sequences + 1]: the rows
    of each sequence, the last of its lengths' tokens; longest: an upper bound of a sequence's rows (n, if not given).  Behind a cache_reserve
    that found no room nothing is stored."""
    dev, kind = torch._C._cuda_getDevice(), _FLOATS.get(k.dtype)
    if kind is None or v.dtype is not k.dtype:
        raise CafeqError("k and v must be float32 or bfloat16, both the same")
    c, ref = _cache(cache, dev)[:2]
    n = k.shape[0]
    if k.shape != (n, c.heads, c.d) or v.shape != k.shape:
        raise CafeqError("k and v must be [n][%d][%d]" % (c.heads, c.d))
    (ldk, hsk), (ldv, hsv) = _head_rows(k, dev, "k"), _head_rows(v, dev, "v")
    ps = _starts(starts, c.sequences, dev)
    if n:
        rc = lib.cafeq_cache_append(ref, k.data_ptr(), v.data_ptr(), kind, n, ldk, hsk, ldv, hsv, ps, _bound(longest, n),
                                    torch._C._cuda_getCurrentRawStream(dev))
        if rc:
            _check(rc)


def cache_values(cache, begin, starts, n, dtype=torch.float32):
    """cafeq_cache_values: (k, v) [n][heads][d], the values of positions begin[i] .. of each sequence i in rows starts[i] .. starts[i + 1] - 1."""
    dev, kind = torch._C._cuda_getDevice(), _FLOATS.get(dtype)
    if kind is None:
        raise CafeqError("dtype must be float32 or bfloat16")
    c, ref = _cache(cache, dev)[:2]
    pb, ps = _operand(begin, dev, torch.int32, (c.sequences,), "begin"), _starts(starts, c.sequences, dev)
    k, v = (cache.k.new_empty((n, c.heads, c.d), dtype=dtype) for _ in range(2))
    if n:
        rc = lib.cafeq_cache_values(ref, pb, ps, n, k.data_ptr(), v.data_ptr(), kind, torch._C._cuda_getCurrentRawStream(dev))
        if rc:
            _check(rc)
    return k, v


def cache_attend(cache, q, starts, longest=None, scale=None, softcap=0.0, window=0, causal=True, lse=False, out=None):
    """cafeq_cache_attend: attention of new tokens q [n][heads_q][d] over the cache, which holds their keys and values already.  scale: d^-1/2 if
    not given; softcap, window: 0 for none; starts, longest as in cache_append.  Returns out, or (out, lse [n][heads_q]) with lse=True.  Behind a
    cache_reserve that found no room out is 0, lse -inf."""
    dev, kind = torch._C._cuda_getDevice(), _FLOATS.get(q.dtype)
    if kind is None:
        raise CafeqError("q must be float32 or bfloat16")
    c, ref, _, _, _, sizes = _cache(cache, dev)
    shape = q.shape
    n, hq, d = shape if len(shape) == 3 else (0, 0, 0)
    if d != c.d or hq < 1 or hq % c.heads:
        raise CafeqError("q must be [n][a multiple of %d][%d]" % (c.heads, c.d))
    if not 0 <= window < 1 << 31:
        raise CafeqError("window must be 0 .. 2^31 - 1")
    ldq, hsq = _head_rows(q, dev, "q")
    if out is None:
        out = torch.empty_strided((n, hq, d), (hq * d, d, 1), dtype=q.dtype, device=q.device)
        ldo, hso = hq * d, d
    else:
        if out.shape != shape or out.dtype is not q.dtype:
            raise CafeqError("out must have the shape and type of q")
        ldo, hso = _head_rows(out, dev, "out")
    sums = torch.empty((n, hq), dtype=torch.float32, device=q.device) if lse else None
    longest = _bound(longest, n)
    a = _pack_attention(q.data_ptr(), out.data_ptr(), 0 if sums is None else sums.data_ptr(), n, ldq, hsq, ldo, hso, longest,
                        _starts(starts, c.sequences, dev), kind, hq, 1 if causal else 0, window, d ** -0.5 if scale is None else scale, softcap)
    if n:
        stream = torch._C._cuda_getCurrentRawStream(dev)
        key = (kind, n, hq, longest, window, causal)
        nbytes = sizes.get(key)
        known = nbytes is not None
        if not known:
            nbytes = lib.cafeq_cache_attend_workspace_bytes(ref, a)
        # the buffer is of this call alone, so that streams share nothing
        ws = q.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
        rc = lib.cafeq_cache_attend(ref, a, _ptr(ws), stream)      # (held until the launch is made: another thread may allocate)
        if rc:
            _check(rc)
        if not known:      # of calls that are refused the size says nothing
            if len(sizes) > 63:
                sizes.clear()
            sizes[key] = nbytes
    return (out, sums) if lse else out


class Reserved(NamedTuple):
    """What cache_reserve returns: the positions of the new tokens, and how many pages or table columns lack (0: there is room)."""
    positions: torch.Tensor
    missing: torch.Tensor


def _pages_call(cache):
    dev = torch._C._cuda_getDevice()
    c, ref, _, nbytes, _, _ = _cache(cache, dev)
    return dev, c, ref, cache.k.new_empty(nbytes, dtype=torch.uint8), torch._C._cuda_getCurrentRawStream(dev)


def cache_reserve(cache, starts, n):
    """cafeq_cache_reserve: room for starts[i + 1] - starts[i] more tokens of each sequence, n in all.  Nothing waits: a caller that cannot be
    sure of room reads `missing` (one int32 on the device); where it is not 0 nothing has changed, positions are 0, and until a reserve finds room
    (for no token: starts of zeros) cache_append stores nothing and cache_attend returns zeros."""
    dev, c, ref, ws, stream = _pages_call(cache)
    positions, missing = cache.refs.new_empty(n), cache.refs.new_empty(1)
    rc = lib.cafeq_cache_reserve(ref, _starts(starts, c.sequences, dev), n, positions.data_ptr() if n else None, missing.data_ptr(), ws.data_ptr(), stream)
    if rc:
        _check(rc)
    return Reserved(positions, missing)


def cache_reorder(cache, sources):
    """cafeq_cache_reorder: row i takes over what row sources[i] held (int32 [sequences]; outside the rows: nothing, which lets its pages go)."""
    dev, c, ref, ws, stream = _pages_call(cache)
    _check(lib.cafeq_cache_reorder(ref, _operand(sources, dev, torch.int32, (c.sequences,), "sources"), ws.data_ptr(), stream))


def cache_compact(cache):
    """cafeq_cache_compact: pages in use move to the front of the pool.  Returns how many there are (int32 [1] on the device)."""
    dev, c, ref, ws, stream = _pages_call(cache)
    used = cache.refs.new_empty(1)
    _check(lib.cafeq_cache_compact(ref, used.data_ptr(), ws.data_ptr(), stream))
    return used
