"""ctypes binding of libcafeq.so: argument marshalling only.

Every function takes torch CUDA tensors (used purely as device memory), builds the
C descriptors of include/cafeq.h and enqueues the call on torch's current stream.
There is no fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
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
