"""Thin ctypes binding of liblarsconv.so: same names as the C ABI, argument marshalling only.

Every function takes objects exposing ``data_ptr()`` (torch tensors on the GPU) or plain integer
addresses, passes them through and raises :class:`LarsConvError` on a non-zero status.  Nothing is
computed here, and there is no fallback: if the HIP library has not been built, loading fails.
"""
from __future__ import annotations

import ctypes
import operator
import os
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblarsconv.so")

LC_OK, LC_ERR_NULL, LC_ERR_SHAPE, LC_ERR_UNSUPPORTED, LC_ERR_WORKSPACE, LC_ERR_LAUNCH, LC_ERR_ALIGN = range(7)
LC_F32, LC_BF16 = 0, 1
LC_NCHW, LC_NHWC = 0, 1
LC_PASS_FWD, LC_PASS_BWD_DATA, LC_PASS_BWD_WEIGHT = 0, 1, 2

EXPORTS = ["conv2d_out_shape", "conv2d_workspace_bytes", "conv2d_fwd", "conv2d_bwd_data", "conv2d_bwd_weight",
           "conv2d_bwd_weight_sq_count", "conv2d_bwd_weight_sq",
           "lars_workspace_bytes", "lars_step", "lars_step_ex", "lars_step_pre", "lars_step_ex_static", "lars_poly_lr", "lars_warmup_poly_lr",
           "relu_fwd", "relu_bwd", "maxpool2x2_fwd", "maxpool2x2_bwd", "global_avgpool_fwd", "global_avgpool_bwd",
           "bias_add", "bias_grad", "softmax_xent", "maxpool_fwd", "maxpool_bwd", "relu_add_bwd",
           "batchnorm_workspace_bytes", "batchnorm_fwd", "batchnorm_bwd", "batchnorm_fwd_ex", "batchnorm_bwd_ex",
           "batchnorm_fwd_t", "batchnorm_bwd_t", "maxpool_fwd_t", "maxpool_bwd_t", "relu_add_bwd_t", "global_avgpool_fwd_t",
           "global_avgpool_bwd_t", "relu_add_bwd_bnsums_t", "relu_add_bwd_bnsums_grid_t", "batchnorm_bwd_presummed_t",
           "conv2d_fwd_stats_count", "conv2d_fwd_stats", "batchnorm_fwd_pre", "batchnorm_fwd_pair_t",
           "rmsnorm_fwd", "rmsnorm_fwd_q8", "rmsnorm_bwd_workspace_bytes", "rmsnorm_bwd",
           "token_logprob_workspace_bytes", "token_logprob_fwd", "token_logprob_bwd",
           "adamw_step", "adamw_step_q8",
           "lc_status_string", "lc_last_error_detail"]


class LarsConvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib().lc_last_error_detail().decode() if status == LC_ERR_LAUNCH else ""
        super().__init__(f"{where}: {status_string(status)} (lc_status {status})" + (f": {detail}" if detail else ""))


class lc_conv_desc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int) for f in
                ("n", "c", "h", "w", "k", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w", "dtype", "layout", "groups")]


@dataclass(frozen=True)
class ConvDesc:
    n: int
    c: int
    h: int
    w: int
    k: int
    r: int
    s: int
    stride_h: int = 1
    stride_w: int = 1
    pad_h: int = 0
    pad_w: int = 0
    dtype: int = LC_F32
    layout: int = LC_NHWC
    groups: int = 1

    def c_struct(self) -> lc_conv_desc:
        return lc_conv_desc(self.n, self.c, self.h, self.w, self.k, self.r, self.s, self.stride_h, self.stride_w,
                            self.pad_h, self.pad_w, self.dtype, self.layout, self.groups)


class lc_rmsnorm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("c", ctypes.c_int), ("x_ld", ctypes.c_int64), ("residual_ld", ctypes.c_int64),
                ("eps", ctypes.c_float), ("dtype", ctypes.c_int)]


class _Kept:
    """A descriptor that keeps its C structure (see _c): what copies and pickles of it leave out."""

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_c_ref"}


@dataclass(frozen=True)
class RmsNormDesc(_Kept):
    rows: int
    c: int
    x_ld: int = 0
    residual_ld: int = 0
    eps: float = 1e-5
    dtype: int = LC_F32

    def c_struct(self) -> lc_rmsnorm_desc:
        return lc_rmsnorm_desc(self.rows, self.c, self.x_ld, self.residual_ld, self.eps, self.dtype)


class lc_token_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("vocab", ctypes.c_int), ("ld", ctypes.c_int64), ("dtype", ctypes.c_int), ("top", ctypes.c_int)]


@dataclass(frozen=True)
class TokenDesc(_Kept):
    rows: int
    vocab: int
    ld: int = 0
    dtype: int = LC_F32
    top: int = 0

    def c_struct(self) -> lc_token_desc:
        return lc_token_desc(self.rows, self.vocab, self.ld, self.dtype, self.top)


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (run ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(python -m paper_1709_05011_amd.build); there is no CPU fallback")
        # torch ships its own HIP runtime (same soname as the system one).  It must be the one in the
        # process before this library is loaded, or device pointers and streams handed over by torch
        # would belong to another runtime instance than the one the kernels are launched with.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        dp = ctypes.POINTER(lc_conv_desc)
        L.conv2d_out_shape.restype = i32
        L.conv2d_out_shape.argtypes = [dp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.conv2d_workspace_bytes.restype = sz
        L.conv2d_workspace_bytes.argtypes = [dp, i32]
        for name in ("conv2d_fwd", "conv2d_bwd_data", "conv2d_bwd_weight"):
            fn = getattr(L, name)
            fn.restype = i32
            fn.argtypes = [dp, vp, vp, vp, vp, sz, vp]
        L.conv2d_bwd_weight_sq_count.restype = sz
        L.conv2d_bwd_weight_sq_count.argtypes = [dp]
        L.conv2d_bwd_weight_sq.restype = i32
        L.conv2d_bwd_weight_sq.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
        L.lars_step_pre.restype = i32
        L.lars_step_pre.argtypes = [i32, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                    vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.lars_workspace_bytes.restype = sz
        L.lars_workspace_bytes.argtypes = [i32, vp]
        L.lars_step.restype = i32
        L.lars_step.argtypes = [i32, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                vp, vp, vp, sz, vp]
        L.lars_step_ex.restype = i32
        L.lars_step_ex.argtypes = [i32, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                   vp, vp, vp, vp, vp, vp, sz, vp]
        L.lars_step_ex_static.restype = i32
        L.lars_step_ex_static.argtypes = [i32, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                          vp, vp, vp, vp, vp, vp]
        L.lars_poly_lr.restype = ctypes.c_float
        L.lars_poly_lr.argtypes = [ctypes.c_float, ctypes.c_int64, ctypes.c_int64, ctypes.c_float]
        L.lars_warmup_poly_lr.restype = ctypes.c_float
        L.lars_warmup_poly_lr.argtypes = [ctypes.c_float, ctypes.c_float, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                          ctypes.c_float]
        L.relu_fwd.argtypes = [vp, vp, sz, vp]
        L.relu_bwd.argtypes = [vp, vp, vp, sz, vp]
        L.maxpool2x2_fwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.maxpool2x2_bwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.global_avgpool_fwd.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp]
        L.global_avgpool_bwd.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp]
        L.bias_add.argtypes = [vp, vp, sz, i32, vp]
        L.bias_grad.argtypes = [vp, vp, sz, i32, vp]
        L.softmax_xent.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
        L.maxpool_fwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, vp]
        L.maxpool_bwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, vp]
        L.relu_add_bwd.argtypes = [vp, vp, vp, vp, sz, vp]
        for name in ("relu_fwd", "relu_bwd", "maxpool2x2_fwd", "maxpool2x2_bwd", "global_avgpool_fwd", "global_avgpool_bwd",
                     "bias_add", "bias_grad", "softmax_xent", "maxpool_fwd", "maxpool_bwd", "relu_add_bwd"):
            getattr(L, name).restype = i32
        L.batchnorm_workspace_bytes.restype = sz
        L.batchnorm_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        L.batchnorm_fwd.restype = i32
        L.batchnorm_fwd.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, ctypes.c_float, i32, vp, sz, vp]
        L.batchnorm_bwd.restype = i32
        L.batchnorm_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, sz, vp]
        L.batchnorm_fwd_ex.restype = i32
        L.batchnorm_fwd_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, ctypes.c_float, i32, i32, vp, sz, vp]
        L.batchnorm_bwd_ex.restype = i32
        L.batchnorm_bwd_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, sz, vp]
        L.batchnorm_fwd_t.restype = i32
        L.batchnorm_fwd_t.argtypes = [i32] + L.batchnorm_fwd_ex.argtypes
        L.batchnorm_bwd_t.restype = i32
        L.batchnorm_bwd_t.argtypes = [i32] + L.batchnorm_bwd_ex.argtypes
        for name in ("maxpool_fwd", "maxpool_bwd", "relu_add_bwd", "global_avgpool_fwd", "global_avgpool_bwd"):
            fn = getattr(L, name + "_t")
            fn.restype = i32
            fn.argtypes = [i32] + getattr(L, name).argtypes
        L.relu_add_bwd_bnsums_t.restype = i32
        L.relu_add_bwd_bnsums_t.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, sz, vp]
        L.relu_add_bwd_bnsums_grid_t.restype = i32
        L.relu_add_bwd_bnsums_grid_t.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, sz, vp]
        L.batchnorm_bwd_presummed_t.restype = i32
        L.batchnorm_bwd_presummed_t.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, sz, vp]
        L.conv2d_fwd_stats_count.restype = sz
        L.conv2d_fwd_stats_count.argtypes = [dp]
        L.conv2d_fwd_stats.restype = i32
        L.conv2d_fwd_stats.argtypes = [dp, vp, vp, vp, vp, vp, sz, vp]
        L.batchnorm_fwd_pair_t.restype = i32
        L.batchnorm_fwd_pair_t.argtypes = [i32, vp, vp, vp, vp, sz, vp, vp, vp, vp, sz, vp, vp, vp, vp, vp, i32, i32, i32, i32, ctypes.c_float,
                                           i32, i32, vp, sz, vp]
        L.batchnorm_fwd_pre.restype = i32
        L.batchnorm_fwd_pre.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, ctypes.c_float, i32, i32, vp, sz, vp, sz, vp]
        rp = ctypes.POINTER(lc_rmsnorm_desc)
        L.rmsnorm_fwd.restype = i32
        L.rmsnorm_fwd.argtypes = [rp, vp, vp, vp, vp, vp, vp, vp]
        L.rmsnorm_fwd_q8.restype = i32
        L.rmsnorm_fwd_q8.argtypes = [rp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.rmsnorm_bwd_workspace_bytes.restype = sz
        L.rmsnorm_bwd_workspace_bytes.argtypes = [rp]
        L.rmsnorm_bwd.restype = i32
        L.rmsnorm_bwd.argtypes = [rp, vp, ctypes.c_int64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        tp = ctypes.POINTER(lc_token_desc)
        L.token_logprob_workspace_bytes.restype = sz
        L.token_logprob_workspace_bytes.argtypes = [tp]
        L.token_logprob_fwd.restype = i32
        L.token_logprob_fwd.argtypes = [tp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.token_logprob_bwd.restype = i32
        L.token_logprob_bwd.argtypes = [tp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int64, vp]
        f32, f64, i64 = ctypes.c_float, ctypes.c_double, ctypes.c_int64
        L.adamw_step.restype = i32
        L.adamw_step.argtypes = [i32, vp, vp, i32, vp, vp, vp, f32, f64, f64, f32, f32, i64, vp, vp, vp, vp]
        L.adamw_step_q8.restype = i32
        L.adamw_step_q8.argtypes = [i32, vp, vp, i32, vp, vp, vp, vp, vp, f32, f64, f64, f32, f32, i64, ctypes.c_uint32, vp, vp, vp, vp]
        L.lc_status_string.restype = ctypes.c_char_p
        L.lc_status_string.argtypes = [i32]
        L.lc_last_error_detail.restype = ctypes.c_char_p
        L.lc_last_error_detail.argtypes = []
        _lib = L
    return _lib


def _ptr(obj) -> Optional[int]:
    if obj is None:
        return None
    try:
        return obj.data_ptr() or None
    except AttributeError:
        return operator.index(obj) or None            # (a whole number: a float is a value that was meant as one, not an address)


def _nbytes(ws) -> int:
    if ws is None:
        return 0
    return ws.numel() * ws.element_size()


_current_stream = None


def _first_current_stream() -> Optional[int]:
    """torch's current stream; once its runtime is up, later calls ask for the handle alone (0.1 us, where the stream object that holds it takes 2.9)."""
    global _current_stream
    import torch
    if torch.cuda.is_initialized():
        raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        _current_stream = lambda: raw(device()) or None
        return _current_stream()
    return torch.cuda.current_stream().cuda_stream or None


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() if _current_stream else _first_current_stream()
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream or None
    return int(stream) or None


def _desc(desc) -> lc_conv_desc:
    return desc.c_struct() if isinstance(desc, ConvDesc) else desc


def _check(status: int, where: str) -> None:
    if status != LC_OK:
        raise LarsConvError(status, where)


def status_string(status: int) -> str:
    return lib().lc_status_string(status).decode()


lc_status_string = status_string


def lc_last_error_detail() -> str:
    return lib().lc_last_error_detail().decode()


def conv2d_out_shape(desc):
    p, q = ctypes.c_int(), ctypes.c_int()
    _check(lib().conv2d_out_shape(ctypes.byref(_desc(desc)), ctypes.byref(p), ctypes.byref(q)), "conv2d_out_shape")
    return p.value, q.value


def conv2d_workspace_bytes(desc, pass_: int) -> int:
    return int(lib().conv2d_workspace_bytes(ctypes.byref(_desc(desc)), pass_))


def conv2d_fwd(desc, x, w, y, workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().conv2d_fwd(ctypes.byref(_desc(desc)), _ptr(x), _ptr(w), _ptr(y), _ptr(workspace), nb, _stream(stream)),
           "conv2d_fwd")


def conv2d_bwd_data(desc, dy, w, dx, workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().conv2d_bwd_data(ctypes.byref(_desc(desc)), _ptr(dy), _ptr(w), _ptr(dx), _ptr(workspace), nb,
                                 _stream(stream)), "conv2d_bwd_data")


def conv2d_bwd_weight(desc, x, dy, dw, workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().conv2d_bwd_weight(ctypes.byref(_desc(desc)), _ptr(x), _ptr(dy), _ptr(dw), _ptr(workspace), nb,
                                   _stream(stream)), "conv2d_bwd_weight")


def conv2d_bwd_weight_sq_count(desc) -> int:
    return int(lib().conv2d_bwd_weight_sq_count(ctypes.byref(_desc(desc))))


def conv2d_bwd_weight_sq(desc, x, dy, dw, dw_sq_pieces, workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().conv2d_bwd_weight_sq(ctypes.byref(_desc(desc)), _ptr(x), _ptr(dy), _ptr(dw), _ptr(dw_sq_pieces), _ptr(workspace),
                                      nb, _stream(stream)), "conv2d_bwd_weight_sq")


def _i64_array(vals: Sequence[int]):
    return (ctypes.c_int64 * max(len(vals), 1))(*vals)


def _ptr_array(objs: Sequence):
    return (ctypes.c_void_p * max(len(objs), 1))(*[_ptr(o) for o in objs])


def lars_workspace_bytes(numel: Sequence[int]) -> int:
    return int(lib().lars_workspace_bytes(len(numel), _i64_array(list(numel))))


class LarsArgs:
    """Host-side pointer and size arrays of one parameter list, marshalled once and reusable."""

    def __init__(self, w: Sequence, g: Sequence, v: Sequence, numel: Optional[Sequence[int]] = None,
                 w_lowp: Optional[Sequence] = None):
        if numel is None:
            numel = [t.numel() for t in w]
        self.n = len(w)
        self.numel = list(numel)
        self.w, self.g, self.v = _ptr_array(w), _ptr_array(g), _ptr_array(v)
        self.numel_arr = _i64_array(self.numel)
        self.w_lowp = _ptr_array(w_lowp) if w_lowp is not None else None
        self._keep = (list(w), list(g), list(v), list(w_lowp) if w_lowp is not None else None)


def lars_step(args: LarsArgs, eta: float, momentum: float, weight_decay: float, lr: float, trust_out=None,
              workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().lars_step(args.n, args.w, args.g, args.v, args.numel_arr, eta, momentum, weight_decay, lr,
                           _ptr(trust_out), args.w_lowp, _ptr(workspace), nb, _stream(stream)), "lars_step")


def _per_tensor_arrays(args: "LarsArgs", eta_per_tensor, weight_decay_per_tensor, skip):
    def farr(a):
        if a is None:
            return None
        if len(a) != args.n:
            raise ValueError("per-tensor array of the wrong length")
        return (ctypes.c_float * max(args.n, 1))(*[float(x) for x in a])
    if skip is not None and len(skip) != args.n:
        raise ValueError("skip list of the wrong length")
    sk = None if skip is None else (ctypes.c_uint8 * max(args.n, 1))(*[1 if x else 0 for x in skip])
    return farr(eta_per_tensor), farr(weight_decay_per_tensor), sk


def lars_step_ex(args: LarsArgs, eta: float, momentum: float, weight_decay: float, lr: float, eta_per_tensor=None,
                 weight_decay_per_tensor=None, skip=None, trust_out=None, workspace=None, stream=None,
                 workspace_bytes: Optional[int] = None) -> None:
    """lars_step with per-tensor coefficients (sequences of floats or None) and a skip list (sequence of 0/1 or None)."""
    e, b, sk = _per_tensor_arrays(args, eta_per_tensor, weight_decay_per_tensor, skip)
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().lars_step_ex(args.n, args.w, args.g, args.v, args.numel_arr, eta, momentum, weight_decay, lr, e, b, sk,
                              _ptr(trust_out), args.w_lowp, _ptr(workspace), nb, _stream(stream)), "lars_step_ex")


def lars_step_pre(args: LarsArgs, eta: float, momentum: float, weight_decay: float, lr: float, g_sq_pieces: Sequence,
                  g_sq_counts: Sequence[int], eta_per_tensor=None, weight_decay_per_tensor=None, skip=None, trust_out=None,
                  workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    """lars_step_ex with sum g^2 of some tensors handed over in pieces (None / 0 entries: computed from g)."""
    if len(g_sq_pieces) != args.n or len(g_sq_counts) != args.n:
        raise ValueError("per-tensor array of the wrong length")
    e, b, sk = _per_tensor_arrays(args, eta_per_tensor, weight_decay_per_tensor, skip)
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().lars_step_pre(args.n, args.w, args.g, args.v, args.numel_arr, eta, momentum, weight_decay, lr, e, b, sk,
                               _ptr_array(g_sq_pieces), _i64_array([int(c) for c in g_sq_counts]), _ptr(trust_out), args.w_lowp,
                               _ptr(workspace), nb, _stream(stream)), "lars_step_pre")


LARS_STATIC_SCRATCH_BYTES = 2 << 20


def lars_step_ex_static(args: LarsArgs, eta: float, momentum: float, weight_decay: float, lr: float, eta_per_tensor=None,
                        weight_decay_per_tensor=None, skip=None, trust_out=None, stream=None) -> None:
    """lars_step_ex on the library's own fixed scratch array (no workspace argument, nothing allocated)."""
    e, b, sk = _per_tensor_arrays(args, eta_per_tensor, weight_decay_per_tensor, skip)
    _check(lib().lars_step_ex_static(args.n, args.w, args.g, args.v, args.numel_arr, eta, momentum, weight_decay, lr, e, b, sk,
                                     _ptr(trust_out), args.w_lowp, _stream(stream)), "lars_step_ex_static")


def lars_poly_lr(base_lr: float, it: int, max_iter: int, power: float = 2.0) -> float:
    return float(lib().lars_poly_lr(base_lr, it, max_iter, power))


def lars_warmup_poly_lr(base_lr: float, start_lr: float, it: int, warmup_iters: int, max_iter: int, power: float = 2.0) -> float:
    return float(lib().lars_warmup_poly_lr(base_lr, start_lr, it, warmup_iters, max_iter, power))


# ---- glue layers of the small whole-path network (argument marshalling only) ----

def relu_fwd(x, y, count: int, stream=None) -> None:
    _check(lib().relu_fwd(_ptr(x), _ptr(y), count, _stream(stream)), "relu_fwd")


def relu_bwd(x, dy, dx, count: int, stream=None) -> None:
    _check(lib().relu_bwd(_ptr(x), _ptr(dy), _ptr(dx), count, _stream(stream)), "relu_bwd")


def maxpool2x2_fwd(x, y, idx, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().maxpool2x2_fwd(_ptr(x), _ptr(y), _ptr(idx), n, c, h, w, layout, _stream(stream)), "maxpool2x2_fwd")


def maxpool2x2_bwd(dy, idx, dx, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().maxpool2x2_bwd(_ptr(dy), _ptr(idx), _ptr(dx), n, c, h, w, layout, _stream(stream)), "maxpool2x2_bwd")


def global_avgpool_fwd(x, y, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().global_avgpool_fwd(_ptr(x), _ptr(y), n, c, h, w, layout, _stream(stream)), "global_avgpool_fwd")


def global_avgpool_bwd(dy, dx, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().global_avgpool_bwd(_ptr(dy), _ptr(dx), n, c, h, w, layout, _stream(stream)), "global_avgpool_bwd")


def bias_add(y, b, rows: int, k: int, stream=None) -> None:
    _check(lib().bias_add(_ptr(y), _ptr(b), rows, k, _stream(stream)), "bias_add")


def bias_grad(dy, db, rows: int, k: int, stream=None) -> None:
    _check(lib().bias_grad(_ptr(dy), _ptr(db), rows, k, _stream(stream)), "bias_grad")


def softmax_xent(logits, labels, loss, dlogits, row_scratch, n: int, k: int, stream=None) -> None:
    _check(lib().softmax_xent(_ptr(logits), _ptr(labels), _ptr(loss), _ptr(dlogits), _ptr(row_scratch), n, k, _stream(stream)),
           "softmax_xent")


def maxpool_fwd(x, y, idx, n: int, c: int, h: int, w: int, window: int, stride: int, pad: int, layout: int, stream=None) -> None:
    _check(lib().maxpool_fwd(_ptr(x), _ptr(y), _ptr(idx), n, c, h, w, window, stride, pad, layout, _stream(stream)), "maxpool_fwd")


def maxpool_bwd(dy, idx, dx, n: int, c: int, h: int, w: int, window: int, stride: int, pad: int, layout: int, stream=None) -> None:
    _check(lib().maxpool_bwd(_ptr(dy), _ptr(idx), _ptr(dx), n, c, h, w, window, stride, pad, layout, _stream(stream)), "maxpool_bwd")


def relu_add_bwd(y, da, db, dx, count: int, stream=None) -> None:
    _check(lib().relu_add_bwd(_ptr(y), _ptr(da), _ptr(db), _ptr(dx), count, _stream(stream)), "relu_add_bwd")


# ---- batch normalisation (training mode) ----

def batchnorm_workspace_bytes(n: int, c: int, h: int, w: int, layout: int) -> int:
    return int(lib().batchnorm_workspace_bytes(n, c, h, w, layout))


def batchnorm_fwd(x, gamma, beta, y, save_mean, save_invstd, n: int, c: int, h: int, w: int, eps: float, layout: int,
                  workspace=None, stream=None) -> None:
    _check(lib().batchnorm_fwd(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(y), _ptr(save_mean), _ptr(save_invstd), n, c, h, w, eps,
                               layout, _ptr(workspace), _nbytes(workspace), _stream(stream)), "batchnorm_fwd")


def batchnorm_bwd(x, dy, gamma, save_mean, save_invstd, dx, dgamma, dbeta, n: int, c: int, h: int, w: int, layout: int,
                  workspace=None, stream=None) -> None:
    _check(lib().batchnorm_bwd(_ptr(x), _ptr(dy), _ptr(gamma), _ptr(save_mean), _ptr(save_invstd), _ptr(dx), _ptr(dgamma),
                               _ptr(dbeta), n, c, h, w, layout, _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "batchnorm_bwd")


def batchnorm_fwd_ex(x, gamma, beta, residual, y, save_mean, save_invstd, n: int, c: int, h: int, w: int, eps: float, relu: bool,
                     layout: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_fwd_ex(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(residual), _ptr(y), _ptr(save_mean), _ptr(save_invstd),
                                  n, c, h, w, eps, int(bool(relu)), layout, _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "batchnorm_fwd_ex")


def batchnorm_bwd_ex(x, dy, gamma, beta, save_mean, save_invstd, dx, dgamma, dbeta, n: int, c: int, h: int, w: int, relu: bool,
                     layout: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_bwd_ex(_ptr(x), _ptr(dy), _ptr(gamma), _ptr(beta), _ptr(save_mean), _ptr(save_invstd), _ptr(dx),
                                  _ptr(dgamma), _ptr(dbeta), n, c, h, w, int(bool(relu)), layout, _ptr(workspace),
                                  _nbytes(workspace), _stream(stream)), "batchnorm_bwd_ex")


# ---- the same layers with the storage type as an argument (LC_BF16: NHWC, channels a multiple of 8) ----

def batchnorm_fwd_t(dtype: int, x, gamma, beta, residual, y, save_mean, save_invstd, n: int, c: int, h: int, w: int, eps: float,
                    relu: bool, layout: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_fwd_t(dtype, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(residual), _ptr(y), _ptr(save_mean),
                                 _ptr(save_invstd), n, c, h, w, eps, int(bool(relu)), layout, _ptr(workspace), _nbytes(workspace),
                                 _stream(stream)), "batchnorm_fwd_t")


def batchnorm_bwd_t(dtype: int, x, dy, gamma, beta, save_mean, save_invstd, dx, dgamma, dbeta, n: int, c: int, h: int, w: int,
                    relu: bool, layout: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_bwd_t(dtype, _ptr(x), _ptr(dy), _ptr(gamma), _ptr(beta), _ptr(save_mean), _ptr(save_invstd), _ptr(dx),
                                 _ptr(dgamma), _ptr(dbeta), n, c, h, w, int(bool(relu)), layout, _ptr(workspace),
                                 _nbytes(workspace), _stream(stream)), "batchnorm_bwd_t")


def maxpool_fwd_t(dtype: int, x, y, idx, n: int, c: int, h: int, w: int, window: int, stride: int, pad: int, layout: int,
                  stream=None) -> None:
    _check(lib().maxpool_fwd_t(dtype, _ptr(x), _ptr(y), _ptr(idx), n, c, h, w, window, stride, pad, layout, _stream(stream)),
           "maxpool_fwd_t")


def maxpool_bwd_t(dtype: int, dy, idx, dx, n: int, c: int, h: int, w: int, window: int, stride: int, pad: int, layout: int,
                  stream=None) -> None:
    _check(lib().maxpool_bwd_t(dtype, _ptr(dy), _ptr(idx), _ptr(dx), n, c, h, w, window, stride, pad, layout, _stream(stream)),
           "maxpool_bwd_t")


def relu_add_bwd_t(dtype: int, y, da, db, dx, count: int, stream=None) -> None:
    _check(lib().relu_add_bwd_t(dtype, _ptr(y), _ptr(da), _ptr(db), _ptr(dx), count, _stream(stream)), "relu_add_bwd_t")


def global_avgpool_fwd_t(dtype: int, x, y, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().global_avgpool_fwd_t(dtype, _ptr(x), _ptr(y), n, c, h, w, layout, _stream(stream)), "global_avgpool_fwd_t")


def global_avgpool_bwd_t(dtype: int, dy, dx, n: int, c: int, h: int, w: int, layout: int, stream=None) -> None:
    _check(lib().global_avgpool_bwd_t(dtype, _ptr(dy), _ptr(dx), n, c, h, w, layout, _stream(stream)), "global_avgpool_bwd_t")


# ---- the gradient at a block's output together with the sums of the batch-norm backward pass behind it ----

def relu_add_bwd_bnsums_t(dtype: int, y, da, db, dx, x_bn, save_mean, save_invstd, n: int, c: int, h: int, w: int, layout: int,
                          workspace=None, stream=None) -> None:
    _check(lib().relu_add_bwd_bnsums_t(dtype, _ptr(y), _ptr(da), _ptr(db), _ptr(dx), _ptr(x_bn), _ptr(save_mean), _ptr(save_invstd),
                                       n, c, h, w, layout, _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "relu_add_bwd_bnsums_t")


def relu_add_bwd_bnsums_grid_t(dtype: int, y, da, db, dx, x_bn, save_mean, save_invstd, n: int, c: int, h: int, w: int, grad_stride: int,
                               layout: int, workspace=None, stream=None) -> None:
    _check(lib().relu_add_bwd_bnsums_grid_t(dtype, _ptr(y), _ptr(da), _ptr(db), _ptr(dx), _ptr(x_bn), _ptr(save_mean),
                                            _ptr(save_invstd), n, c, h, w, grad_stride, layout, _ptr(workspace), _nbytes(workspace),
                                            _stream(stream)),
           "relu_add_bwd_bnsums_grid_t")


def batchnorm_bwd_presummed_t(dtype: int, x, dy, gamma, save_mean, save_invstd, dx, dgamma, dbeta, n: int, c: int, h: int, w: int,
                              layout: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_bwd_presummed_t(dtype, _ptr(x), _ptr(dy), _ptr(gamma), _ptr(save_mean), _ptr(save_invstd), _ptr(dx),
                                           _ptr(dgamma), _ptr(dbeta), n, c, h, w, layout, _ptr(workspace), _nbytes(workspace),
                                           _stream(stream)), "batchnorm_bwd_presummed_t")
# ---- batch-norm statistics out of the convolution's epilogue ----

def conv_route(desc, which: int, stats: bool = False, form: bool = False) -> str:
    """The kernel a pass of a layer ends in, in the library's words (host only; for tests and labels, not part of the C ABI)."""
    fn = lib().lc_selftest_conv_route
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(lc_conv_desc), ctypes.c_int, ctypes.c_int, ctypes.c_char_p, ctypes.c_size_t]
    text = ctypes.create_string_buffer(96)
    _check(fn(ctypes.byref(_desc(desc)), which, int(stats) + 2 * form, text, 96), "conv_route")
    return text.value.decode()


def conv2d_fwd_stats_count(desc) -> int:
    return int(lib().conv2d_fwd_stats_count(ctypes.byref(_desc(desc))))


def conv2d_fwd_stats(desc, x, w, y, stats, workspace=None, stream=None, workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().conv2d_fwd_stats(ctypes.byref(_desc(desc)), _ptr(x), _ptr(w), _ptr(y), _ptr(stats), _ptr(workspace), nb,
                                  _stream(stream)), "conv2d_fwd_stats")


def batchnorm_fwd_pair_t(dtype: int, x, gamma, beta, stats, stats_tiles: int, x2, gamma2, beta2, stats2, stats_tiles2: int, y, save_mean,
                         save_invstd, save_mean2, save_invstd2, n: int, c: int, h: int, w: int, eps: float, relu: bool, layout: int,
                         workspace, stream=None) -> None:
    _check(lib().batchnorm_fwd_pair_t(dtype, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(stats), stats_tiles, _ptr(x2), _ptr(gamma2), _ptr(beta2),
                                      _ptr(stats2), stats_tiles2, _ptr(y), _ptr(save_mean), _ptr(save_invstd), _ptr(save_mean2),
                                      _ptr(save_invstd2), n, c, h, w, eps, int(bool(relu)), layout, _ptr(workspace), _nbytes(workspace),
                                      _stream(stream)), "batchnorm_fwd_pair_t")


def batchnorm_fwd_pre(dtype: int, x, gamma, beta, residual, y, save_mean, save_invstd, n: int, c: int, h: int, w: int, eps: float,
                      relu: bool, layout: int, stats, stats_tiles: int, workspace=None, stream=None) -> None:
    _check(lib().batchnorm_fwd_pre(dtype, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(residual), _ptr(y), _ptr(save_mean),
                                   _ptr(save_invstd), n, c, h, w, eps, int(bool(relu)), layout, _ptr(stats), stats_tiles,
                                   _ptr(workspace), _nbytes(workspace), _stream(stream)), "batchnorm_fwd_pre")


# ---- the output side of a token model: RMS norm with the residual's addition ----

def _c(desc):
    """The C structure of a descriptor (made once for each: descriptors do not change), or of a structure as it is."""
    if isinstance(desc, ctypes.Structure):
        return ctypes.byref(desc)
    made = desc.__dict__.get("_c_ref")
    if made is None:
        made = ctypes.byref(desc.c_struct())
        object.__setattr__(desc, "_c_ref", made)
    return made


def rmsnorm_fwd(desc, x, residual, gamma, total, y, save_rstd=None, stream=None) -> None:
    _check(lib().rmsnorm_fwd(_c(desc), _ptr(x), _ptr(residual), _ptr(gamma), _ptr(total), _ptr(y), _ptr(save_rstd), _stream(stream)),
           "rmsnorm_fwd")


def rmsnorm_fwd_q8(desc, x, residual, gamma, total, y8, scales, group: int = 0, save_rstd=None, stream=None) -> None:
    _check(lib().rmsnorm_fwd_q8(_c(desc), _ptr(x), _ptr(residual), _ptr(gamma), _ptr(total), _ptr(y8), _ptr(scales), group,
                                _ptr(save_rstd), _stream(stream)), "rmsnorm_fwd_q8")


def rmsnorm_bwd_workspace_bytes(desc) -> int:
    return int(lib().rmsnorm_bwd_workspace_bytes(_c(desc)))


def rmsnorm_bwd(desc, total, dy, dtotal, gamma, save_rstd, dx, dgamma, workspace=None, h_ld: int = 0, stream=None,
                workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().rmsnorm_bwd(_c(desc), _ptr(total), h_ld, _ptr(dy), _ptr(dtotal), _ptr(gamma), _ptr(save_rstd), _ptr(dx),
                             _ptr(dgamma), _ptr(workspace), nb, _stream(stream)), "rmsnorm_bwd")


# ---- log probabilities of given tokens, entropy, likeliest alternatives ----

def token_logprob_workspace_bytes(desc) -> int:
    return int(lib().token_logprob_workspace_bytes(_c(desc)))


def token_logprob_fwd(desc, logits, tokens, logprob, entropy=None, lse=None, top_tokens=None, top_logprobs=None, workspace=None, stream=None,
                      workspace_bytes: Optional[int] = None) -> None:
    nb = _nbytes(workspace) if workspace_bytes is None else workspace_bytes
    _check(lib().token_logprob_fwd(_c(desc), _ptr(logits), _ptr(tokens), _ptr(logprob), _ptr(entropy), _ptr(lse), _ptr(top_tokens),
                                   _ptr(top_logprobs), _ptr(workspace), nb, _stream(stream)), "token_logprob_fwd")


def token_logprob_bwd(desc, logits, tokens, lse, entropy, dlogprob, dentropy, dlogits, dlogits_ld: int = 0, stream=None) -> None:
    _check(lib().token_logprob_bwd(_c(desc), _ptr(logits), _ptr(tokens), _ptr(lse), _ptr(entropy), _ptr(dlogprob), _ptr(dentropy),
                                   _ptr(dlogits), dlogits_ld, _stream(stream)), "token_logprob_bwd")


# ---- AdamW over a list of tensors ----

ADAMW_Q8_BLOCK = 256


class AdamWArgs:
    """Host-side pointer and size arrays of one parameter list (fp32 states), marshalled once and reusable.  The entry points take addresses: lists of tensors are checked here (as
    many of each, their types, contiguous, as many elements as the list says, one device); plain addresses are taken as they are."""
    _state = ("torch.float32",)

    def __init__(self, w: Sequence, g: Sequence, m: Sequence, v: Sequence, numel: Optional[Sequence[int]] = None,
                 w_lowp: Optional[Sequence] = None, g_dtype: int = LC_F32):
        if numel is None:
            numel = [t.numel() for t in w]
        self.n, self.numel, self.g_dtype = len(w), list(numel), g_dtype
        if len(self.numel) != self.n:
            raise ValueError(f"{len(self.numel)} sizes for {self.n} tensors")
        self._check("w", w, ("torch.float32",))
        self._check("g", g, ("torch.bfloat16" if g_dtype == LC_BF16 else "torch.float32",))
        self._check("m", m, self._state)
        self._check("v", v, self._state)
        if w_lowp is not None:
            self._check("w_lowp", w_lowp, ("torch.bfloat16",))
        self.w, self.g, self.m, self.v = _ptr_array(w), _ptr_array(g), _ptr_array(m), _ptr_array(v)
        self.numel_arr = _i64_array(self.numel)
        self.w_lowp = _ptr_array(w_lowp) if w_lowp is not None else None
        self._keep = [list(a) for a in (w, g, m, v, w_lowp or [])]

    def _check(self, name: str, tensors: Sequence, types: Sequence[str], per: int = 1) -> None:
        if len(tensors) != self.n:
            raise ValueError(f"{name}: {len(tensors)} tensors for {self.n} of w")
        for i, t in enumerate(tensors):
            if not hasattr(t, "data_ptr"):
                continue
            need = -(-self.numel[i] // per)
            self._device = getattr(self, "_device", t.device)
            if str(t.dtype) not in types or not t.is_contiguous() or t.numel() < need or t.device != self._device:
                raise ValueError(f"{name}[{i}]: a contiguous tensor of {' or '.join(types)} with {need} elements on {self._device} is needed, got {t.dtype} {tuple(t.shape)} "
                                 f"with strides {t.stride()} on {t.device}")


class AdamWQ8Args(AdamWArgs):
    """The same with the states in 8 bits (bytes) and a scale for every ADAMW_Q8_BLOCK elements."""
    _state = ("torch.uint8", "torch.float8_e4m3fn", "torch.float8_e5m2")

    def __init__(self, w: Sequence, g: Sequence, m: Sequence, m_scale: Sequence, v: Sequence, v_scale: Sequence,
                 numel: Optional[Sequence[int]] = None, w_lowp: Optional[Sequence] = None, g_dtype: int = LC_F32):
        super().__init__(w, g, m, v, numel, w_lowp, g_dtype)
        self._check("m_scale", m_scale, ("torch.float32",), ADAMW_Q8_BLOCK)
        self._check("v_scale", v_scale, ("torch.float32",), ADAMW_Q8_BLOCK)
        self.m_scale, self.v_scale = _ptr_array(m_scale), _ptr_array(v_scale)
        self._keep += [list(m_scale), list(v_scale)]


def _decays(args: AdamWArgs, weight_decay_per_tensor):
    if weight_decay_per_tensor is None:
        return None
    if len(weight_decay_per_tensor) != args.n:
        raise ValueError("per-tensor array of the wrong length")
    return (ctypes.c_float * max(args.n, 1))(*[float(x) for x in weight_decay_per_tensor])


def _one_float(grad_scale):
    if hasattr(grad_scale, "data_ptr") and not (grad_scale.numel() == 1 and grad_scale.element_size() == 4 and grad_scale.is_floating_point()):
        raise ValueError(f"grad_scale: one float is needed, got {grad_scale.dtype} {tuple(grad_scale.shape)}")
    return _ptr(grad_scale)


def adamw_step(args: AdamWArgs, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, step: int,
               weight_decay_per_tensor=None, grad_scale=None, stream=None) -> None:
    _check(lib().adamw_step(args.n, args.w, args.g, args.g_dtype, args.m, args.v, args.numel_arr, lr, beta1, beta2, eps, weight_decay, step,
                            _decays(args, weight_decay_per_tensor), _one_float(grad_scale), args.w_lowp, _stream(stream)), "adamw_step")


def adamw_step_q8(args: AdamWQ8Args, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, step: int, seed: int,
                  weight_decay_per_tensor=None, grad_scale=None, stream=None) -> None:
    _check(lib().adamw_step_q8(args.n, args.w, args.g, args.g_dtype, args.m, args.m_scale, args.v, args.v_scale, args.numel_arr, lr, beta1, beta2,
                               eps, weight_decay, step, seed & 0xFFFFFFFF, _decays(args, weight_decay_per_tensor), _one_float(grad_scale), args.w_lowp,
                               _stream(stream)), "adamw_step_q8")
