"""The RMS norm of libcis.so (include/cis_norm.h), forward and backward. Argument checks and
marshalling only, as in ``_binding``."""

from __future__ import annotations

import ctypes

import torch

from . import _binding
from ._binding import CisError, _ptr, _stream

CIS_E4M3 = 2                    # beside cis_dtype_t
NORM_MAX_H = 1 << 22            # CIS_NORM_MAX_H
NORM_GROUPS = (0, 32, 64, 128)

_vp, _i64, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float
_int, _size = ctypes.c_int, ctypes.c_size_t


class _Rows(ctypes.Structure):
    """cis_rows_t"""
    _fields_ = [("data", _vp), ("dtype", ctypes.c_int32), ("stride_t", _i64), ("stride_n", _i64)]


_DECLARED = None


def _lib() -> ctypes.CDLL:
    global _DECLARED
    lib = _binding.load_library()
    if _DECLARED is not lib:
        rows = ctypes.POINTER(_Rows)
        lib.cis_rms_norm_fwd.argtypes = [_i64, _i64, _i64, rows, rows, _vp, _int, _f32, rows, rows,
                                         _vp, _i64, _vp]
        lib.cis_rms_norm_fwd.restype = _int
        lib.cis_rms_norm_workspace_bytes.argtypes = [_i64, _i64, _i64]
        lib.cis_rms_norm_workspace_bytes.restype = _size
        lib.cis_rms_norm_bwd.argtypes = [_i64, _i64, _i64, rows, rows, _vp, _int, _f32, rows, rows,
                                         _vp, _vp, _size, _vp]
        lib.cis_rms_norm_bwd.restype = _int
        _DECLARED = lib
    return lib


_CODES = {torch.bfloat16: _binding.CIS_BF16, torch.float32: _binding.CIS_F32,
          torch.float8_e4m3fn: CIS_E4M3}
_FULL = (torch.bfloat16, torch.float32)


def _shape(name, x):
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3):
        raise ValueError(f"{name} must be a [T, H] or [T, N, H] tensor")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not 1 <= x.shape[-1] <= NORM_MAX_H:
        raise ValueError(f"H must be in [1, {NORM_MAX_H}], got {x.shape[-1]}")
    if x.dim() == 3 and x.shape[1] < 1:
        raise ValueError("N must be at least 1")
    return tuple(x.shape)


def _rows(name, t, shape, dtypes, dev):
    """A tensor as the library takes it, or None."""
    if t is None:
        return None
    if tuple(t.shape) != shape or t.device != dev or t.dtype not in dtypes:
        raise ValueError(f"{name} must be a {list(shape)} tensor of {' or '.join(map(str, dtypes))} "
                         f"on {dev}, got {list(t.shape)} {t.dtype} on {t.device}")
    if shape[-1] > 1 and t.stride(-1) != 1 and t.numel() > 0:
        raise ValueError(f"{name} must have unit column stride")
    return _Rows(t.data_ptr(), _CODES[t.dtype], t.stride(0), t.stride(1) if t.dim() == 3 else 0)


def _check_weight(weight, H, dev):
    if weight is None:
        return 0
    if weight.device != dev or weight.dtype not in _FULL or weight.dim() != 1 \
            or weight.shape[0] != H or not weight.is_contiguous():
        raise ValueError(f"weight must be a contiguous [{H}] bfloat16 or float32 tensor on {dev}")
    return _CODES[weight.dtype]


def _new_rows(shape, dtype, dev):
    """Rows that start at whole 16-byte vectors."""
    per = 16 // dtype.itemsize
    ld = (shape[-1] + per - 1) // per * per
    return torch.empty(*shape[:-1], ld, dtype=dtype, device=dev)[..., :shape[-1]]


def _ref(rows):
    return None if rows is None else ctypes.byref(rows)


class _Call:
    """A call with its outputs allocated up front: run() only launches, on torch's current stream, and
    reads the inputs as they are then."""

    def _finish(self, name, args, dev):
        self.dev, self._name, self._fn, self._args = dev, name, getattr(_lib(), name), args

    def run(self, stream=None) -> dict:
        if torch.cuda.current_device() == self.dev.index:
            rc = self._fn(*self._args, _stream(self.dev) if stream is None else stream)
        else:
            with torch.cuda.device(self.dev):
                rc = self._fn(*self._args, _stream(self.dev) if stream is None else stream)
        if rc != 0:
            raise CisError(self._name, rc)
        return self.out


class RmsNormCall(_Call):
    """y = s * rstd * weight of the rows s = x + residual (cis_rms_norm_fwd). x is [T, H], or [T, N, H]
    (the heads of a packed projection: any strides of whole 16-byte vectors), in bfloat16 or float32;
    residual of x's type or float32, or None; weight [H] or None (ones). out_dtype is bfloat16,
    float32 (x's type by default) or float8_e4m3fn, with a scale per row or per `group` columns.

    run() returns "y", with a residual "residual" (s in the residual's type: the next layer's
    residual and what the backward pass takes), and with e4m3 "scale" [T(, N)] or
    [T(, N), ceil(H / group)] float32, y being about value * scale. y and residual_out give the outputs
    their place: buffers of their own, or an input; residual_out=False leaves the sum out."""

    def __init__(self, x, weight=None, residual=None, *, eps=1e-6, out_dtype=None, group=0, y=None,
                 residual_out=None):
        shape, dev = _shape("x", x), x.device
        H, group = shape[-1], int(group)
        if y is not None and out_dtype is None:
            out_dtype = y.dtype
        out_dtype = x.dtype if out_dtype is None else out_dtype
        if out_dtype not in _CODES:
            raise ValueError(f"out_dtype must be bfloat16, float32 or float8_e4m3fn, got {out_dtype}")
        e4m3 = out_dtype == torch.float8_e4m3fn
        if group not in NORM_GROUPS or (group and not e4m3):
            raise ValueError(f"group must be one of {NORM_GROUPS}, and 0 unless the output is "
                             f"float8_e4m3fn; got {group}")
        rx = _rows("x", x, shape, _FULL, dev)
        rr = _rows("residual", residual, shape, (x.dtype, torch.float32), dev)
        wdt = _check_weight(weight, H, dev)
        if residual is None and residual_out is not None and residual_out is not False:
            raise ValueError("residual_out needs a residual")
        y = _new_rows(shape, out_dtype, dev) if y is None else y
        self.out = {"y": y}
        rs = None
        if residual is not None and residual_out is not False:
            if residual_out is None:
                residual_out = _new_rows(shape, residual.dtype, dev)
            rs = _rows("residual_out", residual_out, shape, (residual.dtype,), dev)
            self.out["residual"] = residual_out
        ry = _rows("y", y, shape, (out_dtype,), dev)
        scale = None
        if e4m3:
            blocks = ((H + group - 1) // group,) if group else ()
            scale = torch.empty(*shape[:-1], *blocks, dtype=torch.float32, device=dev)
            self.out["scale"] = scale
        self._keep = (x, weight, residual, rx, rr, rs, ry)
        self._finish("cis_rms_norm_fwd",
                     (shape[0], shape[1] if len(shape) == 3 else 1, H, _ref(rx), _ref(rr),
                      _ptr(weight), wdt, float(eps), _ref(rs), _ref(ry), _ptr(scale), group), dev)


class RmsNormGradCall(_Call):
    """The gradients of a loss with respect to the rows that were normalised and to the weight
    (cis_rms_norm_bwd), from dy, that with respect to y (bfloat16 or float32: lmhead_loss_bwd's
    "dhidden" is float32). x is what was normalised: RmsNormCall's "residual", or its x where there
    was no residual. dresidual is the gradient that reaches those rows by themselves, or None, of dx's
    type (dx_dtype, or dresidual's, or x's).

    run() returns "dx" (the gradient of x and of the residual both) and, with dweight=True,
    "dweight" [H] float32. dx may be given its place: a buffer of its own, or an input."""

    def __init__(self, dy, x, weight=None, dresidual=None, *, eps=1e-6, dx_dtype=None, dx=None,
                 dweight=True, workspace=None):
        shape, dev = _shape("x", x), x.device
        T, N, H = shape[0], shape[1] if len(shape) == 3 else 1, shape[-1]
        if dx_dtype is None:
            dx_dtype = (dx if dx is not None else dresidual if dresidual is not None else x).dtype
        if dx_dtype not in _FULL:
            raise ValueError(f"dx_dtype must be bfloat16 or float32, got {dx_dtype}")
        rd = _rows("dy", dy, shape, _FULL, dev)
        rx = _rows("x", x, shape, _FULL, dev)
        wdt = _check_weight(weight, H, dev)
        rr = _rows("dresidual", dresidual, shape, (dx_dtype,), dev)
        dx = _new_rows(shape, dx_dtype, dev) if dx is None else dx
        rg = _rows("dx", dx, shape, (dx_dtype,), dev)
        self.out, dw, have = {"dx": dx}, None, 0
        if dweight:
            dw = torch.empty(H, dtype=torch.float32, device=dev)
            nbytes = rms_norm_workspace_bytes(T, N, H)
            if workspace is None:
                workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            have = workspace.numel() * workspace.element_size()
            if workspace.device != dev or have < nbytes:
                raise ValueError(f"workspace must hold {nbytes} bytes on {dev}")
            self.out["dweight"] = dw
        else:
            workspace = None
        self._keep = (dy, x, weight, dresidual, workspace, rd, rx, rr, rg)
        self._finish("cis_rms_norm_bwd",
                     (T, N, H, _ref(rd), _ref(rx), _ptr(weight), wdt, float(eps), _ref(rr), _ref(rg),
                      _ptr(dw), _ptr(workspace), have), dev)


def rms_norm_workspace_bytes(T: int, N: int, H: int) -> int:
    """Bytes of workspace for the backward pass with its weight's gradient."""
    return int(_lib().cis_rms_norm_workspace_bytes(int(T), int(N), int(H)))


def rms_norm(x, weight=None, residual=None, *, eps=1e-6, out_dtype=None, group=0, y=None,
             residual_out=None) -> dict:
    """A RmsNormCall made and run once."""
    return RmsNormCall(x, weight, residual, eps=eps, out_dtype=out_dtype, group=group, y=y,
                       residual_out=residual_out).run()


def rms_norm_bwd(dy, x, weight=None, dresidual=None, *, eps=1e-6, dx_dtype=None, dx=None,
                 dweight=True, workspace=None) -> dict:
    """A RmsNormGradCall made and run once."""
    return RmsNormGradCall(dy, x, weight, dresidual, eps=eps, dx_dtype=dx_dtype, dx=dx,
                           dweight=dweight, workspace=workspace).run()
