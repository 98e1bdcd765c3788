"""The token operators of libcis.so (include/cis_tokens.h): sampling, a row's largest logits, and the
distillation loss. Argument checks and marshalling only, as in ``_binding``."""

from __future__ import annotations

import ctypes

import torch

from . import _binding
from ._binding import CisError, _check_vec, _logits_args, _mask_u8, _new_grad, _ptr, _stream

KL_FORWARD, KL_REVERSE = 0, 1   # cis_kl_t
TOP_MAX_K = 1024                # CIS_TOP_MAX_K

_vp, _i64, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float
_int, _size = ctypes.c_int, ctypes.c_size_t


class _SampleParams(ctypes.Structure):
    """cis_sample_params_t"""
    _fields_ = [("temperature", _f32), ("top_k", ctypes.c_int32), ("top_p", _f32),
                ("min_p", _f32)]


class _DistillParams(ctypes.Structure):
    """cis_distill_params_t"""
    _fields_ = [("kind", ctypes.c_int32), ("temperature", _f32), ("scale", _f32)]


_DECLARED = None


def _lib() -> ctypes.CDLL:
    global _DECLARED
    lib = _binding.load_library()
    if _DECLARED is not lib:
        lib.cis_sample_workspace_bytes.argtypes = [_i64, _i64, _int]
        lib.cis_sample_workspace_bytes.restype = _size
        lib.cis_sample.argtypes = [_vp, _int, _i64, _i64, _i64, _vp, _vp,
                                   ctypes.POINTER(_SampleParams), _vp, _vp, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _size, _vp]
        lib.cis_sample.restype = _int
        lib.cis_top_logits_workspace_bytes.argtypes = [_i64, _i64, _i64, _int]
        lib.cis_top_logits_workspace_bytes.restype = _size
        lib.cis_top_logits.argtypes = [_vp, _int, _i64, _i64, _i64, _vp, _i64, _f32, _vp, _vp, _vp,
                                       _vp, _size, _vp]
        lib.cis_top_logits.restype = _int
        lib.cis_distill_workspace_bytes.argtypes = [_i64, _i64, _i64, _int]
        lib.cis_distill_workspace_bytes.restype = _size
        head = [_vp, _int, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _vp,
                ctypes.POINTER(_DistillParams)]
        lib.cis_distill_fwd.argtypes = head + [_vp, _vp, _vp, _size, _vp]
        lib.cis_distill_fwd.restype = _int
        lib.cis_distill_bwd.argtypes = head + [_vp, _i64, _vp, _vp, _vp, _size, _vp]
        lib.cis_distill_bwd.restype = _int
        _DECLARED = lib
    return lib


class _Call:
    """A call with its outputs and workspace allocated up front: run() only launches, on torch's
    current stream, and reads the inputs as they are then."""

    def _finish(self, name, args, workspace, nbytes, dev):
        if workspace is None:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        elif workspace.device != dev or workspace.numel() * workspace.element_size() < nbytes:
            raise ValueError(f"workspace must hold {nbytes} bytes on {dev}")
        self.dev, self.workspace = dev, workspace
        self.out["workspace"] = workspace
        self._name, self._fn = name, getattr(_lib(), name)
        self._args = args + (_ptr(workspace), workspace.numel() * workspace.element_size())

    def run(self, stream=None) -> dict:
        if torch.cuda.current_device() == self.dev.index:
            rc = self._fn(*self._args, _stream(self.dev) if stream is None else stream)
        else:
            with torch.cuda.device(self.dev):
                rc = self._fn(*self._args, _stream(self.dev) if stream is None else stream)
        if rc != 0:
            raise CisError(self._name, rc)
        return self.out


def _per_row(name, x, T, dtype, dev):
    """A parameter as (value for every row, tensor of one per row): one of the two is None."""
    if isinstance(x, torch.Tensor) and x.dim() > 0:
        return None, _check_vec(name, x, T, dtype, dev)
    return x, None


def _top_k(k):
    """top_k as the library's int32: more than that is more than any row has, and a negative one stays
    one (a ctypes field takes the low bits of what does not fit)."""
    return max(-1, min(int(k), 2 ** 31 - 1))


class SampleCall(_Call):
    """One token per row of logits, drawn with the random numbers u [T] float32 (cis_sample).

    temperature, top_k, top_p and min_p are numbers, or tensors of one value per row (float32;
    top_k int32). run() returns "ids" [T] int64, "logp" (log softmax of the whole row at the id: the
    loss's logp_infer) and "logp_kept" (under the distribution that was drawn from), [T] float32.
    Rows that cannot be drawn from have id -1."""

    def __init__(self, logits, u, mask=None, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                 V=None, workspace=None):
        dtype, T, V, ld = _logits_args(logits, V)
        dev = logits.device
        _check_vec("u", u, T, torch.float32, dev)
        mask = _check_vec("mask", _mask_u8(mask), T, torch.uint8, dev, optional=True)
        temperature, temps = _per_row("temperature", temperature, T, torch.float32, dev)
        top_k, ks = _per_row("top_k", top_k, T, torch.int32, dev)
        top_p, ps = _per_row("top_p", top_p, T, torch.float32, dev)
        min_p, ms = _per_row("min_p", min_p, T, torch.float32, dev)
        self._prm = _SampleParams(1.0 if temperature is None else float(temperature),
                                  0 if top_k is None else _top_k(top_k),
                                  1.0 if top_p is None else float(top_p),
                                  0.0 if min_p is None else float(min_p))
        self._keep = (logits, u, mask, temps, ks, ps, ms)
        self.out = {"ids": torch.empty(T, dtype=torch.int64, device=dev),
                    "logp": torch.empty(T, dtype=torch.float32, device=dev),
                    "logp_kept": torch.empty(T, dtype=torch.float32, device=dev)}
        self._finish("cis_sample",
                     (_ptr(logits), dtype, T, V, ld, _ptr(u), _ptr(mask), ctypes.byref(self._prm),
                      _ptr(temps), _ptr(ks), _ptr(ps), _ptr(ms), _ptr(self.out["ids"]),
                      _ptr(self.out["logp"]), _ptr(self.out["logp_kept"])),
                     workspace, sample_workspace_bytes(T, V, logits.dtype), dev)


class TopLogitsCall(_Call):
    """The K largest logits of each row (cis_top_logits): run() returns "ids" [T, K] int32 and
    "values" [T, K] float32 in falling order (the lowest id first among equals; -1 and -inf past a
    row's last token) and "tail" [T] float32, the log-sum-exp of the other logits / temperature."""

    def __init__(self, logits, K, mask=None, *, temperature=1.0, V=None, workspace=None):
        dtype, T, V, ld = _logits_args(logits, V)
        dev, K = logits.device, int(K)
        if not 1 <= K <= TOP_MAX_K:
            raise ValueError(f"K must be in [1, {TOP_MAX_K}], got {K}")
        mask = _check_vec("mask", _mask_u8(mask), T, torch.uint8, dev, optional=True)
        self._keep = (logits, mask)
        self.out = {"ids": torch.empty(T, K, dtype=torch.int32, device=dev),
                    "values": torch.empty(T, K, dtype=torch.float32, device=dev),
                    "tail": torch.empty(T, dtype=torch.float32, device=dev)}
        self._finish("cis_top_logits",
                     (_ptr(logits), dtype, T, V, ld, _ptr(mask), K, float(temperature),
                      _ptr(self.out["ids"]), _ptr(self.out["values"]), _ptr(self.out["tail"])),
                     workspace, top_logits_workspace_bytes(T, V, K, logits.dtype), dev)


def _check_top(name, t, T, K, dtype, dev):
    if t.device != dev or t.dtype != dtype or t.dim() != 2 or t.shape[0] != T or t.shape[1] != K:
        raise ValueError(f"{name} must be a [{T}, {K}] {dtype} tensor on {dev}, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    if t.stride(1) != 1 and t.numel() > 0:
        raise ValueError(f"{name} must have unit column stride")


def _list_stride(ids, values, T, K):
    """Row stride of the lists, as the library takes it: K entries of a row never share storage
    with another row's. (That of a single row never moves an address.)"""
    if T <= 1:
        return K
    if ids.stride(0) != values.stride(0):
        raise ValueError("top_ids and top_values must have the same row stride")
    if ids.stride(0) < K:
        raise ValueError(f"the rows of top_ids and top_values must not share storage (expanded "
                         f"lists need a contiguous copy): row stride {ids.stride(0)}, K {K}")
    return ids.stride(0)


class DistillCall(_Call):
    """KL between a teacher's lists and the student's logits (cis_distill_fwd, or with bwd=True
    cis_distill_bwd). top_ids [T, K] int32 and top_values [T, K] float32 as TopLogitsCall leaves
    them, or the first columns of longer ones (of one row stride, K at least); tail [T] its tail, or None: the teacher is its list alone (KL_FORWARD only); row_weight [T]
    float32 or None. run() returns "terms" [T], "loss" [1] (their sum) and with bwd "dlogits"; the
    workspace holds the statistics (read_stats)."""

    def __init__(self, logits, top_ids, top_values, tail=None, row_weight=None, mask=None, *,
                 kind=KL_FORWARD, temperature=1.0, scale=1.0, bwd=True, V=None, dlogits=None,
                 workspace=None):
        dtype, T, V, ld = _logits_args(logits, V)
        dev = logits.device
        if top_ids.dim() != 2 or not 1 <= top_ids.shape[1] <= TOP_MAX_K:
            raise ValueError(f"top_ids must be [T, K] with K in [1, {TOP_MAX_K}], got "
                             f"{tuple(top_ids.shape)}")
        K = top_ids.shape[1]
        _check_top("top_ids", top_ids, T, K, torch.int32, dev)
        _check_top("top_values", top_values, T, K, torch.float32, dev)
        ld_top = _list_stride(top_ids, top_values, T, K)
        _check_vec("tail", tail, T, torch.float32, dev, optional=True)
        _check_vec("row_weight", row_weight, T, torch.float32, dev, optional=True)
        mask = _check_vec("mask", _mask_u8(mask), T, torch.uint8, dev, optional=True)
        self._prm = _DistillParams(int(kind), float(temperature), float(scale))
        self.out = {"terms": torch.empty(T, dtype=torch.float32, device=dev),
                    "loss": torch.empty(1, dtype=torch.float32, device=dev)}
        args = (_ptr(logits), dtype, T, V, ld, _ptr(top_ids), _ptr(top_values), K, ld_top,
                _ptr(tail), _ptr(row_weight), _ptr(mask), ctypes.byref(self._prm))
        if bwd:
            if dlogits is None:
                dlogits = _new_grad(T, V, logits)
            if dlogits.dtype != logits.dtype or dlogits.dim() != 2 or dlogits.stride(1) != 1 \
                    or dlogits.shape[0] != T or dlogits.shape[1] < V or dlogits.device != dev:
                raise ValueError("dlogits must be a [T, >=V] tensor like logits")
            # (the row stride of a single row never moves an address)
            args += (_ptr(dlogits), dlogits.stride(0) if T > 1 else ld)
            self.out["dlogits"] = dlogits
        self._keep = (logits, top_ids, top_values, tail, row_weight, mask)
        self._finish("cis_distill_bwd" if bwd else "cis_distill_fwd",
                     args + (_ptr(self.out["terms"]), _ptr(self.out["loss"])), workspace,
                     distill_workspace_bytes(T, V, K, logits.dtype), dev)


def _dtype_code(dtype):
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"dtype must be bfloat16 or float32, got {dtype}")
    return _binding.CIS_BF16 if dtype == torch.bfloat16 else _binding.CIS_F32


def sample_workspace_bytes(T: int, V: int, dtype=torch.bfloat16) -> int:
    return int(_lib().cis_sample_workspace_bytes(int(T), int(V), _dtype_code(dtype)))


def top_logits_workspace_bytes(T: int, V: int, K: int, dtype=torch.bfloat16) -> int:
    return int(_lib().cis_top_logits_workspace_bytes(int(T), int(V), int(K), _dtype_code(dtype)))


def distill_workspace_bytes(T: int, V: int, K: int, dtype=torch.bfloat16) -> int:
    return int(_lib().cis_distill_workspace_bytes(int(T), int(V), int(K), _dtype_code(dtype)))


def sample(logits, u, mask=None, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, V=None,
           workspace=None) -> dict:
    """A SampleCall made and run once."""
    return SampleCall(logits, u, mask, temperature=temperature, top_k=top_k, top_p=top_p,
                      min_p=min_p, V=V, workspace=workspace).run()


def top_logits(logits, K, mask=None, *, temperature=1.0, V=None, workspace=None) -> dict:
    """A TopLogitsCall made and run once."""
    return TopLogitsCall(logits, K, mask, temperature=temperature, V=V, workspace=workspace).run()


def distill_fwd(logits, top_ids, top_values, tail=None, row_weight=None, mask=None, *,
                kind=KL_FORWARD, temperature=1.0, scale=1.0, V=None, workspace=None) -> dict:
    """A forward DistillCall made and run once."""
    return DistillCall(logits, top_ids, top_values, tail, row_weight, mask, kind=kind,
                       temperature=temperature, scale=scale, bwd=False, V=V,
                       workspace=workspace).run()


def distill_bwd(logits, top_ids, top_values, tail=None, row_weight=None, mask=None, *,
                kind=KL_FORWARD, temperature=1.0, scale=1.0, V=None, dlogits=None,
                workspace=None) -> dict:
    """A DistillCall with its gradient made and run once."""
    return DistillCall(logits, top_ids, top_values, tail, row_weight, mask, kind=kind,
                       temperature=temperature, scale=scale, bwd=True, V=V, dlogits=dlogits,
                       workspace=workspace).run()
