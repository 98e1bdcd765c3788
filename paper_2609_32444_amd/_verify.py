"""The verification of drafted tokens of libcis.so (include/cis_verify.h). Argument checks and
marshalling only, as in ``_binding``."""

from __future__ import annotations

import ctypes

import torch

from . import _binding
from ._binding import _check_vec, _logits_args, _offsets, _ptr
from ._tokens import _Call, _dtype_code, _per_row, _SampleParams, _top_k

_vp, _i64 = ctypes.c_void_p, ctypes.c_int64
_int, _size = ctypes.c_int, ctypes.c_size_t

_DECLARED = None


def _lib() -> ctypes.CDLL:
    global _DECLARED
    lib = _binding.load_library()
    if _DECLARED is not lib:
        lib.cis_verify_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _int]
        lib.cis_verify_workspace_bytes.restype = _size
        lib.cis_verify.argtypes = [_vp, _int, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _i64,
                                   ctypes.POINTER(_SampleParams), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _size, _vp]
        lib.cis_verify.restype = _int
        _DECLARED = lib
    return lib


class VerifyCall(_Call):
    """Drafted tokens against the target's logits (cis_verify). Sequence s has the rows
    [seq_offsets[s], seq_offsets[s + 1]) of the target's logits [T, V]: one for each of its drafts and one
    more; the drafts of all sequences follow each other in draft_ids [D] int64 and draft_logits
    [D, V], or None for drafts without a distribution (copied from the prompt, say). u [T] float32 has
    a random number for each draft and, at its last row, for the sequence's draw.

    temperature, top_k, top_p and min_p are those of SampleCall, under which the drafts were drawn too:
    numbers, or tensors of one value per sequence. run() returns "ids" [T] int64 (the accepted drafts
    and the drawn token in each sequence's first rows, -1 behind them), "accepted" [n_seq] int32, "logp"
    (log softmax of the target's whole row at the id: the loss's logp_infer) and "logp_kept" (under the
    distribution that cis.sample would draw from), [T] float32."""

    def __init__(self, logits, draft_ids, u, seq_offsets, draft_logits=None, *, temperature=1.0,
                 top_k=0, top_p=1.0, min_p=0.0, V=None, workspace=None):
        dtype, T, V, ld = _logits_args(logits, V)
        dev = logits.device
        if not isinstance(draft_ids, torch.Tensor) or draft_ids.dim() != 1:
            raise ValueError("draft_ids must be a contiguous int64 [D] tensor")
        D = draft_ids.shape[0]
        _check_vec("draft_ids", draft_ids, D, torch.int64, dev)
        _check_vec("u", u, T, torch.float32, dev)
        if seq_offsets is None:
            raise ValueError("seq_offsets is required")
        offs, n_seq = _offsets(seq_offsets, T, dev)
        Dl, ld_d = 0, 0
        if draft_logits is not None:
            if draft_logits.dim() != 2 or draft_logits.dtype != logits.dtype \
                    or draft_logits.device != dev or draft_logits.shape[0] != D \
                    or draft_logits.shape[1] < V:
                raise ValueError(f"draft_logits must be a [{D}, >={V}] {logits.dtype} tensor on {dev}, "
                                 f"got {tuple(draft_logits.shape)} {draft_logits.dtype} on "
                                 f"{draft_logits.device}")
            _, Dl, _, ld_d = _logits_args(draft_logits, V)
        temperature, temps = _per_row("temperature", temperature, n_seq, torch.float32, dev)
        top_k, ks = _per_row("top_k", top_k, n_seq, torch.int32, dev)
        top_p, ps = _per_row("top_p", top_p, n_seq, torch.float32, dev)
        min_p, ms = _per_row("min_p", min_p, n_seq, torch.float32, dev)
        self._prm = _SampleParams(1.0 if temperature is None else float(temperature),
                                  0 if top_k is None else _top_k(top_k),
                                  1.0 if top_p is None else float(top_p),
                                  0.0 if min_p is None else float(min_p))
        self._keep = (logits, draft_logits, draft_ids, u, offs, temps, ks, ps, ms)
        self.out = {"ids": torch.empty(T, dtype=torch.int64, device=dev),
                    "accepted": torch.empty(n_seq, dtype=torch.int32, device=dev),
                    "logp": torch.empty(T, dtype=torch.float32, device=dev),
                    "logp_kept": torch.empty(T, dtype=torch.float32, device=dev)}
        _lib()   # (declares the entry point)
        # no drafts at all need no logits of theirs
        self._finish("cis_verify",
                     (_ptr(logits), dtype, T, V, ld, _ptr(draft_logits) if Dl else None, D, ld_d,
                      _ptr(draft_ids), _ptr(u), _ptr(offs), n_seq, ctypes.byref(self._prm),
                      _ptr(temps), _ptr(ks), _ptr(ps), _ptr(ms), _ptr(self.out["ids"]),
                      _ptr(self.out["accepted"]), _ptr(self.out["logp"]),
                      _ptr(self.out["logp_kept"])),
                     workspace, verify_workspace_bytes(T, Dl, n_seq, V, logits.dtype), dev)


def verify_workspace_bytes(T: int, D: int, n_seq: int, V: int, dtype=torch.bfloat16) -> int:
    """Bytes of workspace for T rows and D drafts that have logits (0 where they have none)."""
    return int(_lib().cis_verify_workspace_bytes(int(T), int(D), int(n_seq), int(V),
                                                 _dtype_code(dtype)))


def verify(logits, draft_ids, u, seq_offsets, draft_logits=None, *, temperature=1.0, top_k=0,
           top_p=1.0, min_p=0.0, V=None, workspace=None) -> dict:
    """A VerifyCall made and run once."""
    return VerifyCall(logits, draft_ids, u, seq_offsets, draft_logits, temperature=temperature,
                      top_k=top_k, top_p=top_p, min_p=min_p, V=V, workspace=workspace).run()
