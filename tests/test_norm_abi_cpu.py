"""The RMS norm's C ABI on the host: every declared entry point is there, and bad arguments are
rejected before a device is touched. No kernel is launched here."""

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2609_32444_amd as cis
from paper_2609_32444_amd import _norm
from tests.code_objects import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000000   # 256-byte aligned, never dereferenced on these paths
STEP = 0x1000000
NAN, INF = float("nan"), float("inf")


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "cis_norm.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:size_t|int)\s+(cis_\w+)\s*\(", text, flags=re.M))
    assert names == {"cis_rms_norm_fwd", "cis_rms_norm_workspace_bytes", "cis_rms_norm_bwd"}
    lib = cis.load_library()
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    (tmp_path / "t.c").write_text('#include "cis_norm.h"\nint main(void) { return 0; }\n')
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-fsyntax-only",
                    "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(tmp_path / "t.c")], check=True)


def test_workspace_sizes():
    for T, N, H in ((0, 1, 1), (1, 1, 7), (4096, 1, 2048), (70000, 16, 128), (3, 1, 1 << 22)):
        assert cis.rms_norm_workspace_bytes(T, N, H) >= min(T * N, 1) * H * 4
    for bad in ((-1, 1, 8), (1, 0, 8), (1, 1, 0), (1, 1, (1 << 22) + 1), (1 << 30, 2, 8)):
        assert cis.rms_norm_workspace_bytes(*bad) == 0


def test_rows_stay_in_registers():
    """No kernel of the norm keeps a part of its rows in scratch memory."""
    norm = [k for k in kernels(cis.library_path()) if "cis_norm" in k[".name"]]
    assert len(norm) >= 50
    for k in norm:
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, k[".name"]


def _rows(at, dtype=0, st=64, sn=16):
    return None if at is None else _norm._Rows(at, dtype, st, sn)


def _fwd(**kw):
    a = dict(T=4, N=2, H=16, x=_rows(AT), r=_rows(AT + STEP), w=AT + 2 * STEP, wdt=0, eps=1e-6,
             s=_rows(AT + 3 * STEP), y=_rows(AT + 4 * STEP), scale=None, group=0)
    a.update(kw)
    ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
    return _norm._lib().cis_rms_norm_fwd(a["T"], a["N"], a["H"], ref(a["x"]), ref(a["r"]), a["w"],
                                         a["wdt"], a["eps"], ref(a["s"]), ref(a["y"]), a["scale"],
                                         a["group"], None)


Y8 = _rows(AT + 4 * STEP, 2)
SC = AT + 5 * STEP


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(y=None), -1),
    (dict(x=_rows(AT, 5)), -3), (dict(x=_rows(AT, 2)), -3), (dict(y=_rows(AT, 3)), -3),
    (dict(wdt=2), -3), (dict(x=_rows(AT, 1)), -3),                    # the residual is bf16
    (dict(s=_rows(AT + 3 * STEP, 1)), -3), (dict(r=None), -3),        # a sum without a residual
    (dict(T=-1), -2), (dict(N=0), -2), (dict(H=0), -2), (dict(H=(1 << 22) + 1), -2),
    (dict(T=1 << 30), -2), (dict(T=1 << 62), -2), (dict(N=1 << 40, T=1), -2),
    (dict(group=32), -2), (dict(y=Y8, scale=SC, group=16), -2), (dict(y=Y8, scale=SC, group=-1), -2),
    (dict(x=_rows(AT, 0, -64)), -2), (dict(x=_rows(AT, 0, 64, -16)), -2),
    (dict(x=_rows(AT, 0, 1 << 62)), -2),
    (dict(eps=-1e-6), -4), (dict(eps=NAN), -4), (dict(eps=INF), -4),
    (dict(x=_norm._Rows(None, 0, 64, 16)), -1), (dict(y=_norm._Rows(None, 0, 64, 16)), -1),
    (dict(r=_norm._Rows(None, 0, 64, 16)), -1), (dict(y=Y8), -1),
    (dict(x=_rows(AT + 8)), -5), (dict(x=_rows(AT, 0, 68)), -5), (dict(r=_rows(AT, 0, 64, 12)), -5),
    (dict(w=AT + 2), -5), (dict(y=_rows(AT + 4 * STEP + 4, 2), scale=SC), -5),
    (dict(y=Y8, scale=SC + 2), -5),
    (dict(y=_rows(AT + 4 * STEP, 0, 16, 16)), -8),                    # rows that share storage
    (dict(y=_rows(AT + 4 * STEP, 0, 0, 16)), -8), (dict(y=_rows(AT + 4 * STEP, 0, 64, 8)), -8),
    (dict(y=_rows(AT + 64)), -8), (dict(y=_rows(AT, 1)), -8), (dict(y=_rows(AT, 0, 128, 16)), -8),
    (dict(y=_rows(AT + 3 * STEP)), -8),                               # both outputs
    (dict(y=_rows(AT + 2 * STEP)), -8), (dict(y=Y8, scale=AT + 4 * STEP), -8),
    (dict(y=Y8, scale=AT), -8), (dict(y=Y8, scale=AT + 2 * STEP), -8),
    (dict(s=_rows(AT + STEP, 0, 64, 32)), -8),
])
def test_forward_argument_errors(kw, code):
    assert _fwd(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(), dict(y=_rows(AT)), dict(s=_rows(AT + STEP)), dict(y=_rows(AT), s=_rows(AT + STEP)),
    dict(y=_rows(AT + STEP), s=_rows(AT)), dict(w=None), dict(s=None), dict(r=None, s=None),
    dict(y=Y8, scale=SC, group=128), dict(y=_rows(AT + 4 * STEP, 0, 16, 64)),
    dict(x=_rows(AT, 0, 0, 0)), dict(T=0, x=_norm._Rows(None, 0, 0, 0)),
])
def test_good_arguments_reach_the_device(kw):
    """Without a GPU every one of these ends at the check of the device, which is the last."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the GPU's")
    assert _fwd(**kw) == -9


def _bwd(**kw):
    a = dict(T=4, N=2, H=16, dy=_rows(AT), x=_rows(AT + STEP), w=AT + 2 * STEP, wdt=0, eps=1e-6,
             dr=_rows(AT + 3 * STEP), dx=_rows(AT + 4 * STEP), dw=AT + 5 * STEP, ws=AT + 6 * STEP,
             wsb=1 << 20)
    a.update(kw)
    ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
    return _norm._lib().cis_rms_norm_bwd(a["T"], a["N"], a["H"], ref(a["dy"]), ref(a["x"]), a["w"],
                                         a["wdt"], a["eps"], ref(a["dr"]), ref(a["dx"]), a["dw"],
                                         a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), -1), (dict(x=None), -1), (dict(dx=None), -1), (dict(ws=None), -1),
    (dict(dy=_rows(AT, 2)), -3), (dict(x=_rows(AT, 2)), -3), (dict(dx=_rows(AT, 2)), -3),
    (dict(dr=_rows(AT + 3 * STEP, 1)), -3), (dict(wdt=-1), -3), (dict(H=0), -2), (dict(N=0), -2),
    (dict(dy=_rows(AT, 0, -8)), -2), (dict(eps=NAN), -4), (dict(ws=AT + 6 * STEP + 8), -5),
    (dict(wsb=8), -7), (dict(dw=AT + 5 * STEP + 4), -5), (dict(dx=_rows(AT + 4 * STEP + 2)), -5),
    (dict(dx=_rows(AT + 4 * STEP, 0, 0, 16)), -8), (dict(dx=_rows(AT + 16)), -8),
    (dict(dx=_rows(AT + 2 * STEP)), -8), (dict(dw=AT), -8), (dict(dw=AT + 4 * STEP), -8),
    (dict(dw=AT + 6 * STEP), -8), (dict(ws=AT), -8), (dict(ws=AT + 4 * STEP), -8),
    (dict(ws=AT + 2 * STEP), -8), (dict(dw=AT + 2 * STEP), -8),
])
def test_backward_argument_errors(kw, code):
    assert _bwd(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(), dict(dx=_rows(AT)), dict(dx=_rows(AT + STEP)), dict(dx=_rows(AT + 3 * STEP)),
    dict(dw=None, ws=None, wsb=0), dict(dr=None), dict(w=None), dict(dy=_rows(AT, 0, 0, 0)),
    dict(T=0, dy=_norm._Rows(None, 0, 0, 0)),
])
def test_good_backward_arguments_reach_the_device(kw):
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the GPU's")
    assert _bwd(**kw) == -9


def test_binding_refuses():
    x = torch.zeros(4, 16)
    with pytest.raises(ValueError, match="device tensor"):
        cis.rms_norm(x)
    for bad in (torch.zeros(16), torch.zeros(2, 2, 2, 2), [1.0]):
        with pytest.raises(ValueError, match="must be a"):
            cis.rms_norm(bad)
