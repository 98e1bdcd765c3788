"""The C ABI of the verification of drafted tokens on the host: every declared entry point is there, and
bad arguments are rejected before a device is touched. No kernel is launched here."""

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2609_32444_amd as cis
from paper_2609_32444_amd import _tokens, _verify

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # a 256-byte aligned non-null address; never dereferenced on these paths
BIG = 1 << 34
NAN, INF = float("nan"), float("inf")


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "cis_verify.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:size_t|int)\s+(cis_\w+)\s*\(", text, flags=re.M))
    assert names == {"cis_verify_workspace_bytes", "cis_verify"}
    lib = cis.load_library()
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    (tmp_path / "t.c").write_text('#include "cis_verify.h"\nint main(void) { return 0; }\n')
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-fsyntax-only",
                    "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(tmp_path / "t.c")], check=True)


def test_workspace_sizes():
    for dt in (torch.bfloat16, torch.float32):
        for T, D, n in ((0, 0, 0), (0, 0, 3), (1, 0, 1), (320, 256, 64), (5, 4, 1)):
            # a scan and a draw of every row are a part of it
            assert cis.verify_workspace_bytes(T, D, n, 50257, dt) >= cis.sample_workspace_bytes(
                T + D, 50257, dt)
    for bad in ((-1, 0, 1, 8), (1, -1, 1, 8), (1, 0, -1, 8), (1, 0, 1, 0), (1, 0, 1, (1 << 28) + 1),
                (1 << 31, 1, 1, 8), (1, 0, 1 << 32, 8), (1 << 62, 1 << 62, 1, 8)):
        assert cis.verify_workspace_bytes(*bad) == 0
    assert _verify._lib().cis_verify_workspace_bytes(1, 0, 1, 8, 2) == 0


def _verify_call(**kw):
    a = dict(logits=FAKE, dtype=0, T=6, V=8, ld=8, q=FAKE, D=4, ld_d=8, ids=FAKE, u=FAKE, offs=FAKE, n=2,
             temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, temps=None, ks=None, ps=None, ms=None,
             out=FAKE, acc=FAKE, lp=None, lk=None, ws=FAKE, wsb=BIG, prm=True)
    a.update(kw)
    prm = _tokens._SampleParams(a["temperature"], a["top_k"], a["top_p"], a["min_p"])
    return _verify._lib().cis_verify(
        a["logits"], a["dtype"], a["T"], a["V"], a["ld"], a["q"], a["D"], a["ld_d"], a["ids"], a["u"],
        a["offs"], a["n"], ctypes.byref(prm) if a["prm"] else None, a["temps"], a["ks"], a["ps"],
        a["ms"], a["out"], a["acc"], a["lp"], a["lk"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(prm=False), -1), (dict(dtype=5), -3), (dict(T=-1), -2), (dict(V=0), -2), (dict(ld=7), -2),
    (dict(V=(1 << 28) + 1, ld=1 << 29, ld_d=1 << 29), -2), (dict(D=-1), -2), (dict(n=-1), -2),
    (dict(n=0), -2), (dict(T=(1 << 31) + 1), -2), (dict(T=1 << 31, D=1), -2), (dict(n=1 << 40), -2),
    (dict(ld_d=7), -2), (dict(temperature=-1.0), -4), (dict(temperature=NAN), -4),
    (dict(temperature=INF), -4), (dict(top_k=-1), -4), (dict(top_p=0.0), -4), (dict(top_p=NAN), -4),
    (dict(min_p=-0.1), -4), (dict(min_p=1.1), -4), (dict(ws=None), -1), (dict(logits=None), -1),
    (dict(u=None), -1), (dict(out=None), -1), (dict(acc=None), -1), (dict(offs=None), -1),
    (dict(ids=None), -1), (dict(ws=FAKE + 64), -5), (dict(logits=FAKE + 8), -5), (dict(ld=12), -5),
    (dict(q=FAKE + 4), -5), (dict(ld_d=12), -5), (dict(wsb=0), -7),
])
def test_argument_errors(kw, code):
    assert _verify_call(**kw) == code


def test_arrays_replace_their_parameter():
    for kw in (dict(temperature=NAN, temps=FAKE), dict(top_k=-1, ks=FAKE), dict(top_p=NAN, ps=FAKE),
               dict(min_p=NAN, ms=FAKE)):
        assert _verify_call(ws=None, **kw) == -1


@pytest.mark.parametrize("kw", [
    dict(), dict(q=None, ld_d=0), dict(D=0, ids=None, q=None),
    dict(T=0, D=0, n=0, logits=None, u=None, out=None, acc=None, offs=None, ids=None, q=None),
    dict(T=0, D=0, logits=None, u=None, out=None, ids=None, q=None)])
def test_good_arguments_reach_the_device(kw):
    """Without a GPU every one of these ends at the check of the device, which is the last."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the GPU's")
    assert _verify_call(**kw) == -9
