"""The token operators' C ABI on the host: every declared entry point is there, and bad arguments are
rejected before a device is touched. No kernel is launched here."""

import ctypes
import os
import re

import pytest
import torch

import paper_2609_32444_amd as cis
from paper_2609_32444_amd import _tokens
from tests.code_objects import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # a 256-byte aligned non-null address; never dereferenced on these paths
BIG = 1 << 34


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "cis_tokens.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"^\s*(?:size_t|int)\s+(cis_\w+)\s*\(", text, flags=re.M))
    assert names == {"cis_sample_workspace_bytes", "cis_sample", "cis_top_logits_workspace_bytes",
                     "cis_top_logits", "cis_distill_workspace_bytes", "cis_distill_fwd",
                     "cis_distill_bwd"}
    lib = cis.load_library()
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    (tmp_path / "t.c").write_text('#include "cis_tokens.h"\nint main(void) { return 0; }\n')
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-fsyntax-only",
                    "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(tmp_path / "t.c")], check=True)


def test_workspace_sizes():
    bf, f32 = torch.bfloat16, torch.float32
    for T in (0, 1, 7, 4096):
        for dt in (bf, f32):
            assert cis.sample_workspace_bytes(T, 50257, dt) > 0
            assert cis.top_logits_workspace_bytes(T, 50257, 64, dt) > 0
            # the loss workspace's statistics and per-row arrays are a part of it
            assert cis.distill_workspace_bytes(T, 50257, 64, dt) >= 1280 + 18 * T
    for bad in ((-1, 10), (1, 0), (1, (1 << 28) + 1)):
        assert cis.sample_workspace_bytes(*bad) == 0
        assert cis.top_logits_workspace_bytes(*bad, 4) == 0
        assert cis.distill_workspace_bytes(*bad, 4) == 0
    for K in (0, 1025):
        assert cis.top_logits_workspace_bytes(1, 10, K) == 0
        assert cis.distill_workspace_bytes(1, 10, K) == 0
    assert _tokens._lib().cis_sample_workspace_bytes(1, 10, 2) == 0
    with pytest.raises(ValueError):
        cis.sample_workspace_bytes(1, 10, torch.float16)


def _sample(**kw):
    a = dict(logits=FAKE, dtype=0, T=4, V=8, ld=8, u=FAKE, mask=None, temperature=1.0, top_k=0,
             top_p=1.0, min_p=0.0, temps=None, ks=None, ps=None, ms=None, ids=FAKE, lp=None,
             lk=None, ws=FAKE, wsb=BIG, prm=True)
    a.update(kw)
    prm = _tokens._SampleParams(a["temperature"], a["top_k"], a["top_p"], a["min_p"])
    return _tokens._lib().cis_sample(
        a["logits"], a["dtype"], a["T"], a["V"], a["ld"], a["u"], a["mask"],
        ctypes.byref(prm) if a["prm"] else None, a["temps"], a["ks"], a["ps"], a["ms"], a["ids"],
        a["lp"], a["lk"], a["ws"], a["wsb"], None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,code", [
    (dict(prm=False), -1), (dict(dtype=5), -3), (dict(T=-1), -2), (dict(V=0), -2),
    (dict(ld=7), -2), (dict(V=(1 << 28) + 1, ld=1 << 29), -2), (dict(ld=1 << 62), -2),
    (dict(temperature=-1.0), -4), (dict(temperature=NAN), -4), (dict(temperature=INF), -4),
    (dict(top_k=-1), -4), (dict(top_p=0.0), -4), (dict(top_p=1.5), -4), (dict(top_p=NAN), -4),
    (dict(min_p=-0.1), -4), (dict(min_p=1.1), -4), (dict(min_p=NAN), -4),
    (dict(ws=None), -1), (dict(logits=None), -1), (dict(u=None), -1), (dict(ids=None), -1),
    (dict(ws=FAKE + 64), -5), (dict(logits=FAKE + 8), -5), (dict(ld=12), -5), (dict(wsb=0), -7),
])
def test_sample_argument_errors(kw, code):
    assert _sample(**kw) == code


def test_sample_arrays_replace_their_parameter():
    """A parameter that an array replaces is not looked at: the next check is reached."""
    for kw in (dict(temperature=NAN, temps=FAKE), dict(top_k=-1, ks=FAKE),
               dict(top_p=NAN, ps=FAKE), dict(min_p=NAN, ms=FAKE)):
        assert _sample(ws=None, **kw) == -1


def _top(**kw):
    a = dict(logits=FAKE, dtype=0, T=4, V=8, ld=8, mask=None, K=3, temperature=1.0, ids=FAKE,
             values=FAKE, tail=None, ws=FAKE, wsb=BIG)
    a.update(kw)
    return _tokens._lib().cis_top_logits(
        a["logits"], a["dtype"], a["T"], a["V"], a["ld"], a["mask"], a["K"], a["temperature"],
        a["ids"], a["values"], a["tail"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), -3), (dict(T=-1), -2), (dict(V=0), -2), (dict(ld=7), -2), (dict(K=0), -2),
    (dict(K=1025), -2), (dict(temperature=0.0), -4), (dict(temperature=NAN), -4),
    (dict(temperature=INF), -4), (dict(temperature=1e-30), -4), (dict(ws=None), -1),
    (dict(logits=None), -1), (dict(ids=None), -1), (dict(values=None), -1),
    (dict(ws=FAKE + 64), -5), (dict(logits=FAKE + 8), -5), (dict(dtype=1, ld=9), -5),
    (dict(wsb=1), -7),
])
def test_top_argument_errors(kw, code):
    assert _top(**kw) == code


def _distill(bwd=True, **kw):
    a = dict(logits=FAKE, dtype=0, T=4, V=8, ld=8, ids=FAKE, values=FAKE, K=3, ldt=3, tail=FAKE,
             weight=None, mask=None, kind=0, temperature=1.0, scale=1.0, dl=FAKE * 16, ldg=8,
             ws=FAKE, wsb=BIG, prm=True)
    a.update(kw)
    prm = _tokens._DistillParams(a["kind"], a["temperature"], a["scale"])
    head = (a["logits"], a["dtype"], a["T"], a["V"], a["ld"], a["ids"], a["values"], a["K"],
            a["ldt"], a["tail"], a["weight"], a["mask"], ctypes.byref(prm) if a["prm"] else None)
    if bwd:
        return _tokens._lib().cis_distill_bwd(*head, a["dl"], a["ldg"], None, None, a["ws"],
                                              a["wsb"], None)
    return _tokens._lib().cis_distill_fwd(*head, None, None, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(prm=False), -1), (dict(dtype=2), -3), (dict(T=-1), -2), (dict(V=0), -2),
    (dict(ld=7), -2), (dict(K=0), -2), (dict(K=1025, ldt=1025), -2), (dict(ldt=2), -2),
    (dict(kind=2), -4), (dict(temperature=0.0), -4), (dict(temperature=NAN), -4),
    (dict(temperature=1e30), -4), (dict(scale=NAN), -4), (dict(scale=INF), -4),
    (dict(kind=1, tail=None), -4), (dict(ws=None), -1), (dict(logits=None), -1),
    (dict(ids=None), -1), (dict(values=None), -1), (dict(ws=FAKE + 64), -5),
    (dict(logits=FAKE + 8), -5), (dict(V=7, ld=7), -5), (dict(wsb=100), -7),
])
def test_distill_argument_errors(bwd, kw, code):
    assert _distill(bwd, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dl=None), -1), (dict(ldg=7), -2), (dict(dl=FAKE * 16 + 8), -5), (dict(ldg=12), -5),
    (dict(dl=FAKE, ldg=16), -8), (dict(dl=FAKE + 32), -8),
])
def test_distill_gradient_argument_errors(kw, code):
    assert _distill(True, **kw) == code


def test_binding_rejects_wrong_tensors():
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):   # not on a device
        cis.sample(z, torch.zeros(2))
    with pytest.raises(ValueError):
        cis.top_logits(z, 4)
    with pytest.raises(ValueError):
        cis.distill_fwd(z, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3))


def test_lists_whose_rows_share_storage_are_refused():
    """The kernels read entry t * ld_top + k: no list passes whose storage ends before that."""
    T, K = 5, 4
    base = torch.zeros(T * 8, dtype=torch.int32)

    def lists(step, rows=T):
        return (base.as_strided((rows, K), (step, 1)),
                base.float().as_strided((rows, K), (step, 1)))

    for step in (K, K + 1, 8):
        ld = _tokens._list_stride(*lists(step), T, K)
        assert ld == step and (T - 1) * ld + K <= base.numel()
    for step in (0, 1, K - 1):
        with pytest.raises(ValueError, match="share storage"):
            _tokens._list_stride(*lists(step), T, K)
    with pytest.raises(ValueError, match="same row stride"):
        _tokens._list_stride(lists(8)[0], lists(K)[1], T, K)
    # one row, or none: its stride never moves an address
    for rows in (0, 1):
        for step in (0, 1, 8):
            assert _tokens._list_stride(*lists(step, rows), rows, K) == K


def test_top_k_beyond_int32_stays_beyond_every_row():
    """The library's field holds 32 bits: 2^32 + 5 would be 5 there, 2^31 negative."""
    def field(k):
        return _tokens._SampleParams(1.0, _tokens._top_k(k), 1.0, 0.0).top_k

    for k in (0, 5, 2 ** 31 - 1):
        assert field(k) == k
    for k in (2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 80):
        assert field(k) == 2 ** 31 - 1   # V is 2^28 at most
    for k in (-1, -3, -2 ** 31 - 1, -2 ** 32):
        assert field(k) < 0


def test_weights_of_uncut_rows_leave_eight_waves():
    """The sampler's sum of uncut rows unpacks a vector at a time: at most 64 registers, 8 waves to a SIMD."""
    weigh = [k for k in kernels(cis.library_path()) if "cis_weigh_kernel" in k[".name"] and "ELb0ELb0E" in k[".name"]]
    assert len(weigh) == 2    # bf16 and float32
    for k in weigh:
        assert k[".vgpr_count"] <= 64, k[".name"]
