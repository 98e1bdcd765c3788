"""The RMS norm on the GPU against the float64 oracle (oracle/norm.py).

Tolerances. u = 2^-24 is half a step of float32. The sum is x + residual rounded to float32 (exact
there: one rounding, the same as torch's) and to the residual's type, and compared bit for bit.
  * rstd is formed in double and rounded once (u); y = (s rstd) w adds u twice, and the sums in double
    less than u in all: 4u, relative, and half a step of the output's type.
  * e4m3: scale is the largest |y| (4u) over 448 (u): 6u. The values stand for y: y / scale is off by
    4u for y, 6u for the scale, u for the quotient (12u in all are allowed); then half a step of e4m3,
    2^-4 of the value or 2^-10 where it is below the least normal 2^-6.
  * dx = rstd (g - xh m) + dr, m = mean(g xh). g rounds once (u |g|). m = (sum of s g in double)
    rstd / H: u |m| for rstd and u |m| for its own rounding, and u mean(|g xh|) for the g that are
    summed, which may be far more than |m| where they cancel. xh rounds twice, its product with m and
    the difference once each, the factor rstd twice. In all 4u of rstd |g|, and of rstd |xh| 8u |m| +
    u mean(|g xh|): under 9u of rstd (|g| + |xh| mean(|g xh|)), u of the result for the last sum, and half
    a step of its type.
  * dweight sums n products of 3 roundings in float32 (n u of the sum of their sizes at most, and 4u)
    and rounds once more.
Subnormal float32 results add 2^-149 to each.
"""

import math

import numpy as np
import pytest
import torch

import paper_2609_32444_amd as cis
from oracle import norm as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF = {BF: 2.0 ** -8, F32: U}
TINY = 2.0 ** -149


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _store(a, dtype, pad=0, fill=math.nan):
    """A tensor in rows of whole 16-byte vectors and `pad` more, the padding filled with NaNs."""
    per = 16 // dtype.itemsize
    ld = (a.shape[-1] + per - 1) // per * per + pad * per
    s = torch.full((*a.shape[:-1], ld), fill, device=DEV).to(dtype)
    s[..., :a.shape[-1]] = a.to(dtype)
    return s[..., :a.shape[-1]]


def _rand(shape, dtype, seed, size=1.0, pad=0):
    g = _gen(seed)
    a = torch.randn(*shape, generator=g, device=DEV) * size
    a *= torch.exp(torch.randn(*shape[:-1], 1, generator=g, device=DEV))
    return _store(a, dtype, pad)


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, tol):
    got = _np(got)
    bad = ~(np.abs(got - want) <= tol + TINY)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} off, worst "
                           f"{np.max(np.abs(got - want)[bad] / (tol + TINY)[bad])} of the tolerance")


def _check_y(out, y, group=0, dtype=None):
    got = out["y"]
    dtype = dtype or got.dtype
    if dtype != F8:
        _near(got, y, (4 * U + HALF[dtype]) * np.abs(y))
        return
    scale = orc.scales(y, group)
    have = _np(out["scale"]).reshape(scale.shape)
    assert np.all(np.abs(have - scale) <= 6 * U * scale)
    n = group or y.shape[-1]
    s = np.repeat(have, n, axis=-1)[..., :y.shape[-1]]
    q = np.abs(y / s)
    # (a quotient may lie 12u beyond a step's end)
    step = np.maximum(2.0 ** -4 * q, 2.0 ** -10) * (1 + 16 * U) + 12 * U * q
    assert np.all(np.abs(_np(got) - y / s) <= step)
    assert np.all(np.abs(_np(got)) <= 448)


def _check_fwd(x, w, r, out, eps, group=0):
    s = x
    if r is not None:
        s = (x.float() + r.float()).to(r.dtype)
        if "residual" in out:
            assert torch.equal(out["residual"], s)
    y = orc.forward(_np(s), 1.0 if w is None else _np(w), float(np.float32(eps)))
    _check_y(out, y, group)


# lengths at and beside those where a kernel's shape changes, odd ones and the smallest
SIZES = [1, 2, 7, 8, 9, 15, 31, 32, 33, 40, 63, 64, 65, 79, 127, 128, 129, 250, 256, 257, 391, 511, 512, 513, 1000, 1023,
         1024, 1025, 2040, 2048, 2049, 4095, 4096, 4097, 5120, 8191, 8192, 8193, 16383, 16384, 16385,
         32768, 32769, 50001]
TYPES = [(BF, None), (F32, None), (BF, BF), (BF, F32), (F32, F32)]


@pytest.mark.parametrize("H", SIZES)
def test_forward_sizes(H):
    """Every width, over all types in turn, with rows that fill a workgroup and some more."""
    for i, (xt, rt) in enumerate(TYPES):
        T = 37 if H <= 4096 else 5
        x = _rand((T, H), xt, H + i, pad=i % 2)
        r = None if rt is None else _rand((T, H), rt, H + 50 + i, 3.0, pad=i % 3)
        w = [None, _rand((H,), BF, 1), _rand((H,), F32, 2)][(i + H) % 3]
        w = w if w is None else w.contiguous()
        for out_dtype in (BF, F32):
            out = cis.rms_norm(x, w, r, eps=1e-6, out_dtype=out_dtype)
            _check_fwd(x, w, r, out, 1e-6)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("H", SIZES)
def test_e4m3_sizes(H, group):
    T = 21 if H <= 4096 else 3
    xt, rt = TYPES[(H + group // 32) % 5]
    x = _rand((T, H), xt, H, pad=1)
    r = None if rt is None else _rand((T, H), rt, H + 9)
    w = _rand((H,), F32, 3)
    out = cis.rms_norm(x, w.contiguous(), r, eps=1e-5, out_dtype=F8, group=group)
    assert out["scale"].shape == ((T, (H + group - 1) // group) if group else (T,))
    _check_fwd(x, w, r, out, 1e-5, group)


def _check_quotients(x, w, r, group, eps=1e-6):
    """Scales and values from the same call's float32 y by the definition, bit for bit: y, the scale and the
    quotient are one float32 rounding each, and that is rounded to e4m3."""
    y = cis.rms_norm(x, w, r, eps=eps, out_dtype=F32)["y"]
    out = cis.rms_norm(x, w, r, eps=eps, out_dtype=F8, group=group)
    H = y.shape[-1]
    n = group or H
    blocks = torch.nn.functional.pad(y, (0, -H % n)).view(y.shape[0], -1, n)
    top = blocks.abs().amax(2)
    # (a quotient by a tensor: one by a number is a product with its reciprocal on the device)
    scale = (top / torch.full_like(top, 448.0)).clamp(min=2.0 ** -126)
    assert torch.equal(out["scale"].view(scale.shape), scale)
    want = (blocks / scale[:, :, None]).view(y.shape[0], -1)[:, :H].to(F8)
    off = out["y"].view(torch.uint8) != want.view(torch.uint8)
    assert not off.any(), f"{int(off.sum())} of {off.numel()} values"


@pytest.mark.parametrize("T,H", [(300, 5120), (600, 5120), (700, 2048), (20000, 72), (9000, 200), (3000, 516),
                                 (200, 16384), (70, 32768), (60, 40001), (1, 2048)])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_e4m3_values_are_the_quotients_rounded(T, H, group):
    """bf16 rows and weights have products of 16 bits, whose quotients often are halfway between two values."""
    w = _rand((H,), BF, 3).contiguous()
    _check_quotients(_rand((T, H), BF, 1), w, _rand((T, H), BF, 2, 3.0), group)
    _check_quotients(_rand((T, H), F32, 4), None, None, group)


@pytest.mark.parametrize("H", [64, 3000, 40000])
def test_e4m3_quotients_of_extreme_scales(H):
    """Scales at the least one and just above it (the values subnormal numbers of float32), and near the end of float32."""
    x = torch.randn(9, H, generator=_gen(H), device=DEV)
    for size in (2.0 ** -149, 2.0 ** -140, 2.0 ** -126, 2.0 ** -120, 2.0 ** -117, 2.0 ** -60, 2.0 ** 60, 2.0 ** 124):
        w = torch.full((H,), size, device=DEV)
        for group in (0, 32):
            _check_quotients(_store(x, F32), w, None, group, eps=0.0)


@pytest.mark.parametrize("T", [512, 513, 1100])
@pytest.mark.parametrize("H", [513, 1000, 1024, 1025, 2040, 2048, 2049, 4095, 4096, 4097, 5120, 8191,
                               8192, 8193])
def test_sizes_of_many_rows(H, T):
    """Either side of the count of rows from which a lane takes several groups, every type."""
    w = _rand((H,), F32, 3).contiguous()
    for i, (xt, rt) in enumerate(TYPES):
        x = _rand((T, H), xt, H + i)
        r = None if rt is None else _rand((T, H), rt, H + 50 + i, 3.0)
        out_dtype, group = [(BF, 0), (F8, 0), (F32, 0), (F8, 128), (F8, 32)][i]
        out = cis.rms_norm(x, w, r, eps=1e-6, out_dtype=out_dtype, group=group)
        rows = torch.cat([torch.arange(8), torch.arange(T - 8, T), torch.randint(0, T, (40,))])
        some = {k: v[rows] for k, v in out.items()}
        _check_fwd(x[rows], w, None if r is None else r[rows], some, 1e-6, group)
        if r is not None:
            assert torch.equal(out["residual"], (x.float() + r.float()).to(rt))


@pytest.mark.parametrize("T", [1, 2, 3, 63, 64, 65, 1000, 5000, 20011])
@pytest.mark.parametrize("H", [64, 640, 2048])
def test_row_counts(T, H):
    x, r = _rand((T, H), BF, T), _rand((T, H), BF, T + 1)
    w = _rand((H,), BF, 5).contiguous()
    out = cis.rms_norm(x, w, r)
    _check_fwd(x, w, r, out, 1e-6)
    dy = _rand((T, H), F32, 7)
    _check_bwd(dy, out["residual"], w, None, cis.rms_norm_bwd(dy, out["residual"], w), 1e-6)


def _check_bwd(dy, s, w, dr, out, eps, dy_np=None, s_np=None, dr_np=None):
    dy_np, s_np = _np(dy) if dy_np is None else dy_np, _np(s) if s_np is None else s_np
    dr_np = dr_np if dr_np is not None or dr is None else _np(dr)
    dx, dw, size_w, size = orc.backward(dy_np, s_np, 1.0 if w is None else _np(w),
                                        float(np.float32(eps)), dr_np)
    _near(out["dx"], dx, 9 * U * size + (U + HALF[out["dx"].dtype]) * np.abs(dx))
    if "dweight" in out:
        n = s_np.size // s_np.shape[-1]
        _near(out["dweight"], dw, (n + 4) * U * size_w + U * np.abs(dw))


@pytest.mark.parametrize("H", SIZES)
def test_backward_sizes(H):
    for i, (dt, xt, gt) in enumerate([(BF, BF, BF), (F32, BF, BF), (F32, BF, F32), (BF, F32, F32),
                                      (F32, F32, F32), (F32, F32, BF), (BF, BF, F32), (BF, F32, BF)]):
        T = 37 if H <= 4096 else 5
        dy, s = _rand((T, H), dt, H + i, 1e-3, pad=i % 2), _rand((T, H), xt, H + 30 + i, 3.0)
        w = [None, _rand((H,), BF, 1), _rand((H,), F32, 2)][(i + H) % 3]
        w = w if w is None else w.contiguous()
        dr = None if i % 2 else _rand((T, H), gt, H + 60, 1e-3, pad=1)
        out = cis.rms_norm_bwd(dy, s, w, dr, eps=1e-5, dx_dtype=gt)
        _check_bwd(dy, s, w, dr, out, 1e-5)
        alone = cis.rms_norm_bwd(dy, s, w, dr, eps=1e-5, dx_dtype=gt, dweight=False)
        assert torch.equal(alone["dx"], out["dx"]) and "dweight" not in alone


def _share(H):
    """(parts of dweight's sums, rows that a part takes side by side) where there are rows enough for all parts."""
    rows = 1 << 20
    nbytes = cis.rms_norm_workspace_bytes(rows, 1, H) - (rows * 4 if H > 8192 else 0)
    groups = (H + 7) // 8
    side = 1 if groups > 64 else 256 // max(4, 1 << (groups - 1).bit_length())
    return nbytes // (4 * H), side


def _whole(T, H):
    g = _gen(T + H)
    return (torch.randint(-8, 9, (T, H), generator=g, device=DEV),
            torch.randint(0, 2, (T, H), generator=g, device=DEV) * 2 - 1)


def _check_turns(T, H, dt, xt, place=None, dr=True):
    """Rows that a part's lanes take one after the other. A lane adds as many products as it takes turns, then those of
    the rows beside it: dweight's tolerance is that count (turns + side, and 3 roundings a product), not the rows'. And with
    rows of +-1, eps = 0 and whole numbers for dy every product and sum is exact, so that a row left out or
    taken twice shows whatever its size."""
    parts, side = _share(H)
    turns = -(-T // (parts * side))
    w = _rand((H,), F32, 2).contiguous()
    d = _rand((T, H), xt, 60, 1e-3) if dr else None
    buffers = lambda dy, s: (dy, s, {"dx": dy} if place == 0 else {"dx": s} if place == 1 else {})  # noqa: E731
    dy, s = _rand((T, H), dt, T, 1e-3), _rand((T, H), xt, T + 1, 3.0)
    dy_np, s_np = _np(dy), _np(s)
    gy, gs, kw = buffers(dy, s)
    out = cis.rms_norm_bwd(gy, gs, w, d, eps=1e-5, **kw)
    dx, dw, size_w, size = orc.backward(dy_np, s_np, _np(w), float(np.float32(1e-5)), None if d is None else _np(d))
    _near(out["dx"], dx, 9 * U * size + (U + HALF[out["dx"].dtype]) * np.abs(dx))
    _near(out["dweight"], dw, (turns + side + 4) * U * size_w + U * np.abs(dw))
    whole, sign = _whole(T, H)
    gy, gs, kw = buffers(_store(whole, dt), _store(sign, xt))
    out = cis.rms_norm_bwd(gy, gs, w, d, eps=0.0, **kw)
    assert torch.equal(out["dweight"].long(), (whole * sign).sum(0))


@pytest.mark.parametrize("H", [20, 64, 100, 128, 256, 391, 512, 1000, 2048, 3000, 4100, 5632, 8192])
def test_backward_takes_rows_in_turn(H):
    """One row more than all parts take at once, and several turns of which the last is of some parts."""
    parts, side = _share(H)
    all_at_once = parts * side
    _check_turns(all_at_once + 1, H, BF, BF)
    _check_turns(2 * all_at_once + side + 3, H, F32, BF, dr=False)
    if H <= 512:
        _check_turns(all_at_once + side // 2 + 1, H, F32, F32, place=1)
        _check_turns(3 * all_at_once - 1, H, BF, F32, dr=False)
    else:
        _check_turns(4 * parts + 77, H, F32, F32, place=0)


def test_backward_of_many_rows_to_the_last_one():
    T = (1 << 21) + 77
    for H, dt, xt in ((9, BF, BF), (40, F32, F32)):
        whole, sign = _whole(T, H)
        out = cis.rms_norm_bwd(_store(whole, dt), _store(sign, xt), eps=0.0)
        assert torch.equal(out["dweight"].long(), (whole * sign).sum(0))


@pytest.mark.parametrize("place", [None, 0, 1])
@pytest.mark.parametrize("T,H", [(257, 8200), (700, 8200), (1300, 8200), (143, 16400), (76, 33001), (400, 33001)])
def test_backward_of_long_rows_takes_them_in_turn(T, H, place):
    """More rows than parts, a part's turns not a multiple of the loop's unrolling; in place, where the sums go first."""
    parts, side = _share(H)
    assert T > parts and side == 1
    _check_turns(T, H, BF, BF, place)
    _check_turns(T, H, F32, F32, place, dr=place is None)


@pytest.mark.parametrize("D", [64, 128, 80, 200])
def test_heads_of_a_packed_projection(D):
    """Queries and keys between others' columns, tokens or heads outermost, in place."""
    T, nq, nk = 50, 6, 2
    ld = (nq + 2 * nk) * D
    for dtype in (BF, F32):
        qkv = _rand((T, ld), dtype, D)
        keep = qkv.clone()
        w = _rand((D,), F32, 3).contiguous()
        q, k = (qkv[:, :nq * D].view(T, nq, D),
                qkv[:, nq * D:(nq + nk) * D].view(T, nk, D))
        out_q = cis.rms_norm(q, w, y=q)
        out_k = cis.rms_norm(k, w, y=k)
        v0 = (nq + nk) * D
        assert torch.equal(qkv[:, v0:], keep[:, v0:])
        kq, kk = keep[:, :nq * D].reshape(T, nq, D), keep[:, nq * D:v0].reshape(T, nk, D)
        _check_fwd(kq, w, None, {"y": out_q["y"]}, 1e-6)
        _check_fwd(kk, w, None, {"y": out_k["y"]}, 1e-6)
        # heads outermost in memory, and the gradients of the same rows
        by_head = _rand((nq, T, D), dtype, 9).transpose(0, 1)
        out = cis.rms_norm(by_head, w)
        _check_fwd(by_head, w, None, out, 1e-6)
        out8 = cis.rms_norm(by_head, w, out_dtype=F8)
        assert out8["scale"].shape == (T, nq)
        _check_fwd(by_head, w, None, out8, 1e-6)
        g = cis.rms_norm_bwd(by_head, kq, w, dx=torch.empty_like(kq))
        _check_bwd(by_head, kq, w, None, g, 1e-6)


def test_broadcast_rows():
    """A gradient or residual that is one row for all."""
    T, H = 33, 520
    x, w = _rand((T, H), BF, 1), _rand((H,), BF, 2).contiguous()
    one = _rand((1, H), BF, 3).expand(T, H)
    out = cis.rms_norm(x, w, one)
    _check_fwd(x, w, one, out, 1e-6)
    _check_bwd(one, x, w, None, cis.rms_norm_bwd(one, x, w), 1e-6)
    with pytest.raises(cis.CisError):
        cis.rms_norm(x, w, one, residual_out=one)


@pytest.mark.parametrize("H", [72, 640, 2056, 6000, 40000])
def test_outputs_in_place_of_inputs(H):
    T = 9
    for dtype in (BF, F32):
        w = _rand((H,), BF, 2).contiguous()
        x0, r0 = _rand((T, H), dtype, 3), _rand((T, H), dtype, 4)
        want = cis.rms_norm(x0, w, r0)
        for yi, si in ((0, 1), (1, 0), (0, None), (1, None), (None, 0), (None, 1)):
            bufs = [_store(x0, dtype), _store(r0, dtype)]
            out = cis.rms_norm(bufs[0], w, bufs[1], y=None if yi is None else bufs[yi],
                               residual_out=None if si is None else bufs[si])
            assert torch.equal(out["y"], want["y"])
            assert torch.equal(out["residual"], want["residual"])
            out = cis.rms_norm(_store(x0, dtype), w, bufs[1].copy_(r0), residual_out=False)
            assert torch.equal(out["y"], want["y"]) and "residual" not in out
        out8 = cis.rms_norm(x0, w, r0, out_dtype=F8)
        buf = _store(r0, dtype)
        out = cis.rms_norm(x0, w, buf, out_dtype=F8, residual_out=buf)
        assert torch.equal(out["y"].view(torch.uint8), out8["y"].view(torch.uint8))
        assert torch.equal(out["scale"], out8["scale"]) and torch.equal(buf, want["residual"])
        out = cis.rms_norm(x0, w, r0, out_dtype=F8, residual_out=False)
        assert torch.equal(out["y"].view(torch.uint8), out8["y"].view(torch.uint8))
        # the gradient in place of each of its inputs
        dr0 = _rand((T, H), dtype, 6)
        want = cis.rms_norm_bwd(r0, x0, w, dr0)
        for i in range(3):
            bufs = [_store(r0, dtype), _store(x0, dtype), _store(dr0, dtype)]
            out = cis.rms_norm_bwd(bufs[0], bufs[1], w, bufs[2], dx=bufs[i])
            assert torch.equal(out["dx"], want["dx"])
            assert torch.equal(out["dweight"], want["dweight"])


@pytest.mark.parametrize("H", [5, 130, 2050, 9001, 33001])
def test_padding_is_neither_used_nor_written(H):
    T = 6
    w = _rand((H,), F32, 1).contiguous()
    x, r = _rand((T, H), BF, 2, pad=2), _rand((T, H), F32, 3, pad=1)
    for dtype in (BF, F32, F8):
        per = 16 // dtype.itemsize
        ld = (H + per - 1) // per * per + per
        base = torch.full((T, ld), 7.0, device=DEV).to(dtype)
        sums = torch.full((T, (H + 7) // 4 * 4), 7.0, device=DEV)
        out = cis.rms_norm(x, w, r, y=base[:, :H], residual_out=sums[:, :H])
        assert torch.all(base[:, H:].float() == 7) and torch.all(sums[:, H:] == 7)
        _check_fwd(x, w, r, out, 1e-6)
    dx = torch.full((T, (H + 15) // 8 * 8), 7.0, device=DEV).to(BF)
    out = cis.rms_norm_bwd(x, r, w, dx=dx[:, :H])
    assert torch.all(dx[:, H:] == 7)
    _check_bwd(x, r, w, None, out, 1e-6)


@pytest.mark.parametrize("H", [100, 1500, 9000, 40000])
def test_nan_and_infinity_stay_in_their_rows(H):
    T = 6
    x = _rand((T, H), F32, H)
    x[1, H // 2], x[3, H - 1], x[4, 0] = math.nan, math.inf, -math.inf
    good = [0, 2, 5]
    w = torch.ones(H, device=DEV)
    y = orc.forward(_np(x[good]), 1.0, float(np.float32(1e-6)))
    for dtype in (BF, F32):
        out = cis.rms_norm(x, w, out_dtype=dtype)["y"]
        _check_y({"y": out[good]}, y, dtype=dtype)
        assert torch.isnan(out[1]).all() and torch.isnan(out[3, H - 1]) and torch.isnan(out[4, 0])
        assert torch.all(out[3, :H - 1] == 0) and torch.all(out[4, 1:] == 0)
    for group in (0, 32):
        out = cis.rms_norm(x, w, out_dtype=F8, group=group)
        assert torch.isnan(out["scale"][1]).all() and torch.isnan(out["y"][1].float()).all()
        _check_y({"y": out["y"][good], "scale": out["scale"][good]}, y, group)
    # a weight that is not finite, one column of it
    w[H // 3] = math.inf
    out = cis.rms_norm(x, w, out_dtype=F8, group=32)
    at = H // 3 // 32
    sc = out["scale"][good]
    assert torch.isinf(sc[:, at]).all() and torch.isfinite(sc[:, :at]).all()
    assert torch.isnan(out["y"][good, H // 3].float()).all()
    assert torch.all(out["y"][good, at * 32:H // 3].float() == 0)
    g = cis.rms_norm_bwd(x, torch.randn(T, H, device=DEV), None)["dx"]
    assert torch.isfinite(g[good]).all() and torch.isnan(g[1]).all()


@pytest.mark.parametrize("H", [24, 700, 12000, 34000])
@pytest.mark.parametrize("size,eps", [(2.0 ** 100, 1e-6), (2.0 ** -100, 0.0), (2.0 ** -60, 1e-30),
                                      (2.0 ** 126, 0.0), (2.0 ** -120, 0.0)])
def test_sizes_of_values(H, size, eps):
    """Squares beyond float32 either way."""
    x = torch.rand(4, H, generator=_gen(H), device=DEV) + 0.5
    x = _store(x * size, F32)
    w = _rand((H,), F32, 1).contiguous()
    out = cis.rms_norm(x, w, eps=eps)
    _check_fwd(x, w, None, out, eps)
    dy = _rand((4, H), F32, 2)
    got = cis.rms_norm_bwd(dy, x, w, eps=eps)
    # (gradients beyond float32 have no place in it)
    if size > 2.0 ** -110:
        _check_bwd(dy, x, w, None, got, eps)


def test_zero_rows_and_least_scales():
    x = torch.zeros(3, 64, device=DEV)
    x[1] = 1e-37
    assert torch.all(cis.rms_norm(x, eps=1e-6)["y"][[0, 2]] == 0)
    assert torch.isnan(cis.rms_norm(x, eps=0.0)["y"][0]).all()
    out = cis.rms_norm(x, eps=1.0, out_dtype=F8)
    assert torch.all(out["scale"] == 2.0 ** -126)
    assert torch.all(out["y"][[0, 2]].float() == 0)
    # 1e-37 / 2^-126 = 8.5: halfway cases aside, the nearest e4m3 value
    assert torch.all(out["y"][1].float() == torch.tensor(1e-37 * 2.0 ** 126).to(F8).float())
    g = cis.rms_norm_bwd(torch.ones(3, 64, device=DEV), x, eps=1e-6)
    assert torch.all(g["dx"][0] == 1e3) or torch.allclose(g["dx"][0], torch.tensor(1e3, device=DEV))


def test_no_rows():
    for H in (8, 40000):
        x = torch.empty(0, H, dtype=BF, device=DEV)
        assert cis.rms_norm(x, None, x)["y"].shape == (0, H)
        assert cis.rms_norm(x, out_dtype=F8, group=32)["scale"].shape == (0, (H + 31) // 32)
        assert torch.all(cis.rms_norm_bwd(x, x)["dweight"] == 0)


def test_more_rows_than_a_launch():
    T, H = (1 << 21) + 77, 9
    x = torch.randn(T, 16, generator=_gen(1), device=DEV).to(BF)[:, :H]
    out = cis.rms_norm(x)["y"]
    f = x.float()
    want = f * torch.rsqrt((f * f).mean(1, keepdim=True) + 1e-6)
    # plain float32: rstd off by 6u there, 4u here, and half a step each
    assert torch.all((out.float() - want).abs() <= (2 * 2.0 ** -8 + 16 * U) * want.abs())
    g = cis.rms_norm_bwd(x, x)
    dw = (x.double() * (f * torch.rsqrt((f * f).mean(1, keepdim=True) + 1e-6)).double()).sum(0)
    # all terms are positive: x^2 rstd
    assert torch.all((g["dweight"].double() - dw).abs() <= 2.0 ** -10 * dw)
    _check_bwd(x[-300:], x[-300:], None, None, {"dx": g["dx"][-300:]}, 1e-6)


def test_offsets_beyond_32_bits():
    """Rows more than 2^32 bytes behind the first, by many rows and by their stride."""
    H = 8200
    T = (1 << 32) // (H * 2) + 40
    x = torch.zeros(T, H, dtype=BF, device=DEV)
    x[-30:] = _rand((30, H), BF, 1)
    w = _rand((H,), BF, 2).contiguous()
    out = cis.rms_norm(x, w, y=x)["y"]
    _check_fwd(_rand((30, H), BF, 1), w, None, {"y": out[-30:]}, 1e-6)
    far = torch.zeros(3 * (1 << 31) // 2, dtype=BF, device=DEV)
    rows = far.as_strided((3, 2048), (1 << 30, 1))
    rows.copy_(_rand((3, 2048), BF, 4))
    keep = rows.clone()
    _check_fwd(keep, None, None, cis.rms_norm(rows), 1e-6)
    g = cis.rms_norm_bwd(rows, rows, dx=rows)
    _check_bwd(keep, keep, None, None, g, 1e-6)


def test_streams_graphs_and_repeats():
    """Two calls at once, a captured and replayed one, and the same bits every time."""
    T, H = 700, 2048
    w = _rand((H,), BF, 1).contiguous()
    x, r, dy = _rand((T, H), BF, 2), _rand((T, H), F32, 3), _rand((T, H), F32, 4)
    x2 = _rand((T, H), BF, 5)
    fwd = cis.RmsNormCall(x, w, r, out_dtype=F8, group=128)
    bwd = cis.RmsNormGradCall(dy, fwd.out["residual"], w)
    snap = lambda: [t.clone() for c in (fwd, bwd) for k, t in sorted(c.out.items())]  # noqa: E731
    same = lambda a, b: all(torch.equal(p.view(torch.uint8), q.view(torch.uint8))  # noqa: E731
                            for p, q in zip(a, b))
    fwd.run(), bwd.run()
    first = snap()
    keep = x.clone()
    x.copy_(x2)
    fwd.run(), bwd.run()
    second = snap()
    assert not same(first, second)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fwd.run(), bwd.run()
    torch.cuda.current_stream().wait_stream(side)
    assert same(snap(), second)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd.run(), bwd.run()
    for rep in range(4):
        x.copy_(keep if rep % 2 == 0 else x2)
        for c in (fwd, bwd):
            for t in c.out.values():
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(snap(), first if rep % 2 == 0 else second)
        torch.randn(1000, 1000, device=DEV).sum().item()
    # two backward passes at once, each with a workspace of its own
    calls = [cis.RmsNormGradCall(dy, t, w) for t in (_rand((T, H), F32, 8), _rand((T, H), F32, 9))]
    alone = [{k: v.clone() for k, v in c.run().items()} for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for s, c in zip(streams, calls):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.run()
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for c, want in zip(calls, alone):
        assert all(torch.equal(c.out[k], want[k]) for k in want)


def test_binding_refuses():
    x = torch.zeros(4, 16, device=DEV, dtype=BF)
    w = torch.ones(16, device=DEV)
    bad = [
        lambda: cis.rms_norm(x.half()), lambda: cis.rms_norm(x, w[:8]), lambda: cis.rms_norm(x, w.half()),
        lambda: cis.rms_norm(x, torch.ones(32, device=DEV)[::2]), lambda: cis.rms_norm(x, w.cpu()),
        lambda: cis.rms_norm(x, w, x[:2]), lambda: cis.rms_norm(x.float(), w, x),
        lambda: cis.rms_norm(x, w, group=32), lambda: cis.rms_norm(x, w, out_dtype=torch.float16),
        lambda: cis.rms_norm(x, w, out_dtype=F8, group=48), lambda: cis.rms_norm(x.t(), w[:4]),
        lambda: cis.rms_norm(x, w, residual_out=x), lambda: cis.rms_norm(x, w, y=x[:2]),
        lambda: cis.rms_norm(x, w, x, residual_out=torch.zeros(4, 16, device=DEV)),
        lambda: cis.rms_norm(torch.zeros(4, 0, device=DEV)),
        lambda: cis.rms_norm_bwd(x[:2], x), lambda: cis.rms_norm_bwd(x, x, dx_dtype=torch.float16),
        lambda: cis.rms_norm_bwd(x, x, None, x.float(), dx_dtype=BF),
        lambda: cis.rms_norm_bwd(x, x, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(cis.CisError):   # rows that do not start at whole vectors
        cis.rms_norm(torch.zeros(4, 9, device=DEV, dtype=BF))
    with pytest.raises(cis.CisError):
        cis.rms_norm(x, w, eps=-1.0)
    with pytest.raises(cis.CisError):
        cis.rms_norm(x, w, y=x.expand(4, 16)[:1].expand(4, 16))
