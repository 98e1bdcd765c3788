"""The token operators on the GPU against the float64 oracle (oracle/tokens.py).

Draws and ranks are whole numbers and compared exactly. A draw's weights come from the definition's
float32 exponents through torch.exp2 on the same device, whose result equals the hardware's exp2
wherever a weight is not 0; everything after them is exact arithmetic in the oracle.

Tolerances of computed values. u = 2^-24. A softmax exponent x c - R rounds once (u |x c - R|), and
the reference and the log of the sum round once each, so for rows whose exponents stay below 128 in
base 2 a log-probability is off by at most about 2^-24 (128 + 2 * 32) ln 2 < 8e-6, a probability by
that relative, to which exp2 and the sums add below 2e-6: TOL = 1e-5.
"""

import math

import numpy as np
import pytest
import torch

import paper_2609_32444_amd as cis
from oracle import tokens as orc

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOL = 1e-5
DTYPES = [torch.bfloat16, torch.float32]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _store(z, dtype, pad=0, fill=float("nan")):
    """[T, V] logits in rows of whole 16-byte vectors and `pad` more of them; the padding holds
    NaNs, which no result may show."""
    T, V = z.shape
    epv = 16 // dtype.itemsize
    ld = (V + epv - 1) // epv * epv + pad * epv
    s = torch.full((max(T, 1), ld), fill, dtype=dtype, device=DEV)
    s[:T, :V] = z.to(dtype)
    return s[:T, :V]


def _np(t):
    return t.float().cpu().numpy()


# ------------------------------------------------------------------------------------------
# Sampling
# ------------------------------------------------------------------------------------------

def _logits(T, V, seed, kind="normal"):
    g = _gen(seed)
    z = torch.randn(T, V, generator=g, device=DEV) * 3
    if kind == "ties":
        z = z.round()
    if kind == "banned":
        z[torch.rand(T, V, generator=g, device=DEV) < 0.6] = -math.inf
    if kind == "peaked":
        z[torch.arange(T), torch.randint(0, V, (T,), generator=g, device=DEV)] += 25
    if kind == "lowest":
        z[torch.rand(T, V, generator=g, device=DEV) < 0.6] = torch.finfo(torch.bfloat16).min
    return z


def _weights(z, temp):
    """The weights of a row's draw (numpy int64) and whether the row is greedy."""
    t = orc.draw_exponents(z, temp)
    if t is None:
        t = orc.draw_exponents(z, 1.0)
        return np.where(t == 0, orc.ONE, 0).astype(np.int64), True
    w = torch.exp2(torch.from_numpy(t).to(DEV)) * orc.ONE
    return w.long().cpu().numpy(), False


def _check_sample(logits, u, out, temp=1.0, top_k=0, top_p=1.0, min_p=0.0, mask=None):
    T = logits.shape[0]
    at = lambda x, t: float(x[t]) if isinstance(x, torch.Tensor) else x  # noqa: E731
    zs, us = _np(logits), u.cpu().numpy()
    ids, lp, lk = (out[k].cpu().numpy() for k in ("ids", "logp", "logp_kept"))
    for t in range(T):
        z = zs[t]
        if (mask is not None and not mask[t]) or not orc.drawable(z):
            assert (ids[t], lp[t], lk[t]) == (-1, 0.0, 0.0), t
            continue
        q, greedy = _weights(z, at(temp, t))
        y, want = orc.draw(z, q, us[t], int(at(top_k, t)), at(top_p, t), at(min_p, t), greedy)
        assert ids[t] == y, (t, ids[t], y)
        assert abs(lk[t] - want) <= 2.0 ** -23 * abs(want)      # rounded once
        ref = orc.log_softmax_at(z, y)
        # the difference of two logits and the log of a sum round; a sum near 1 keeps its excess
        assert abs(lp[t] - ref) <= TOL * min(1.0, abs(ref)) + 2.0 ** -22 * abs(ref), (lp[t], ref)


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.6), dict(temperature=7.5),
            dict(top_k=1), dict(top_k=5), dict(top_k=40), dict(top_k=1 << 30), dict(top_p=0.3),
            dict(top_p=0.9), dict(top_p=0.999999), dict(min_p=0.1), dict(min_p=1.0),
            dict(top_k=30, top_p=0.8, min_p=0.01, temperature=1.3),
            dict(temperature=1e-3, top_p=0.5), dict(temperature=1e-42), dict(temperature=1e30)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["normal", "ties", "banned", "peaked", "lowest"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 1000, 4097])
def test_sample(V, kind, dtype):
    T = 9
    logits = _store(_logits(T, V, V + len(kind), kind), dtype, pad=V % 3)
    u = torch.rand(T, generator=_gen(V), device=DEV)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    for s in SETTINGS:
        out = cis.sample(logits, u, **s)
        kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
        _check_sample(logits, u, out, **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(3, 50257), (2, 151936), (1, 262144), (1, 300001)])
def test_sample_long_rows(T, V, dtype):
    for kind in ("normal", "ties", "banned", "peaked"):
        logits = _store(_logits(T, V, 5, kind), dtype)
        u = torch.rand(T, generator=_gen(T), device=DEV)
        for s in (dict(), dict(top_k=50, top_p=0.9, temperature=0.7), dict(top_p=0.95),
                  dict(top_k=V // 2), dict(top_k=1500), dict(min_p=0.02), dict(temperature=0.0)):
            out = cis.sample(logits, u, **s)
            kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
            _check_sample(logits, u, out, **kw)


@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "one block"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_sample_orders_of_a_row(order, dtype):
    """Rows whose large logits lie together or are all the same."""
    V = 20000
    j = torch.arange(V, device=DEV, dtype=torch.float32)
    z = {"rising": j / 2000, "falling": -j / 2000, "equal": 0 * j + 1.5,
         "two values": (j % 3 == 1).float(),
         "one block": torch.where((j >= 7000) & (j < 9000), j % 17 / 8 + 4, -j / V)}[order]
    logits = _store(z.expand(8, V), dtype)
    u = torch.linspace(0, 0.999, 8, device=DEV)
    for s in (dict(), dict(top_k=7), dict(top_k=700), dict(top_k=1024), dict(top_k=5000),
              dict(top_p=0.5), dict(top_p=0.01), dict(top_k=900, top_p=0.6), dict(min_p=0.9),
              dict(temperature=0.0)):
        out = cis.sample(logits, u, **s)
        kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
        _check_sample(logits, u, out, **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(1, 1025), (1, 40000), (5, 262144), (130, 9000), (600, 4097),
                                 (2100, 1500)])
def test_sample_top_p_over_rows_and_parts(T, V, dtype):
    """The cut of top_p by few rows in parts, by one workgroup per row, and by more rows than are
    listed at once; wide and narrow steps, min_p above and below the cut."""
    pick = slice(None, None, max(1, T // 40))
    for kind in ("normal", "ties", "peaked"):
        logits = _store(_logits(T, V, 7, kind), dtype)
        u = torch.rand(T, generator=_gen(T + V), device=DEV)
        u[0], u[-1] = 0.0, 1 - 2.0 ** -24
        for s in (dict(top_p=0.95), dict(top_p=0.5, temperature=0.7), dict(top_p=1e-6),
                  dict(top_p=0.9, min_p=0.3), dict(top_p=0.8, min_p=1e-4, temperature=2.0)):
            out = cis.sample(logits, u, **s)
            kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
            _check_sample(logits[pick], u[pick],
                          {k: v[pick] for k, v in out.items() if k != "workspace"}, **kw)


def test_sample_top_p_of_a_very_long_row():
    V = 3_900_001
    logits = _store(_logits(1, V, 2), torch.float32)
    u = torch.full((1,), 0.7, device=DEV)
    _check_sample(logits, u, cis.sample(logits, u, top_p=0.9), top_p=0.9)


def test_sample_signed_zeros_are_ties():
    z = torch.zeros(4, 32, device=DEV)
    z[:, ::2] = -0.0
    z[:, 20:] = -1
    u = torch.tensor([0.0, 0.3, 0.6, 0.99], device=DEV)
    for dtype in DTYPES:
        logits = _store(z, dtype)
        assert cis.sample(logits, u, top_k=4)["ids"].tolist() == [0, 1, 2, 3]
        assert cis.sample(logits, u, temperature=0.0)["ids"].tolist() == [0] * 4


def test_sample_rows_of_their_own():
    """Parameters per row, with some out of range: those rows are not drawn."""
    T, V = 64, 3001
    g = _gen(3)
    logits = _store(_logits(T, V, 8), torch.float32)
    u = torch.rand(T, generator=g, device=DEV)
    pick = lambda v, dt: torch.tensor(v, dtype=dt, device=DEV)[  # noqa: E731
        torch.randint(0, len(v), (T,), generator=g, device=DEV)]
    temp = pick([0.0, 0.5, 1.0, 2.0], torch.float32)
    k = pick([0, 1, 20, 1000, 5000], torch.int32)
    p = pick([0.2, 0.9, 1.0], torch.float32)
    m = pick([0.0, 0.05], torch.float32)
    mask = torch.rand(T, generator=g, device=DEV) < 0.8
    out = cis.sample(logits, u, mask, temperature=temp, top_k=k, top_p=p, min_p=m)
    _check_sample(logits, u, out, temp, k, p, m, mask.cpu().numpy())
    bad = [(temp, -1.0), (temp, math.nan), (temp, math.inf), (k, -1), (p, 0.0), (p, 1.1),
           (p, math.nan), (m, -0.1), (m, 1.5), (m, math.nan), (u, 1.0), (u, -0.1), (u, math.nan)]
    for i, (x, v) in enumerate(bad):
        x[i] = v
    out = cis.sample(logits, u, temperature=temp, top_k=k, top_p=p, min_p=m)
    assert (out["ids"][:len(bad)] == -1).all() and (out["ids"][len(bad):] >= 0).all()
    assert not out["logp"][:len(bad)].any() and not out["logp_kept"][:len(bad)].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 5000])
def test_sample_rows_without_a_draw(V, dtype):
    z = _logits(6, V, 9)
    z[0] = -math.inf
    z[1, V // 2] = math.nan
    z[2, V - 1] = math.inf
    z[3, 1:] = -math.inf
    z[4] = torch.finfo(torch.bfloat16).min
    logits = _store(z, dtype)
    u = torch.full((6,), 0.5, device=DEV)
    for s in (dict(), dict(top_k=3), dict(top_p=0.5), dict(temperature=0.0)):
        out = cis.sample(logits, u, **s)
        kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
        _check_sample(logits, u, out, **kw)
        assert out["ids"][:3].tolist() == [-1] * 3 and int(out["ids"][3]) == 0


def test_sample_feeds_the_loss():
    """The recorded log-probability is the loss's own where both see the same logits."""
    T, V = 64, 32000
    logits = _store(_logits(T, V, 4), torch.bfloat16)
    out = cis.sample(logits, torch.rand(T, generator=_gen(1), device=DEV))
    loss = cis.loss_fwd(logits, out["ids"], out["logp"], torch.ones(T, device=DEV), lam=2.3)
    assert (loss["logp_train"] - out["logp"]).abs().max() < 2e-6
    assert (loss["w"] - 1).abs().max() < 4e-6


# ------------------------------------------------------------------------------------------
# Largest logits
# ------------------------------------------------------------------------------------------

def _check_top(logits, K, out, temp=1.0, mask=None):
    zs = _np(logits)
    ids, vals, tail = (out[k].cpu().numpy() for k in ("ids", "values", "tail"))
    assert ids.shape == vals.shape == (logits.shape[0], K)
    for t, z in enumerate(zs):
        if mask is not None and not mask[t]:
            assert (ids[t] == -1).all() and (vals[t] == -np.inf).all() and tail[t] == -np.inf
            continue
        want = orc.top_list(z, K, temp)
        assert np.array_equal(ids[t], want.ids), t
        assert np.array_equal(vals[t], want.values.astype(np.float32)), t
        if math.isfinite(want.tail):
            assert abs(tail[t] - want.tail) <= TOL + 2.0 ** -22 * abs(want.tail), (t, tail[t])
        else:
            assert np.array_equal(tail[t], np.float32(want.tail), equal_nan=True), t


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["normal", "ties", "banned", "peaked", "lowest"])
@pytest.mark.parametrize("V", [1, 2, 9, 64, 1000, 4097])
def test_top(V, kind, dtype):
    T = 9
    logits = _store(_logits(T, V, V + len(kind), kind), dtype, pad=V % 3)
    for K in (1, 2, 8, 63, 256, 1000, 1024):
        _check_top(logits, K, cis.top_logits(logits, K))
    _check_top(logits, 5, cis.top_logits(logits, 5, temperature=2.5), 2.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(3, 50257), (2, 151936), (1, 262144), (1, 300001)])
def test_top_long_rows(T, V, dtype):
    for kind in ("normal", "ties", "peaked"):
        logits = _store(_logits(T, V, 6, kind), dtype)
        for K in (1, 20, 256, 1024):
            _check_top(logits, K, cis.top_logits(logits, K, temperature=0.7), 0.7)


@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "one block"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_top_orders_of_a_row(order, dtype):
    V = 20000
    j = torch.arange(V, device=DEV, dtype=torch.float32)
    z = {"rising": j / 2000, "falling": -j / 2000, "equal": 0 * j + 1.5,
         "two values": (j % 3 == 1).float(),
         "one block": torch.where((j >= 7000) & (j < 9000), j % 17 / 8 + 4, -j / V)}[order]
    logits = _store(z.expand(3, V), dtype)
    for K in (1, 7, 64, 500, 1024):
        _check_top(logits, K, cis.top_logits(logits, K))


@pytest.mark.parametrize("dtype", DTYPES)
def test_top_of_spread_rows(dtype):
    """Rows whose K-th logit lies far below the largest, near it, or among logits of every size."""
    V = 30000
    g = _gen(21)
    z = torch.randn(8, V, generator=g, device=DEV) * 3
    z[0, 5000] += 40.0                                     # one logit stands out
    z[1, torch.arange(0, V, 97, device=DEV)] += 300.0      # some 300 do
    z[2] = z[2] * 1e30
    z[3] = z[3] * 1e-30
    z[4] = torch.sign(z[4]) * torch.exp(z[4] * 10)         # every size
    z[5] = z[5] * 1e-3 + 100.0                             # close together
    z[6, 17], z[6, 18] = 3e38, 2.9e38
    z[7] = torch.where(z[7] > 6, z[7] + 1000, z[7] / 1000)
    logits = _store(z, dtype)
    u = torch.rand(8, generator=g, device=DEV)
    for K in (1, 5, 64, 256, 310, 1000):
        _check_top(logits, K, cis.top_logits(logits, K))
        _check_sample(logits, u, cis.sample(logits, u, top_k=K), top_k=K)


def test_top_masked_and_not_finite():
    V, K = 3000, 40
    z = _logits(8, V, 12)
    z[1, 17] = math.nan
    z[2, 2999] = math.inf
    z[3] = -math.inf
    z[4, 10:] = -math.inf
    mask = torch.tensor([1, 1, 1, 1, 1, 0, 1, 0], dtype=torch.uint8, device=DEV)
    for dtype in DTYPES:
        logits = _store(z, dtype, pad=2)
        _check_top(logits, K, cis.top_logits(logits, K, mask), mask=mask.cpu().numpy())


# ------------------------------------------------------------------------------------------
# Distillation
# ------------------------------------------------------------------------------------------

def _teacher(zt, K, temp, seed, holes=0.0):
    """Lists of the teacher's logits [T, V], in a shuffled order, some entries empty."""
    T, V = zt.shape
    K = min(K, V)
    v, i = zt.topk(K, dim=1)
    tail = torch.logsumexp((zt / temp).scatter(1, i, -math.inf), dim=1)
    perm = torch.rand(T, K, generator=_gen(seed), device=DEV).argsort(1)
    v, i = v.gather(1, perm), i.gather(1, perm)
    hole = torch.rand(T, K, generator=_gen(seed + 1), device=DEV) < holes
    return torch.where(hole, -1, i).to(torch.int32), v.contiguous(), tail


def _bf16_step(x):
    return np.maximum(np.abs(x) * 2.0 ** -8, 2.0 ** -126)


def _check_distill(logits, ids, values, tail, out, *, reverse=False, temp=1.0, scale=1.0,
                   weight=None, mask=None):
    zs, i, v = _np(logits), ids.cpu().numpy(), values.cpu().numpy()
    tl = None if tail is None else tail.cpu().numpy()
    terms = out["terms"].cpu().numpy()
    grads = _np(out["dlogits"]) if "dlogits" in out else None
    bf16 = logits.dtype == torch.bfloat16
    loss, size, n_valid, n_bad = 0.0, 0.0, 0, 0
    for t in range(zs.shape[0]):
        w = 1.0 if weight is None else float(weight[t])
        r = orc.distill_row(zs[t], i[t], v[t], None if tl is None else tl[t], reverse, temp, w,
                            float(np.float32(scale)), mask is None or bool(mask[t]))
        n_valid += r.valid
        n_bad += r.bad
        if not r.valid:
            assert terms[t] == 0.0
            assert grads is None or not grads[t].any(), t
            continue
        cf = abs(w * scale)
        # errors of the log-probabilities, weighed by the class's share of the first argument
        d = math.sqrt(2 * max(r.kl, 0.0)) + 1e-6
        assert abs(terms[t] - r.term) <= cf * (4 * TOL * d + 8 * TOL * TOL) + 4e-6 * abs(r.term), \
            (t, terms[t], r.term)
        loss, size = loss + r.term, size + abs(r.term) + cf * TOL * d
        if grads is None:
            continue
        listed = np.zeros(zs.shape[1], bool)
        listed[i[t][i[t] >= 0]] = True
        ratio = r.q_rest / r.p_rest if r.p_rest > 0 else 0.0
        err = 2 * TOL * np.where(listed, r.p + r.q, r.p * (1 + ratio))
        if reverse:
            with np.errstate(divide="ignore", invalid="ignore"):
                dd = np.abs(r.grad * temp / (w * scale if cf else 1.0))
            err += 2 * TOL * (r.p * (1 + abs(r.kl)) + np.nan_to_num(dd))
        tol = err * cf / temp + 2e-6 * np.abs(r.grad) + 2.0 ** -126
        if bf16:
            tol = tol + _bf16_step(r.grad)
        off = np.abs(grads[t] - r.grad)
        assert (off <= tol).all(), (t, int((off > tol).sum()), float((off / tol).max()))
    assert abs(float(out["loss"]) - loss) <= 8 * size * TOL + 2.0 ** -23 * abs(loss) + 1e-12
    st = cis.read_stats(out["workspace"])
    assert (st["n_valid"], st["n_bad_id"], st["n_nonfinite"]) == (n_valid, n_bad, 0)


KINDS = [dict(), dict(tail=False), dict(reverse=True), dict(temp=2.0, scale=0.01),
         dict(temp=0.5, reverse=True, scale=-3.0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,K", [(1, 1), (2, 1), (7, 7), (9, 3), (65, 64), (1000, 16), (1024, 1),
                                 (1025, 200), (5003, 1024), (50257, 64), (151936, 256),
                                 (262144, 33)])
def test_distill(V, K, dtype):
    T = 5 if V < 10000 else 2
    zt = torch.randn(T, V, generator=_gen(V + K), device=DEV) * 2.5
    z = zt + torch.randn(T, V, generator=_gen(V), device=DEV)
    logits = _store(z, dtype, pad=K % 3)
    for n, s in enumerate(KINDS):
        temp = s.get("temp", 1.0)
        ids, values, tail = _teacher(zt, K, temp, n)
        tail = tail if s.get("tail", True) else None
        if s.get("reverse") and K >= V:
            continue   # the tail is empty: the student's share of it is not covered
        kw = dict(kind=cis.KL_REVERSE if s.get("reverse") else cis.KL_FORWARD, temperature=temp,
                  scale=s.get("scale", 1.0))
        ref = dict(reverse=s.get("reverse", False), temp=temp, scale=s.get("scale", 1.0))
        out = cis.distill_bwd(logits, ids, values, tail, **kw)
        _check_distill(logits, ids, values, tail, out, **ref)
        fwd = cis.distill_fwd(logits, ids, values, tail, **kw)
        _check_distill(logits, ids, values, tail, fwd, **ref)


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_lists_of_neighbours(dtype):
    """Lists that fill whole vectors, run along the row, or meet in one place of the table."""
    T, V = 3, 300000
    zt = torch.randn(T, V, generator=_gen(1), device=DEV) * 2
    logits = _store(zt + torch.randn(T, V, generator=_gen(2), device=DEV), dtype)
    for stride, K in ((1, 1024), (8, 500), (4, 37), (65536, 4), (32768, 9), (293, 1023)):
        ids = (torch.arange(K, device=DEV) * stride % V).to(torch.int32).expand(T, K).contiguous()
        ids[1] = V - 1 - ids[1]
        values = zt.gather(1, ids.long())
        tail = torch.logsumexp(zt.scatter(1, ids.long(), -math.inf), dim=1)
        for reverse in (False, True):
            out = cis.distill_bwd(logits, ids, values, tail,
                                  kind=cis.KL_REVERSE if reverse else cis.KL_FORWARD)
            _check_distill(logits, ids, values, tail, out, reverse=reverse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [100, 9000])
def test_distill_rows_that_do_not_count(V, dtype):
    """Masked rows, empty lists, ids out of range, repeated ids, weights of 0, empty entries."""
    T, K = 12, 10
    zt = torch.randn(T, V, generator=_gen(1), device=DEV) * 2
    logits = _store(zt + torch.randn(T, V, generator=_gen(2), device=DEV), dtype, pad=1)
    ids, values, tail = _teacher(zt, K, 1.0, 3)
    ids[1] = -1
    ids[2, 3] = V
    ids[3, 0] = -2
    ids[4, 7] = ids[4, 2]
    ids[5, 1:] = -1
    ids[6, ::2] = -1
    ids[9] = ids[9, 0]
    weight = torch.rand(T, generator=_gen(4), device=DEV)
    weight[7] = 0.0
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[8] = 0
    tail = torch.logsumexp(  # of what the lists have left
        torch.stack([zt[t].index_fill(0, ids[t][(ids[t] >= 0) & (ids[t] < V)].long(), -math.inf)
                     for t in range(T)]), dim=1)
    for reverse in (False, True):
        out = cis.distill_bwd(logits, ids, values, tail, weight, mask,
                              kind=cis.KL_REVERSE if reverse else cis.KL_FORWARD)
        _check_distill(logits, ids, values, tail, out, reverse=reverse, weight=weight, mask=mask)
    every = cis.distill_bwd(logits, ids, values, tail, weight, torch.zeros_like(mask))
    assert not every["terms"].any() and not every["dlogits"].any() and float(every["loss"]) == 0


def test_distill_not_finite_rows_are_counted():
    T, V, K = 6, 500, 4
    zt = torch.randn(T, V, generator=_gen(1), device=DEV)
    z = zt.clone()
    z[0, 3] = math.nan
    z[1, 3] = math.inf
    z[2] = -math.inf
    ids, values, tail = _teacher(zt, K, 1.0, 2)
    values[3, 1] = math.nan
    tail[4] = math.inf
    for dtype in DTYPES:
        out = cis.distill_bwd(_store(z, dtype), ids, values, tail)
        st = cis.read_stats(out["workspace"])
        assert (st["n_valid"], st["n_bad_id"], st["n_nonfinite"]) == (6, 0, 5)
        assert math.isfinite(float(out["terms"][5]))


def test_distill_student_far_from_its_teacher():
    """A student whose mass is all outside, or all inside, the list."""
    T, V, K = 4, 2000, 8
    zt = torch.randn(T, V, generator=_gen(1), device=DEV)
    ids, values, tail = _teacher(zt, K, 1.0, 2)
    z = zt.clone()
    z[0].index_add_(0, ids[0].long(), torch.full((K,), 30.0, device=DEV))
    z[1].index_add_(0, ids[1].long(), torch.full((K,), -30.0, device=DEV))
    z[2].index_fill_(0, ids[2].long(), 60.0)
    logits = _store(z, torch.float32)
    for reverse in (False, True):
        out = cis.distill_bwd(logits, ids, values, tail,
                              kind=cis.KL_REVERSE if reverse else cis.KL_FORWARD)
        _check_distill(logits, ids, values, tail, out, reverse=reverse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(7, 1001), (5, 50257), (300, 2048)])
def test_distill_in_place_and_padding(T, V, dtype):
    """The gradient may replace the logits; columns past V are left alone."""
    zt = torch.randn(T, V, generator=_gen(1), device=DEV) * 2
    logits = _store(zt + 1e-1 * torch.randn(T, V, generator=_gen(2), device=DEV), dtype, pad=2,
                    fill=7.0)
    ids, values, tail = _teacher(zt, 20, 1.0, 3)
    g = torch.full_like(_store(zt, dtype, pad=3, fill=5.0)._base, 5.0)[:, :V]
    out = cis.distill_bwd(logits, ids, values, tail, dlogits=g)
    assert (g._base[:, V:] == 5.0).all()
    inp = logits._base.clone()[:, :V]
    res = cis.distill_bwd(inp, ids, values, tail, dlogits=inp)
    assert torch.equal(inp, out["dlogits"]) and torch.equal(res["terms"], out["terms"])
    assert (inp._base[:, V:] == 7.0).all()


def test_distill_strided_lists():
    """Lists that are the first columns of longer ones."""
    T, V = 40, 3000
    zt = torch.randn(T, V, generator=_gen(1), device=DEV) * 2
    logits = _store(zt + torch.randn(T, V, generator=_gen(2), device=DEV), torch.bfloat16)
    top = cis.top_logits(_store(zt, torch.float32), 100)
    ids, values = top["ids"][:, :30], top["values"][:, :30]
    tail = torch.logsumexp(zt.scatter(1, ids.long(), -math.inf), dim=1)
    out = cis.distill_bwd(logits, ids, values, tail)
    _check_distill(logits, ids, values, tail, out)


def test_lists_feed_the_distillation():
    """A student at its teacher, through the teacher's list: no loss, no gradient beyond
    rounding."""
    T, V = 50, 20000
    z = _store(torch.randn(T, V, generator=_gen(1), device=DEV) * 3, torch.float32)
    for temp in (1.0, 2.0):
        top = cis.top_logits(z, 100, temperature=temp)
        for kind in (cis.KL_FORWARD, cis.KL_REVERSE):
            out = cis.distill_bwd(z, top["ids"], top["values"], top["tail"], kind=kind,
                                  temperature=temp)
            assert out["terms"].abs().max() < TOL * TOL and out["dlogits"].abs().max() < 2 * TOL


# ------------------------------------------------------------------------------------------
# Calls
# ------------------------------------------------------------------------------------------

def _calls(T, V, seed, dtype=torch.bfloat16, K=24):
    zt = torch.randn(T, V, generator=_gen(seed), device=DEV) * 2.5
    logits = _store(zt, dtype)
    ids, values, tail = _teacher(zt + 0.3 * torch.randn(T, V, generator=_gen(seed + 1), device=DEV),
                                 K, 1.0, 3)
    u = torch.rand(T, generator=_gen(seed + 2), device=DEV)
    mask = (torch.rand(T, generator=_gen(seed + 3), device=DEV) < 0.9).to(torch.uint8)
    return [cis.SampleCall(logits, u, mask, top_k=50, top_p=0.9, temperature=0.8),
            cis.SampleCall(logits, u, mask), cis.SampleCall(logits, u, mask, top_p=0.9),
            cis.TopLogitsCall(logits, K, mask),
            cis.DistillCall(logits, ids, values, tail, None, mask, bwd=False),
            cis.DistillCall(logits, ids, values, tail, None, mask)], (logits, ids, values, tail, u)


def _copy(out):
    return {k: v.clone() for k, v in out.items() if k != "workspace"}


def _same(a, b):
    return all(torch.equal(a[k].contiguous().view(torch.uint8), b[k].contiguous().view(torch.uint8))
               for k in a)


SHAPES = [(1, 50257), (64, 50257), (700, 8192), (3000, 1000), (40, 151936)]


@pytest.mark.parametrize("T,V", SHAPES)
def test_calls_repeat_bit_for_bit_and_run_on_other_streams(T, V):
    calls, _ = _calls(T, V, 31)
    first = [_copy(c.run()) for c in calls]
    others, _ = _calls(T, V, 77)
    for rep in range(2):
        side = [torch.cuda.Stream() for _ in range(2)]
        for s in side:
            s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side[0]):
            got = [c.run() for c in calls]
        with torch.cuda.stream(side[1]):
            for c in others:
                c.run()
        for s in side:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(first, got)):
            assert _same(a, b), (rep, i)


@pytest.mark.parametrize("T,V", [(1, 50257), (300, 8192), (40, 151936)])
def test_calls_in_a_graph(T, V):
    """Captured once, replayed on rewritten inputs with eager work and a synchronisation between."""
    calls, ins = _calls(T, V, 5)
    _, other = _calls(T, V, 6)
    for c in calls:
        c.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for c in calls:
            c.run()
    keep = [x.clone() for x in ins]
    for rep in range(4):
        for x, y in zip(ins, other if rep % 2 else keep):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        got = [_copy(c.out) for c in calls]
        junk = torch.randn(1 << 20, device=DEV).sum()
        torch.cuda.synchronize()
        want = [_copy(c.run()) for c in calls]
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert _same(a, b), (rep, i, float(junk))


def test_no_rows():
    z = torch.empty(0, 64, device=DEV, dtype=torch.bfloat16)
    e = torch.empty(0, device=DEV)
    assert cis.sample(z, e)["ids"].shape == (0,)
    assert cis.top_logits(z, 4)["ids"].shape == (0, 4)
    out = cis.distill_bwd(z, torch.empty(0, 4, dtype=torch.int32, device=DEV),
                          torch.empty(0, 4, device=DEV), e)
    torch.cuda.synchronize()
    assert float(out["loss"]) == 0.0 and cis.read_stats(out["workspace"])["n_valid"] == 0


def test_wrong_arguments_are_refused():
    z = torch.zeros(4, 64, device=DEV)
    u = torch.zeros(4, device=DEV)
    ids = torch.zeros(4, 2, dtype=torch.int32, device=DEV)
    vals = torch.zeros(4, 2, device=DEV)
    for bad in (lambda: cis.sample(z, u[:3]), lambda: cis.sample(z, u.double()),
                lambda: cis.sample(z.half(), u), lambda: cis.sample(z, u, top_k=u),
                lambda: cis.sample(z, u, temperature=torch.zeros(3, device=DEV)),
                lambda: cis.top_logits(z, 0), lambda: cis.top_logits(z, 1025),
                lambda: cis.top_logits(z.t(), 2),
                lambda: cis.distill_bwd(z, ids.long(), vals),
                lambda: cis.distill_bwd(z, ids, vals[:, :1]),
                lambda: cis.distill_bwd(z, ids, vals, u[:2]),
                lambda: cis.distill_bwd(z, ids, vals, dlogits=z.bfloat16()),
                lambda: cis.sample(z, u, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cis.sample(z, u, top_p=0.0), lambda: cis.sample(z, u, temperature=-1.0),
                lambda: cis.sample(z, u, top_k=-3), lambda: cis.sample(z, u, min_p=2.0),
                lambda: cis.top_logits(z, 2, temperature=0.0),
                lambda: cis.distill_bwd(z, ids, vals, kind=cis.KL_REVERSE),
                lambda: cis.distill_bwd(z, ids, vals, temperature=math.nan),
                lambda: cis.sample(z[:, 1:], u)):
        with pytest.raises(cis.CisError):
            bad()


def test_rows_beyond_4_gib():
    """Row offsets past 2^32 bytes and past 2^31 elements."""
    T, V, K = 16500, 131080, 6
    logits = torch.zeros(T, V, dtype=torch.bfloat16, device=DEV)
    assert logits.numel() > 1 << 31
    last = torch.randn(3, V, generator=_gen(1), device=DEV) * 3
    logits[-3:] = last.bfloat16()
    u = torch.rand(T, generator=_gen(2), device=DEV)
    out = cis.sample(logits, u)
    tail3 = {k: v[-3:] for k, v in out.items() if k != "workspace"}
    _check_sample(logits[-3:], u[-3:], tail3)
    at = (u[:-3].double() * float(V * orc.ONE)).long() // orc.ONE   # equal logits
    assert torch.equal(out["ids"][:-3], at)
    top = cis.top_logits(logits, K)
    _check_top(logits[-3:], K, {k: v[-3:] for k, v in top.items() if k != "workspace"})
    assert (top["ids"][:-3] == torch.arange(K, device=DEV)).all()
    g = cis.distill_bwd(logits, top["ids"], top["values"], top["tail"], dlogits=logits.clone())
    assert float(g["loss"]) < 1e-3 and not g["dlogits"].isnan().any()
    ids, values, tail = _teacher(last + torch.randn_like(last), K, 1.0, 3)
    i, v, tl = top["ids"].clone(), top["values"].clone(), top["tail"].clone()
    i[-3:], v[-3:], tl[-3:] = ids, values, tail
    out = cis.distill_bwd(logits, i, v, tl)
    sub = cis.distill_bwd(logits[-3:].clone(), ids, values, tail)
    _check_distill(logits[-3:], ids, values, tail, sub)
    assert (out["dlogits"][-3:].float() - sub["dlogits"].float()).abs().max() < 1e-2
    assert (out["terms"][-3:] - sub["terms"]).abs().max() < TOL


def test_shared_lists_are_refused():
    """Lists that all rows share have the storage of one row."""
    T, V, K = 5, 64, 4
    z = torch.zeros(T, V, device=DEV)
    ids = torch.arange(K, dtype=torch.int32, device=DEV).expand(T, K)
    values = torch.zeros(K, device=DEV).expand(T, K)
    for call in (cis.distill_fwd, cis.distill_bwd):
        with pytest.raises(ValueError, match="share storage"):
            call(z, ids, values)
    out = cis.distill_fwd(z, ids.contiguous(), values.contiguous())
    _check_distill(z, ids, values, None, out)
    out = cis.distill_fwd(z[:1], ids[:1], values[:1])
    _check_distill(z[:1], ids[:1], values[:1], None, out)


def test_top_k_beyond_int32_keeps_every_token():
    logits = _store(_logits(40, 500, 3), torch.float32)
    u = torch.rand(40, generator=_gen(5), device=DEV)
    for k in (2 ** 31, 2 ** 32 + 5):
        _check_sample(logits, u, cis.sample(logits, u, top_k=k), top_k=0)
    with pytest.raises(cis.CisError):
        cis.sample(logits, u, top_k=-2 ** 32)


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, 2100), (torch.float32, 1050)])
def test_lists_and_draws_of_logits_beyond_the_caches(dtype, T):
    """More than 192 MiB of logits, which the scan does not keep for a later read."""
    V = 50003
    logits = _store(_logits(T, V, 13, "peaked"), dtype)
    assert logits.stride(0) * T * dtype.itemsize > 192 << 20
    u = torch.rand(T, generator=_gen(14), device=DEV)
    rows = torch.randperm(T, generator=torch.Generator().manual_seed(1))[:40].to(DEV)

    def some(out):
        return {k: v[rows] for k, v in out.items() if k != "workspace"}

    for K in (8, 256, 1024):
        _check_top(logits[rows], K, some(cis.top_logits(logits, K)))
    for s in (dict(), dict(top_k=20), dict(top_k=2000), dict(top_p=0.9),
              dict(top_k=900, top_p=0.8, min_p=0.001)):
        _check_sample(logits[rows], u[rows], some(cis.sample(logits, u, **s)), **s)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temp", [2.0 ** -64, 1e-9, 1e-3, 30.0, 2.0 ** 64])
@pytest.mark.parametrize("V", [40, 3000, 60000])
def test_top_tail_at_the_ends_of_the_temperatures(V, temp, dtype):
    """The tail far from 0, where all but one of its terms vanish, and where all are alike."""
    z = _logits(5, V, 17)
    z[1] += 100.0
    z[2] -= 3000.0
    z[3, :V // 2] = torch.finfo(torch.bfloat16).min * 1e-20
    logits = _store(z, dtype)
    for K in (1, 30, 300):
        _check_top(logits, K, cis.top_logits(logits, K, temperature=temp), temp)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_rows_than_a_launch_takes(dtype):
    """2^20 rows are one launch of a workgroup each."""
    T, V = (1 << 20) + 77, 24
    logits = _store(_logits(T, V, 19), dtype)
    u = torch.rand(T, generator=_gen(20), device=DEV)
    rows = torch.tensor([0, 5, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T - 1], device=DEV)

    def some(out):
        return {k: v[rows] for k, v in out.items() if k != "workspace"}

    for s in (dict(), dict(top_k=3), dict(top_p=0.7, min_p=0.1), dict(temperature=0.0)):
        kw = {{"temperature": "temp"}.get(k, k): v for k, v in s.items()}
        out = cis.sample(logits, u, **s)
        assert (out["ids"] >= 0).all()
        _check_sample(logits[rows], u[rows], some(out), **kw)
    _check_top(logits[rows], 5, some(cis.top_logits(logits, 5)))
