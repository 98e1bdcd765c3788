"""The distillation loss on the GPU against its formulas in 64 bits, in log space: classes of any size
beside each other, logits and temperatures anywhere in their ranges.

Tolerances, u = 2^-24. A class's log-probability comes from the exponent of a difference of logits,
x = (z - M) / temperature, which takes four roundings (the difference, the factor's two, the product:
8 u |x| leaves room), minus the log of a sum, of which
  * the terms have their own exponents' errors, weighed by their shares (8 u E|x|),
  * the sum has 4 roundings for every vector that a thread adds and 40 u for the rest of the tree,
  * the log and the conversion to natural units round at its own size (4 u of either);
64 u cover the hardware's exp2, log and the last roundings. What follows from the log-probabilities
has these errors times its derivatives, and 32 u of its own for its arithmetic."""

import math

import pytest
import torch

import paper_2609_32444_amd as cis

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
INF = math.inf
DTYPES = [torch.bfloat16, torch.float32]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _store(z, dtype, pad=0, fill=float("nan")):
    """[T, V] logits in rows of whole 16-byte vectors, the padding holding NaNs."""
    T, V = z.shape
    epv = 16 // dtype.itemsize
    ld = (V + epv - 1) // epv * epv + pad * epv
    s = torch.full((max(T, 1), ld), fill, dtype=dtype, device=DEV)
    s[:T, :V] = z.to(dtype)
    return s[:T, :V]


def _lists(zt, K, temp, seed=0, tail=True, holes=0.0):
    """The K largest logits of a teacher [T, V] in a shuffled order, some entries empty, and the
    log-sum-exp of what the lists leave."""
    T, V = zt.shape
    K = min(K, V)
    v, i = zt.topk(K, dim=1)
    perm = torch.rand(T, K, generator=_gen(seed), device=DEV).argsort(1)
    v, i = v.gather(1, perm).contiguous(), i.gather(1, perm).to(torch.int32)
    i[torch.rand(T, K, generator=_gen(seed + 1), device=DEV) < holes] = -1
    if not tail:
        return i, v, None
    out = torch.zeros(T, V + 1, dtype=torch.bool, device=DEV)
    out.scatter_(1, torch.where(i < 0, V, i).long(), True)
    y = (zt.double() / temp).masked_fill(out[:, :V], -INF)
    return i, v, torch.logsumexp(y, 1).float()


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _classes(x, rest):
    """log shares of the classes (x [T, K], rest [T]; -inf: nothing) and the log of the whole."""
    lse = torch.logaddexp(torch.logsumexp(x, 1), rest)
    share = torch.cat([x, rest[:, None]], 1) - lse[:, None]
    near = -torch.log1p(torch.exp(torch.logsumexp(x, 1) - rest))
    share[:, -1] = torch.where(rest > torch.logsumexp(x, 1), near, share[:, -1])
    return share, lse


def _kl_parts(la, lb):
    """a log(a / b) - a + b of each class."""
    a, b, d = la.exp(), lb.exp(), la - lb
    part = torch.where(d.abs() < 0.5, a * (torch.expm1(-d) + d), a * d - a + b)
    return torch.where(la == -INF, b, part)


def _minus(la, lb):
    """a - b."""
    d = la - lb
    return torch.where(d.abs() < 0.5, lb.exp() * torch.expm1(d), la.exp() - lb.exp())


def _zero(x, where):
    return torch.where(where, torch.zeros_like(x), x)


def _check(logits, ids, values, tail, out, *, reverse=False, temp=1.0, scale=1.0, weight=None,
           mask=None, rows=slice(None), n_nonfinite=0, stats=True):
    """All rows of a call, or `rows` of them (stats=False: their outputs alone)."""
    pick = lambda t: None if t is None else t[rows]  # noqa: E731
    z, ids, values, tail, weight, mask = map(pick, (logits, ids, values, tail, weight, mask))
    bf16, z = z.dtype == torch.bfloat16, z.double()
    T, V = z.shape
    temp, scale = _f32(temp), _f32(scale)
    on = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask != 0
    ids = ids.long()
    inside = (ids >= 0) & (ids < V)
    at = torch.where(inside, ids, V)
    count = torch.zeros(T, V + 1, device=DEV).scatter_add_(1, at, torch.ones_like(at).float())
    bad = on & (((ids != -1) & ~inside).any(1) | (count[:, :V] > 1).any(1))
    valid = on & ~bad & inside.any(1)
    listed = count[:, :V] > 0
    # the student's and the teacher's exponents, relative to their largest; log shares
    y = z / temp
    x = y - y.amax(1, keepdim=True)
    xk = x.gather(1, torch.where(inside, ids, 0)).masked_fill(~inside, -INF)
    xr = x.masked_fill(listed, -INF)
    lr = torch.logsumexp(xr, 1)
    lp, p_lse = _classes(xk, lr)
    t = (values.double() / temp).masked_fill(~inside, -INF)
    tt = torch.full_like(lr, -INF) if tail is None else tail.double()
    top = torch.maximum(t.amax(1), tt)[:, None]
    t, tt = t - top, tt - top[:, 0]
    lq, q_lse = _classes(t, tt)
    p, q = lp.exp(), lq.exp()
    none = (lp == -INF) & (lq == -INF)   # empty entries, and a rest that neither has
    d = _zero(lp - lq, none)
    kl = _zero(_kl_parts(lp, lq) if reverse else _kl_parts(lq, lp), none).sum(1)
    factor = p * (d - kl[:, None]) if reverse else _minus(lp, lq)
    factor = _zero(factor, lp == -INF if reverse else none)
    part = torch.exp(xr - lr[:, None]).masked_fill((lr == -INF)[:, None], 0.0)
    w = scale * (1.0 if weight is None else weight.double()) * torch.ones(T, device=DEV).double()
    w = torch.where(valid, w, 0.0)
    cf = (w / temp)[:, None]
    # errors of the log-probabilities
    vecs = min(20, -(-V * logits.element_size() // 16) // 64 + 1)
    own = 64 + 40 + 4 * vecs

    def size(x):
        return torch.where(x == -INF, 0.0, x).abs()

    spread = (x.exp() * size(x)).sum(1) / p_lse.exp()
    ep = U * (8 * size(torch.cat([xk, lr[:, None]], 1)) + 4 * size(lp)
              + (8 * spread + 4 * p_lse.abs() + own)[:, None])
    spread = (t.exp() * size(t)).sum(1) / q_lse.exp()
    eq = U * (8 * size(torch.cat([t, tt[:, None]], 1)) + 4 * size(lq)
              + (8 * spread + 4 * q_lse.abs() + own)[:, None])
    first, second, ef, es = (p, q, ep, eq) if reverse else (q, p, eq, ep)
    moved = _zero(first * d, first == 0).abs() * (ef + 32 * U) + (q - p).abs() * (es + 32 * U)
    e_kl = _zero(moved, none).sum(1) + 32 * U * kl + 2.0 ** -120
    terms, tol_t = _zero(w * kl, w == 0), w.abs() * e_kl
    assert not out["terms"][rows][~valid].any()
    got = out["terms"][rows].double()
    fine = (got - terms).abs() <= tol_t
    assert fine.all(), (int((~fine).sum()), got[~fine][:4], terms[~fine][:4], tol_t[~fine][:4])
    if stats:
        loss = float(out["loss"])
        assert abs(loss - float(terms.sum())) <= float(tol_t.sum()) + 64 * U * float(terms.abs().sum())
        st = cis.read_stats(out["workspace"])
        assert (st["n_valid"], st["n_bad_id"], st["n_nonfinite"]) == (int(valid.sum()),
                                                                      int(bad.sum()), n_nonfinite)
    if "dlogits" not in out:
        return
    if reverse:
        e_factor = size(factor) * ep + p * (ep + eq + e_kl[:, None])
    else:
        e_factor = p * ep + q * eq
    e_factor = _zero(e_factor + 32 * U * size(factor), none)
    grad = part * factor[:, -1:]
    tol = part * e_factor[:, -1:] + grad.abs() * U * (8 * size(x) + own
                                                      + (8 * spread.abs() + 32)[:, None])

    def put(a, b):   # (empty entries go to a column of their own)
        return torch.cat([a, a[:, :1]], 1).scatter_(1, at, b)[:, :V]

    grad, tol = put(grad, factor[:, :-1]) * cf, put(tol, e_factor[:, :-1]) * cf.abs()
    grad, tol = _zero(grad, cf == 0), tol + 2.0 ** -126
    if bf16:
        tol = tol + grad.abs() * 2.0 ** -8
    got = out["dlogits"][rows].double()
    off = (got - grad).abs()
    fine = off <= tol
    assert fine.all(), (int((~fine).sum()), (~fine).nonzero()[:4].tolist(), got[~fine][:4],
                        grad[~fine][:4], tol[~fine][:4])


def _both(logits, ids, values, tail, **kw):
    """The loss alone and with its gradient."""
    args = dict(kind=cis.KL_REVERSE if kw.get("reverse") else cis.KL_FORWARD,
                temperature=kw.get("temp", 1.0), scale=kw.get("scale", 1.0))
    w, m = kw.get("weight"), kw.get("mask")
    for call in (cis.distill_fwd, cis.distill_bwd):
        _check(logits, ids, values, tail, call(logits, ids, values, tail, w, m, **args), **kw)


# Rows of the fused pass (a wave's, and 256 threads'), and of the pass in parts.
WIDTHS = [(1000, 0), (3000, 1), (10000, 0), (20000, 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temp", [1.0, 0.1, 0.01, 0.001, 50.0])
@pytest.mark.parametrize("V,pad", WIDTHS)
def test_logits_far_from_zero(V, pad, temp, dtype):
    """What is common to a row's logits is of no account, however large beside the temperature."""
    T, K = 6, 40
    g = _gen(V)
    zt = torch.randn(T, V, generator=g, device=DEV) * (2.0 * temp)
    noise = torch.randn(T, V, generator=g, device=DEV) * temp
    for offset in (0.0, 100.0, -1000.0, 30000.0):
        # (rounded as stored first: the teacher has lists of the same numbers)
        teacher = _store(zt + offset, dtype).float()
        logits = _store(teacher + noise, dtype, pad=pad)
        for tail, reverse in ((False, False), (True, False), (True, True)):
            lists = _lists(teacher, K, temp, tail=tail)
            _both(logits, *lists, temp=temp, reverse=reverse, scale=0.25)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temp", [1e-6, 1e-9, 2.0 ** -64, 1e9, 2.0 ** 64])
@pytest.mark.parametrize("V,pad", WIDTHS)
def test_temperatures_at_the_ends_of_their_range(V, pad, temp, dtype):
    T, K = 6, 40
    g = _gen(V + 1)
    zt = torch.randn(T, V, generator=g, device=DEV) * 2
    logits = _store(zt + 0.1 * torch.randn(T, V, generator=g, device=DEV) + 7.0, dtype, pad=pad)
    lists = _lists(_store(zt, dtype).float(), K, temp, tail=False)
    _both(logits, *lists, temp=temp)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,pad", WIDTHS)
def test_rows_of_the_lowest_value(V, pad, dtype):
    """Logits set to the type's lowest value: the whole row, the listed ones, all others."""
    T, K = 4, 12
    g = _gen(V + 2)
    lowest = torch.finfo(dtype).min
    zt = torch.randn(T, V, generator=g, device=DEV) * 2
    ids, values, tail = _lists(zt, K, 1.0)
    z = zt + torch.randn(T, V, generator=g, device=DEV)
    z[0] = lowest
    z[1].index_fill_(0, ids[1].long(), lowest)
    z[2, torch.rand(V, generator=g, device=DEV) < 0.7] = lowest
    z[3] = z[3].index_copy(0, ids[3].long(), torch.full((K,), 1.0, device=DEV))
    logits = _store(z, dtype, pad=pad)
    # (a listed token of the lowest value makes a forward KL of some 1e38)
    _both(logits, ids, values, tail, scale=1e-6)
    alone = z.index_fill(0, torch.tensor([0, 1], device=DEV), lowest)
    alone = torch.full_like(alone, lowest).scatter(1, ids.long(), values)
    _both(_store(alone, dtype, pad=pad), ids, values, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gap", [20.0, 60.0, 90.0, 140.0, 500.0])
@pytest.mark.parametrize("V,pad", WIDTHS)
def test_classes_far_below_each_other(V, pad, gap, dtype):
    """Listed tokens, or all others, with probabilities far below what 32 bits hold: their logarithms
    are ordinary numbers, and so are the loss and its gradient."""
    T, K = 6, 10
    g = _gen(V + 3)
    zt = torch.randn(T, V, generator=g, device=DEV)
    ids, values, tail = _lists(zt, K, 1.0, holes=0.1)
    listed = torch.zeros(T, V, dtype=torch.bool, device=DEV)
    listed.scatter_(1, torch.where(ids < 0, ids.max(1, keepdim=True).values, ids).long(), True)
    z = zt + torch.randn(T, V, generator=g, device=DEV)
    z[0] += listed[0] * gap             # the student has next to nothing outside the list
    z[1] -= listed[1] * gap             # ... or within it
    z[2, ids[2].max()] += gap           # ... or all of it in one token
    far = tail.clone()
    far[3] -= gap                       # the teacher has next to nothing outside the list
    far[4] += gap                       # ... or within it
    z[5] += listed[5] * gap             # both of them
    far[5] -= gap
    weight = torch.rand(T, generator=g, device=DEV) + 0.5
    for scale in (1.0, 65536.0):
        for reverse in (False, True):
            _both(_store(z, dtype, pad=pad), ids, values, far, weight=weight, reverse=reverse,
                  scale=scale)
    # by the temperature alone
    for reverse in (False, True):
        _both(_store(z, dtype, pad=pad), ids, values, tail / 0.05, temp=0.05, reverse=reverse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,pad", WIDTHS)
def test_weight_of_zero_in_rows_that_are_not_finite(V, pad, dtype):
    """A row of weight 0 has term 0 and a zero gradient, whatever its logits and its list hold."""
    T, K = 8, 10
    g = _gen(V + 4)
    zt = torch.randn(T, V, generator=g, device=DEV)
    ids, values, tail = _lists(zt, K, 1.0)
    other = [int(next(j for j in range(V) if j not in set(i))) for i in ids.tolist()]
    z = zt + torch.randn(T, V, generator=g, device=DEV)
    z[0, other[0]] = math.nan
    z[1, other[1]] = INF
    z[2, ids[2, 0]] = math.nan
    z[3, ids[3, 0]] = INF
    z[4] = -INF
    values[5, 3] = math.nan
    tail[6] = math.nan
    weight = torch.zeros(T, device=DEV)
    weight[7] = 1.0
    logits = _store(z, dtype, pad=pad)
    for kind in (cis.KL_FORWARD, cis.KL_REVERSE):
        out = cis.distill_bwd(logits, ids, values, tail, weight, kind=kind)
        assert not out["terms"][:7].any() and not out["dlogits"][:7].any()
        assert out["dlogits"][7].any() and float(out["loss"]) == float(out["terms"][7]) > 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 1024])
def test_reverse_with_every_token_listed(V, dtype):
    """Nothing is left outside the lists, of the teacher or of the student."""
    T = 7
    g = _gen(V + 5)
    zt = torch.randn(T, V, generator=g, device=DEV) * 2
    z = zt + torch.randn(T, V, generator=g, device=DEV)
    for temp in (1.0, 0.25):
        ids, values, tail = _lists(zt, V, temp)
        assert (tail == -INF).all()
        for reverse in (True, False):
            _both(_store(z, dtype, pad=1), ids, values, tail, reverse=reverse, temp=temp)
        _both(_store(z, dtype), ids, values, None, temp=temp)


# ------------------------------------------------------------------------------------------
# Every width of the fused pass, and the pass in parts beside it
# ------------------------------------------------------------------------------------------

def _mixed(T, V, K, dtype, seed, *, pad=0, extra=0):
    """Rows of which some are masked, some have weight 0, an empty list, empty entries, ids out of range or
    repeated ids, in no order; lists as the first K columns of longer ones."""
    g = _gen(seed)

    def some(share):
        return torch.rand(T, generator=g, device=DEV) < share

    zt = torch.randn(T, V, generator=g, device=DEV) * 2.5
    ids, values, tail = _lists(zt, K, 1.0, seed=seed)
    logits = _store(zt.add_(torch.randn(T, V, generator=g, device=DEV)), dtype, pad=pad, fill=3.0)
    holes = some(0.3)[:, None] & (torch.rand(ids.shape, generator=g, device=DEV) < 0.3)
    ids = torch.where(holes, -1, ids)
    ids[some(0.1)] = -1
    ids[some(0.05), 1] = V
    ids[some(0.05), 2] = -7
    twice = some(0.1)
    ids[twice, 3] = ids[twice, 0]
    weight = torch.rand(T, generator=g, device=DEV) + 0.1
    weight[some(0.1)] = 0.0
    mask = (~some(0.2)).to(torch.uint8)
    wide_i = torch.zeros(T, K + extra, dtype=torch.int32, device=DEV)
    wide_v = torch.zeros(T, K + extra, device=DEV)
    wide_i[:, :K], wide_v[:, :K] = ids, values
    return logits, wide_i[:, :K], wide_v[:, :K], tail, weight, mask


def _check_mixed(case, kind, rows, scale=0.5):
    """A call with the gradient beside its logits and in their place, and the loss alone: the chosen rows
    against the formulas, and what all rows have to be."""
    logits, ids, values, tail, weight, mask = case
    T, V = logits.shape
    kw = dict(kind=kind, scale=scale)
    out = cis.distill_bwd(*case, **kw)
    ref = dict(reverse=kind == cis.KL_REVERSE, scale=scale, weight=weight, mask=mask, rows=rows,
               stats=False)
    _check(logits, ids, values, tail, out, **ref)
    fwd = cis.distill_fwd(*case, **kw)
    _check(logits, ids, values, tail, fwd, **ref)
    # what counts
    on = mask != 0
    order = torch.where((ids < 0) | (ids >= V), -1 - torch.arange(ids.shape[1], device=DEV),
                        ids).sort(1).values
    bad = (((ids != -1) & ((ids < 0) | (ids >= V))).any(1) | (order[:, 1:] == order[:, :-1]).any(1))
    valid = on & ~bad & (ids >= 0).any(1)
    live = valid & (weight != 0)
    for o in (out, fwd):
        assert not o["terms"][~live].any() and (o["terms"][live] != 0).all()
        total = o["terms"].double()
        assert abs(float(o["loss"]) - float(total.sum())) <= 64 * U * float(total.abs().sum())
        st = cis.read_stats(o["workspace"])
        assert (st["n_valid"], st["n_bad_id"], st["n_nonfinite"]) == (int(valid.sum()),
                                                                      int((on & bad).sum()), 0)
    assert not out["dlogits"][~live].any() and out["dlogits"][live].any(1).all()
    # in place, whatever the rows hold besides; the columns past V stay
    base = logits._base if logits._base is not None else logits
    place = base.clone()[:T, :V]
    res = cis.distill_bwd(place, ids, values, tail, weight, mask, dlogits=place, **kw)
    assert torch.equal(place, out["dlogits"]) and torch.equal(res["terms"], out["terms"])
    if base.shape[1] > V:
        assert (place._base[:, V:] == 3.0).all()


def _some_rows(T, n, seed=0):
    rows = torch.randperm(T, generator=torch.Generator().manual_seed(seed))[:n].tolist()
    return sorted(set(rows) | {0, T - 1})


# Vectors of 16 bytes per row, one in each step of the fused pass (and beyond what it holds), and the
# largest number of rows that go in parts there.
STEPS = [(37, 0), (300, 0), (620, 448), (1100, 448), (2001, 0), (3000, 320), (4050, 320),
         (5101, 320), (6600, 144), (8650, 144), (12200, 112), (15300, 112), (19456, 112),
         (19457, 112), (26000, 112)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [40, 300])
@pytest.mark.parametrize("nvec,most", STEPS)
def test_every_step_and_the_rows_beside_it(nvec, most, K, dtype):
    V = nvec * (16 // dtype.itemsize) - nvec % 3
    K = min(K, V // 2)
    for T in ([20] if most == 0 else [most, most + 1]):
        case = _mixed(T, V, K, dtype, nvec + T, pad=nvec % 2, extra=nvec % 5)
        for kind in (cis.KL_FORWARD, cis.KL_REVERSE):
            _check_mixed(case, kind, _some_rows(T, 10, nvec))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nvec,T", [(90, 9000), (1000, 9000), (2000, 2600), (6000, 1300),
                                    (13000, 700), (20500, 530)])
def test_rows_of_several_rounds(nvec, T, dtype):
    """More rows than workgroups at once: what one row leaves in shared memory is gone for the next."""
    V = nvec * (16 // dtype.itemsize) - 1
    case = _mixed(T, V, 50, dtype, nvec)
    _check_mixed(case, cis.KL_FORWARD, _some_rows(T, 30, nvec))
    _check_mixed(case, cis.KL_REVERSE, _some_rows(T, 30, nvec + 1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,T", [(2500, 30), (70000, 150), (300000, 113)])
def test_lists_that_share_places_of_the_table(V, T, dtype):
    """Ids that fill whole vectors, run along the row, or fall into one place of the fused pass's table,
    with rows enough for that pass."""
    g = _gen(V)
    zt = torch.randn(T, V, generator=g, device=DEV) * 2
    logits = _store(zt + torch.randn(T, V, generator=g, device=DEV), dtype, pad=1)
    rows = [0, 1, 2, T // 2, T - 1]
    for stride, K in ((1, 1024), (8, 280), (4, 37), (16384, 9), (32768, 9), (293, 230), (65536, 4)):
        K = min(K, (V - 1) // stride + 1)
        ids = (torch.arange(K, device=DEV) * stride).to(torch.int32).expand(T, K).contiguous()
        ids[1::2] = V - 1 - ids[1::2]
        values = zt.gather(1, ids.long())
        tail = torch.logsumexp(zt.scatter(1, ids.long(), -INF), dim=1)
        for reverse in (False, True):
            out = cis.distill_bwd(logits, ids, values, tail,
                                  kind=cis.KL_REVERSE if reverse else cis.KL_FORWARD)
            _check(logits, ids, values, tail, out, reverse=reverse, rows=rows, stats=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [1, 40, 64, 200, 1000])
@pytest.mark.parametrize("T,V", [(513, 2000), (900, 33001), (2000, 5000)])
def test_loss_alone_over_many_rows(T, V, K, dtype):
    """The loss without its gradient by one wave per row, on either side of 512 rows."""
    g = _gen(T + K)
    case = list(_mixed(T, V, max(K, 8), dtype, T, pad=1))
    case[1], case[2] = case[1][:, :K].contiguous(), case[2][:, :K].contiguous()
    case[3] = torch.randn(T, generator=g, device=DEV)
    for kind in (cis.KL_FORWARD, cis.KL_REVERSE):
        rows = _some_rows(T, 25, K)
        out = cis.distill_fwd(*case, kind=kind)
        ref = dict(reverse=kind == cis.KL_REVERSE, weight=case[4], mask=case[5])
        _check(*case[:4], out, rows=rows, stats=False, **ref)
        few = [x[:500] for x in case]
        _check(*few[:4], cis.distill_fwd(*few, kind=kind), rows=[r for r in rows if r < 500],
               stats=False, reverse=ref["reverse"], weight=few[4], mask=few[5])


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, 2100), (torch.float32, 1050)])
def test_loss_alone_of_logits_beyond_the_caches(dtype, T):
    """More than 192 MiB of logits, which the scan does not keep for a later read."""
    case = _mixed(T, 50003, 40, dtype, 3)
    assert case[0].stride(0) * T * dtype.itemsize > 192 << 20
    rows = _some_rows(T, 25)
    _check(*case[:4], cis.distill_fwd(*case), rows=rows, stats=False, weight=case[4], mask=case[5])


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_rows_than_a_launch_takes(dtype):
    """2^20 rows are one launch of a wave each; the fused pass takes any number in rounds."""
    T, V = (1 << 20) + 77, 24
    case = _mixed(T, V, 6, dtype, 9)
    rows = [0, 5, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T - 1]
    for kind in (cis.KL_FORWARD, cis.KL_REVERSE):
        _check_mixed(case, kind, rows)
