"""Performance cases of the token operators around the loss: sampling from logits, a teacher's
largest logits, and the distillation loss against such a list.

  sample   one token per row of logits [T, V], drawn with a given random number from the softmax at
           a temperature, cut by top-k, top-p and min-p; with the log-probability that the loss
           takes as logp_infer.
  top      the K largest logits of each row in order, and the log-sum-exp of all the others: what
           a teacher leaves behind for each token.
  distill  KL between a teacher given by such a list and the student's logits [T, V], forward
           only or with the gradient.

``run`` computes them in plain torch, in 32 bits (draws and ranks in integers, which are exact), or
through the package's calls where ``own`` is set. Logits follow the rollouts of ``workloads``: Zipf
ranks as the bias of the token ids plus normal noise, and confident rows with one peaked logit.
"""

from __future__ import annotations

import math

import torch

own = False

LOG2E = 1.4426950408889634
ONE = 1 << 28           # a draw's weight of a row's largest logit
INF = math.inf


def _sample(name, T, V, **kw):
    c = dict(name=name, kind="sample", T=T, V=V, dtype="bfloat16", temperature=1.0, top_k=0,
             top_p=1.0, min_p=0.0, per_row=False, banned=0.0, peak=0.5, mask=1.0)
    c.update(kw)
    return c


def _top(name, T, V, K, **kw):
    c = dict(name=name, kind="top", T=T, V=V, K=K, dtype="bfloat16", temperature=1.0, banned=0.0,
             peak=0.5, mask=1.0)
    c.update(kw)
    return c


def _distill(name, T, V, K, **kw):
    c = dict(name=name, kind="distill", T=T, V=V, K=K, dtype="bfloat16", temperature=1.0,
             reverse=False, tail=True, bwd=True, weighted=False, peak=0.5, mask=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # One request that decodes alone: every microsecond is a token's latency.
        _sample("sample one token", 1, 151936, temperature=0.7, top_k=50, top_p=0.9),
        # A serving batch whose requests each have their own settings, in float32, an odd
        # vocabulary, some of them held to a grammar.
        _sample("sample mixed requests", 64, 50257, dtype="float32", per_row=True, banned=0.5),
        # A rollout batch: temperature 1, nothing cut, the log-probabilities recorded.
        _sample("sample rollout", 512, 151936),
        # Nucleus sampling over a wide vocabulary: how much is kept differs from row to row.
        _sample("sample nucleus wide", 256, 262144, top_p=0.95, temperature=0.8),
        # A teacher's first choices along one short response.
        _top("top 8 short response", 96, 151936, 8),
        # A teacher's dump over 6000 positions, the 256 largest logits of each.
        _top("top 256 dump", 6000, 151936, 256),
        # float32 logits, an odd vocabulary and an odd list, at the distillation temperature; a
        # tenth of the rows is prompt.
        _top("top 20 ragged f32", 1777, 50257, 20, dtype="float32", temperature=2.0, mask=0.9,
             banned=0.1),
        # A debugging-sized batch in float32: launches count.
        _distill("distill tiny f32", 256, 1024, 16, dtype="float32"),
        # The validation loss of a small batch: no gradient.
        _distill("distill forward", 8192, 32768, 64, bwd=False),
        # The step of an on-policy distillation run on a packed rollout batch.
        _distill("distill rollout", 16384, 151936, 64),
        # Reverse KL at a temperature, weighted tokens, an odd vocabulary and row count.
        _distill("distill reverse ragged", 3001, 50257, 100, reverse=True, temperature=2.0,
                 weighted=True, mask=0.9),
        # One short response against long lists that were stored without their tail.
        _distill("distill short response", 96, 151936, 256, tail=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "top", "distill"])
    f32 = rng.random() < 0.25
    dt = "float32" if f32 else "bfloat16"
    rows, cells = {"sample": (1, 512 * 151936), "top": (16, 6000 * 151936),
                   "distill": (16, 16384 * 151936)}[kind]
    while True:
        T = _log_int(rng, rows, cells // 151936)
        V = _log_int(rng, 1024, 262144)
        if T * V * (2 if f32 else 1) <= cells:
            break
    peak = rng.choice([0.0, 0.5, 0.8])
    if kind == "sample":
        return dict(kind=kind, T=T, V=V, dtype=dt, temperature=rng.choice([0.0, 0.6, 1.0, 1.0, 1.3]),
                    top_k=rng.choice([0, 0, 1, 20, 50, 500, V // 2]),
                    top_p=rng.choice([1.0, 1.0, 0.8, 0.95, 0.999]),
                    min_p=rng.choice([0.0, 0.0, 0.05, 0.3]), per_row=rng.random() < 0.3,
                    banned=rng.choice([0.0, 0.0, 0.5]), peak=peak, mask=rng.choice([1.0, 0.9]))
    K = _log_int(rng, 1, 512)
    if kind == "top":
        return dict(kind=kind, T=T, V=V, K=K, dtype=dt, temperature=rng.choice([1.0, 1.0, 0.7, 2.0]),
                    banned=rng.choice([0.0, 0.0, 0.1]), peak=peak, mask=rng.choice([1.0, 0.75]))
    reverse = rng.random() < 0.4
    return dict(kind=kind, T=T, V=V, K=K, dtype=dt, temperature=rng.choice([1.0, 1.0, 2.0, 4.0]),
                reverse=reverse, tail=reverse or rng.random() < 0.6, bwd=rng.random() < 0.75,
                weighted=rng.random() < 0.5, peak=peak, mask=rng.choice([1.0, 0.9, 0.6]))


# ------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------

def _rows(n, V, peak, g):
    """Logits of n rows in float32."""
    z = torch.randn(n, V, generator=g, device="cuda").mul_(2.0)
    z -= 1.1 * torch.log(torch.arange(1, V + 1, device="cuda", dtype=torch.float32))
    at = torch.arange(n, device="cuda")[torch.rand(n, generator=g, device="cuda") < peak]
    col = torch.randint(0, V, (n,), generator=g, device="cuda")[at]
    z[at, col] = z.amax(dim=1)[at] + 4.69
    return z


def _row_steps(T, V):
    step = max(1, min(T, (1 << 27) // V))
    return [slice(r, min(T, r + step)) for r in range(0, T, step)]


def _logits(case):
    """[T, V] with rows of whole 16-byte vectors."""
    dt = getattr(torch, case["dtype"])
    epv = 16 // dt.itemsize
    ld = (case["V"] + epv - 1) // epv * epv
    return torch.zeros(case["T"], ld, dtype=dt, device="cuda")[:, :case["V"]]


def _choose(values, T, g, dtype):
    v = torch.tensor(values, dtype=dtype, device="cuda")
    return v[torch.randint(0, len(values), (T,), generator=g, device="cuda")]


def _prepare(case, seed):
    T, V = case["T"], case["V"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case, logits=_logits(case))
    mask = (torch.rand(T, generator=g, device="cuda") < case["mask"]).to(torch.uint8)
    s["mask"] = None if case["mask"] == 1.0 else mask
    if case["kind"] == "distill":
        K, tau = min(case["K"], V), case["temperature"]
        s["ids"] = torch.empty(T, K, dtype=torch.int32, device="cuda")
        s["values"] = torch.empty(T, K, device="cuda")
        s["tail"] = torch.empty(T, device="cuda")
        for r in _row_steps(T, V):
            z = _rows(r.stop - r.start, V, case["peak"], g)
            v, i = z.topk(K, dim=1)
            s["values"][r], s["ids"][r] = v, i
            s["tail"][r] = torch.logsumexp(z.scatter(1, i, -INF) / tau, dim=1)
            # the student is some way from its teacher
            s["logits"][r] = z.add_(torch.randn(z.shape, generator=g, device="cuda"))
            del z
        if not case["tail"]:
            s["tail"] = None
        s["weight"] = torch.rand(T, generator=g, device="cuda") * 2 if case["weighted"] else None
        s["scale"] = 1.0 / max(int(mask.sum()), 1)
        return s
    for r in _row_steps(T, V):
        z = _rows(r.stop - r.start, V, case["peak"], g)
        if case["banned"]:  # tokens that a grammar rules out, in that share of the rows
            some = torch.rand(z.shape[0], 1, generator=g, device="cuda") < case["banned"]
            z.masked_fill_((torch.rand(z.shape, generator=g, device="cuda") < 0.7) & some, -INF)
        s["logits"][r] = z
        del z
    if case["kind"] == "sample":
        s["u"] = torch.rand(T, generator=g, device="cuda")
        s["temperature"], s["top_k"] = case["temperature"], min(case["top_k"], V)
        s["top_p"], s["min_p"] = case["top_p"], case["min_p"]
        if case["per_row"]:
            f = torch.float32
            s["temperature"] = _choose([0.0, 0.6, 0.8, 1.0, 1.3], T, g, f)
            s["top_k"] = _choose([0, 1, 20, 50], T, g, torch.int32)
            s["top_p"] = _choose([0.9, 0.95, 1.0], T, g, f)
            s["min_p"] = _choose([0.0, 0.0, 0.05], T, g, f)
    return s


def prepare(case, seed):
    s = _prepare(case, seed)
    if own:  # the handle that a decoding or training loop keeps over its buffers
        import paper_2609_32444_amd as cis
        if case["kind"] == "sample":
            s["call"] = cis.SampleCall(s["logits"], s["u"], s["mask"], temperature=s["temperature"],
                                       top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        elif case["kind"] == "top":
            s["call"] = cis.TopLogitsCall(s["logits"], case["K"], s["mask"],
                                          temperature=case["temperature"])
        else:
            s["call"] = cis.DistillCall(
                s["logits"], s["ids"], s["values"], s["tail"], s["weight"], s["mask"],
                kind=cis.KL_REVERSE if case["reverse"] else cis.KL_FORWARD,
                temperature=case["temperature"], scale=s["scale"], bwd=case["bwd"])
    return s


# ------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------

NAMES = {"sample": ("ids", "logp", "logp_kept"), "top": ("ids", "values", "tail"),
         "distill": ("terms", "loss", "dlogits")}


def run(state):
    case = state["case"]
    if own:
        out = state["call"].run()
        return {k: out[k] for k in NAMES[case["kind"]] if k in out}
    return {"sample": _plain_sample, "top": _plain_top, "distill": _plain_distill}[case["kind"]](
        case, state)


def _on(state):
    """[T] truth values of the rows that count."""
    if state["mask"] is None:
        return torch.ones(state["logits"].shape[0], dtype=torch.bool, device="cuda")
    return state["mask"] != 0


def _per_row(x, T, dtype):
    return torch.as_tensor(x, dtype=dtype, device="cuda").expand(T)[:, None]


def _plain_sample(case, s):
    """Weights are whole multiples of 2^-28 of the largest one, so their sums are exact in any
    order: q_j = floor(2^28 2^((z_j - max) log2(e) / temperature))."""
    T, V = s["logits"].shape
    z = s["logits"].float()
    on = _on(s)
    tau = _per_row(s["temperature"], T, torch.float32)
    k = _per_row(s["top_k"], T, torch.int64)
    top_p = _per_row(s["top_p"], T, torch.float32).double()
    min_p = _per_row(s["min_p"], T, torch.float32).double()
    x = z - z.amax(dim=1, keepdim=True)
    c = torch.div(torch.full_like(tau, LOG2E), torch.where(tau == 0, 1.0, tau))
    q = (torch.exp2(x * c) * ONE).to(torch.int64)
    # in order of the logits, the lowest id first among equals, every cut keeps a first part
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    cum = q.gather(1, order).cumsum(1)
    n = torch.where(k == 0, V, k)
    enough = cum.double() >= top_p * cum.gather(1, n - 1).double()
    n_p = torch.where(top_p >= 1, V, 1 + (~enough).sum(1, keepdim=True))
    n_m = (q.double() >= min_p * ONE).sum(1, keepdim=True)
    n = torch.where(tau == 0, 1, torch.minimum(torch.minimum(n, n_p), n_m))
    kept = torch.zeros_like(q, dtype=torch.bool).scatter_(
        1, order, torch.arange(V, device="cuda") < n)
    # the draw, in order of the ids
    cdf = torch.where(kept, q, 0).cumsum(1)
    total = cdf[:, -1:]
    at = (s["u"][:, None].double() * total.double()).long()
    ids = (cdf <= torch.minimum(at, total - 1)).sum(1, keepdim=True)
    logp = x.gather(1, ids) - torch.log(torch.exp(x).sum(1, keepdim=True))
    logp_kept = torch.log(q.gather(1, ids).double() / total.double()).float()
    off = ~on[:, None]
    return {"ids": ids.masked_fill(off, -1)[:, 0], "logp": logp.masked_fill(off, 0.0)[:, 0],
            "logp_kept": logp_kept.masked_fill(off, 0.0)[:, 0]}


def _plain_top(case, s):
    T, V = s["logits"].shape
    K = case["K"]
    z = torch.where(_on(s)[:, None], s["logits"].float(), -INF) + 0.0
    # whole numbers in the order of (logit, lowest id first)
    bits = z.view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32)
    key += V - 1 - torch.arange(V, device="cuda")
    best = key.topk(min(K, V), dim=1).values
    ids = V - 1 - (best & 0xFFFFFFFF)
    values = z.gather(1, ids)
    x = z.scatter_(1, ids, -INF) / case["temperature"]
    top = x.amax(dim=1).clamp(min=-3e38)
    tail = top + torch.log(torch.exp(x - top[:, None]).sum(1))
    ids = ids.masked_fill(values == -INF, -1).to(torch.int32)
    pad = (0, K - ids.shape[1])
    return {"ids": torch.nn.functional.pad(ids, pad, value=-1),
            "values": torch.nn.functional.pad(values, pad, value=-INF), "tail": tail}


def _log_shares(x, rest):
    """log of each share exp(x_k) / total and rest / total, total = sum_k exp(x_k) + rest."""
    e = torch.exp(x)
    total = e.sum(1, keepdim=True) + rest
    near_one = torch.log1p(-e.sum(1, keepdim=True) / total)
    return x - torch.log(total), torch.where(rest > 0.5 * total, near_one,
                                             torch.log(rest / total))


def _plain_distill(case, s):
    T, V = s["logits"].shape
    tau, ids = case["temperature"], s["ids"].long()
    on = _on(s)
    a = s["scale"] * (torch.ones(T, device="cuda") if s["weight"] is None else s["weight"])
    a = torch.where(on, a, 0.0)
    # the teacher: log q of its list and of everything else
    t = s["values"] / tau
    tail = torch.full_like(t[:, :1], -INF) if s["tail"] is None else s["tail"][:, None]
    top = torch.maximum(t.amax(dim=1, keepdim=True), tail)
    lq, lq_rest = _log_shares(t - top, torch.exp(tail - top))
    # the student: log p of the same, the rest summed by itself
    x = s["logits"].float()
    x = (x - x.amax(dim=1, keepdim=True)) / tau
    e = torch.exp(x)
    xk = x.gather(1, ids)
    rest = e.scatter(1, ids, 0.0).sum(1, keepdim=True)
    total = torch.exp(xk).sum(1, keepdim=True) + rest
    lp, lp_rest = _log_shares(xk, rest)
    # sum of a log(a/b) as the sum of a log(a/b) - a + b, whose terms do not cancel
    d, d_rest = lp - lq, lp_rest - lq_rest
    p, p_rest, q, q_rest = (torch.exp(v) for v in (lp, lp_rest, lq, lq_rest))
    if case["reverse"]:
        kl = (p * (torch.expm1(-d) + d)).sum(1, keepdim=True)
        kl += torch.where(p_rest > 0, p_rest * (torch.expm1(-d_rest) + d_rest), q_rest)
        on_list, on_rest = p * (d - kl), d_rest - kl
    else:
        kl = (q * (torch.expm1(d) - d)).sum(1, keepdim=True)
        kl += torch.where(q_rest > 0, q_rest * (torch.expm1(d_rest) - d_rest), p_rest)
        on_list, on_rest = p - q, -torch.expm1(-d_rest)
    terms = a * kl[:, 0]
    out = {"terms": terms, "loss": terms.sum()[None]}
    if case["bwd"]:
        grad = (e / total * on_rest).scatter_(1, ids, on_list)
        out["dlogits"] = (grad * (a / tau)[:, None]).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------

def work(case):
    T, V = case["T"], case["V"]
    es = 4 if case["dtype"] == "float32" else 2
    n = T * case["mask"] * V * es + (T if case["mask"] < 1.0 else 0)
    if case["kind"] == "sample":
        n += T * (4 + 8 + 4 + 4 + (16 if case["per_row"] else 0))
        return {"bytes": int(n), "flops": 3 * T * V}
    if case["kind"] == "top":
        return {"bytes": int(n + T * (8 * case["K"] + 4)), "flops": 3 * T * V}
    n += T * (8 * min(case["K"], V) + (4 if case["tail"] else 0) + (4 if case["weighted"] else 0) + 4)
    n += T * V * es if case["bwd"] else 0
    return {"bytes": int(n), "flops": (6 if case["bwd"] else 3) * T * V}


# ------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions, a block of rows at a time
# ------------------------------------------------------------------------------------------

def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _exact_sample(s, z, r):
    def of(name):
        x = s[name]
        return x[r].double() if isinstance(x, torch.Tensor) else torch.full(
            (z.shape[0],), _f32(x), dtype=torch.float64, device="cuda")
    tau, k, top_p, min_p, u = (of(n) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    n, V = z.shape
    v, order = torch.sort(z, dim=1, descending=True, stable=True)
    warm = tau > 0
    # a weight's exponent is a float32 product by definition
    c = torch.div(torch.full_like(tau, LOG2E), torch.where(warm, tau, 1.0)).float()
    e = ((v - v[:, :1]).float() * c[:, None]).double()
    q = torch.floor(torch.exp2(e) * ONE)
    rank = torch.arange(V, device="cuda", dtype=torch.float64)[None, :]
    keep = (rank < torch.where(k > 0, k, V)[:, None]) & (q >= (min_p * ONE)[:, None])
    in_k = torch.where(rank < torch.where(k > 0, k, V)[:, None], q, 0.0)
    before = in_k.cumsum(1) - in_k
    keep &= (before < (top_p * in_k.sum(1))[:, None]) | (top_p >= 1.0)[:, None]
    keep = torch.where(warm[:, None], keep, rank < 1)
    kept = torch.zeros_like(q).scatter_(1, order, torch.where(keep, q, 0.0))
    cdf = kept.cumsum(1)
    at = torch.floor(u * cdf[:, -1])
    ids = torch.searchsorted(cdf, at[:, None], right=True).clamp(max=V - 1)
    logp = torch.log_softmax(z, dim=1).gather(1, ids)[:, 0]
    return {"ids": None, "logp": logp,
            "logp_kept": torch.log(kept.gather(1, ids)[:, 0] / cdf[:, -1])}


def _exact_top(case, z):
    K, V = case["K"], z.shape[1]
    v, order = torch.sort(z, dim=1, descending=True, stable=True)
    n = min(K, V)
    values = torch.full((z.shape[0], K), -INF, dtype=torch.float64, device="cuda")
    values[:, :n] = v[:, :n]
    rest = v[:, n:] / case["temperature"]
    tail = torch.logsumexp(rest, dim=1) if V > n else torch.full_like(values[:, 0], -INF)
    return {"ids": None, "values": values, "tail": tail}


def _exact_distill(case, s, z, r):
    tau, ids = case["temperature"], s["ids"][r].long()
    t = s["values"][r].double() / tau
    if s["tail"] is not None:
        t = torch.cat([t, s["tail"][r].double()[:, None]], dim=1)
    q = torch.softmax(t, dim=1)
    if s["tail"] is None:
        q = torch.cat([q, torch.zeros_like(q[:, :1])], dim=1)
    p_all = torch.softmax(z / tau, dim=1)
    p = torch.cat([p_all.gather(1, ids), p_all.scatter(1, ids, 0.0).sum(1, keepdim=True)], dim=1)
    if case["reverse"]:
        ratio = torch.log(p) - torch.log(q)
        kl = (p * ratio).sum(1, keepdim=True)
        per = ratio - kl            # of p_j, in each class
    else:
        kl = torch.xlogy(q, q) - torch.xlogy(q, p)
        kl = kl.sum(1, keepdim=True)
        per = 1.0 - q / p
    scale = s["scale"] if s["weight"] is None else s["scale"] * s["weight"][r].double()
    a = torch.where(_on(s)[r], scale, 0.0)[:, None]
    out = {"terms": (a * kl)[:, 0]}
    if case["bwd"]:
        on_list = p_all.gather(1, ids) * per[:, :-1]
        out["dlogits"] = (p_all * per[:, -1:]).scatter_(1, ids, on_list) * (a / tau)
    return out


def exact(case, seed):
    s = _prepare(case, seed)
    T, V = s["logits"].shape
    step = max(1, min(T, (1 << 27) // V))
    parts = []
    for r0 in range(0, T, step):
        r = slice(r0, min(T, r0 + step))
        z = s["logits"][r].double()
        if case["kind"] == "distill":
            parts.append(_exact_distill(case, s, z, r))
            continue
        off = ~_on(s)[r]
        if case["kind"] == "sample":
            out = _exact_sample(s, z, r)
            fill = 0.0
        else:
            out = _exact_top(case, z)
            fill = -INF
        for k, v in out.items():
            if v is not None:
                v[off] = fill
        parts.append(out)
    out = {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
    if case["kind"] == "distill":
        out["loss"] = out["terms"].sum()[None]
    return out
