"""Performance cases of the operators at the two ends of the LM head: the RMS norm that makes the
hidden states in front of it, and the verification of drafted tokens on the logits behind it.

  norm      y = s rstd w of rows s = x + residual, rstd = 1 / sqrt(mean(s^2) + eps), in 16 or 32 bits,
            or in e4m3 with a scale for every row or for every block of a row.
  grad      its backward pass: the gradient of s (with what comes along the residual added) and of
            the weight.
  verify    sequences of drafted tokens against the target's logits, from given random numbers: how
            many are accepted, the token drawn at the first rejection or after the last draft, and
            the log-probabilities that the loss takes as logp_infer.

``run`` computes them in plain torch, in 32 bits (a draw's weights and sums in integers, which are
exact, and what is compared with them in 64), or through the package's calls where ``own`` is set.
"""

from __future__ import annotations

import math

import torch

own = False

LOG2E = 1.4426950408889634
ONE = 1 << 28           # a draw's weight of a row's largest logit
INF = math.inf
E4M3_MAX = 448.0
E4M3_LEAST = 2.0 ** -126   # the least scale of e4m3 values


def _norm(name, T, H, **kw):
    c = dict(name=name, kind="norm", T=T, H=H, x="bfloat16", stream="bfloat16", w="bfloat16",
             out="bfloat16", group=0, residual=True, eps=1e-6)
    c.update(kw)
    return c


def _grad(name, T, H, **kw):
    c = dict(name=name, kind="grad", T=T, H=H, dy="bfloat16", stream="bfloat16", w="bfloat16",
             dx="bfloat16", residual=True, eps=1e-6)
    c.update(kw)
    return c


def _verify(name, B, K, V, **kw):
    c = dict(name=name, kind="verify", B=B, K=K, V=V, dtype="bfloat16", temperature=1.0, top_k=0,
             top_p=1.0, min_p=0.0, per_seq=False, ragged=False, draft=True, peak=0.5)
    c.update(kw)
    return c


def listed():
    return [
        # A layer's norm of one request that decodes alone: latency.
        _norm("norm one token", 1, 2048),
        # The norm in front of the LM head over a packed batch, at the head's width.
        _norm("norm packed batch", 16384, 2048),
        # A wide model's residual stream in float32 beside bf16 layers, the next layer's input in
        # 8 bits with a scale per token.
        _norm("norm 8 bits per token", 8192, 8192, stream="float32", out="float8_e4m3fn"),
        # A serving batch whose next product takes 8 bits with a scale for each 128 columns.
        _norm("norm 8 bits blocks", 300, 5120, out="float8_e4m3fn", group=128),
        # The norm of each head's queries: many short rows, no residual.
        _norm("norm heads", 16384 * 16, 128, residual=False, w="float32"),
        # The backward pass behind the LM head: its dL/dh is float32.
        _grad("norm grad head", 16384, 2048, dy="float32", residual=False),
        # A layer's backward pass, the residual stream's own gradient added; odd rows and width.
        _grad("norm grad ragged", 3001, 4100, w="float32"),
        # One request with four drafted tokens: latency.
        _verify("verify one request", 1, 4, 151936),
        # A rollout batch at temperature 1, nothing cut, four drafted tokens each.
        _verify("verify rollout", 64, 4, 151936),
        # Nucleus sampling with longer drafts.
        _verify("verify nucleus", 32, 7, 151936, temperature=0.8, top_p=0.95),
        # Requests with their own settings and as many drafts as each has, in float32, an odd
        # vocabulary.
        _verify("verify mixed requests", 48, 8, 50257, dtype="float32", per_seq=True, ragged=True),
        # Drafts copied from the prompt, which have no distribution of their own, decoded greedily.
        _verify("verify copied greedy", 128, 10, 151936, draft=False, ragged=True, temperature=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "grad", "verify", "verify"])
    if kind == "verify":
        f32 = rng.random() < 0.25
        while True:
            B, K, V = _log_int(rng, 1, 256), rng.randint(1, 12), _log_int(rng, 1024, 262144)
            draft = rng.random() < 0.75
            rows = B * (2 * K + 1 if draft else K + 1)
            if rows * V * (2 if f32 else 1) <= 576 * 151936:
                break
        return dict(kind=kind, B=B, K=K, V=V, dtype="float32" if f32 else "bfloat16",
                    temperature=rng.choice([0.0, 0.6, 1.0, 1.0, 1.3]),
                    top_k=rng.choice([0, 0, 1, 20, 50, 500]),
                    top_p=rng.choice([1.0, 1.0, 0.8, 0.95, 0.999]),
                    min_p=rng.choice([0.0, 0.0, 0.05, 0.3]), per_seq=rng.random() < 0.3,
                    ragged=rng.random() < 0.5, draft=draft, peak=rng.choice([0.0, 0.5, 0.8]))
    while True:
        T, H = _log_int(rng, 1, 262144), _log_int(rng, 32, 32768)
        if T * H <= 16384 * 2048:
            break
    w = rng.choice(["bfloat16", "float32"])
    x, stream = rng.choice([("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")])
    if kind == "norm":
        residual = rng.random() < 0.7
        out = rng.choice(["bfloat16", "bfloat16", "float32", "float8_e4m3fn", "float8_e4m3fn"])
        return dict(kind=kind, T=T, H=H, x=x, stream=stream if residual else x, w=w, out=out,
                    group=rng.choice([0, 32, 64, 128]) if out == "float8_e4m3fn" else 0,
                    residual=residual, eps=rng.choice([1e-6, 1e-5]))
    return dict(kind=kind, T=T, H=H, dy=rng.choice([x, "float32"]), stream=stream, w=w, dx=stream,
                residual=rng.random() < 0.7, eps=rng.choice([1e-6, 1e-5]))


# ------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------

def _matrix(T, n, dtype):
    """[T, n] with rows of whole 16-byte vectors."""
    dt = getattr(torch, dtype)
    epv = 16 // dt.itemsize
    ld = (n + epv - 1) // epv * epv
    return torch.zeros(T, ld, dtype=dt, device="cuda")[:, :n]


def _activations(T, H, dtype, g, size):
    """Rows of different sizes, a few columns far larger than the others."""
    m = _matrix(T, H, dtype)
    a = torch.randn(T, H, generator=g, device="cuda")
    a *= size * torch.exp(0.5 * torch.randn(T, 1, generator=g, device="cuda"))
    far = torch.randint(0, H, (max(1, H // 512),), generator=g, device="cuda")
    a[:, far] *= 20.0
    m.copy_(a)
    return m


def _weight(H, dtype, g):
    return (1.0 + 0.3 * torch.randn(H, generator=g, device="cuda")).to(getattr(torch, dtype))


def _rows(n, V, peak, g):
    """Logits of n rows in float32: Zipf ranks as the bias of the token ids plus normal noise, and
    confident rows with one peaked logit."""
    z = torch.randn(n, V, generator=g, device="cuda").mul_(2.0)
    z -= 1.1 * torch.log(torch.arange(1, V + 1, device="cuda", dtype=torch.float32))
    at = torch.arange(n, device="cuda")[torch.rand(n, generator=g, device="cuda") < peak]
    col = torch.randint(0, V, (n,), generator=g, device="cuda")[at]
    z[at, col] = z.amax(dim=1)[at] + 4.69
    return z


def _choose(values, n, g, dtype):
    v = torch.tensor(values, dtype=dtype, device="cuda")
    return v[torch.randint(0, len(values), (n,), generator=g, device="cuda")]


def _lengths(case):
    """Target rows of each sequence: one more than its drafts, which are 0 to K where ragged."""
    B, K = case["B"], case["K"]
    return [1 + b * (K + 1) // B if case["ragged"] else K + 1 for b in range(B)]


def _prepare_verify(case, s, g):
    B, K, V = case["B"], case["K"], case["V"]
    n = torch.tensor(_lengths(case), dtype=torch.int64, device="cuda")
    n = n[torch.randperm(B, generator=g, device="cuda")]
    s["offsets"] = torch.nn.functional.pad(n.cumsum(0), (1, 0))
    T = int(s["offsets"][-1])
    for name, values, dt in (("temperature", [0.0, 0.6, 0.8, 1.0, 1.3], torch.float32),
                             ("top_k", [0, 1, 20, 50], torch.int32),
                             ("top_p", [0.9, 0.95, 1.0], torch.float32),
                             ("min_p", [0.0, 0.0, 0.05], torch.float32)):
        s[name] = _choose(values, B, g, dt) if case["per_seq"] else case[name]
    if not case["per_seq"]:
        s["top_k"] = min(case["top_k"], V)
    s["u"] = torch.rand(T, generator=g, device="cuda")
    s["logits"] = _matrix(T, V, case["dtype"])
    z = _rows(T, V, case["peak"], g)
    s["logits"].copy_(z)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), n)
    last = s["offsets"][1:][seq] - 1
    rows = torch.arange(T, device="cuda")
    rows = rows[rows != last]       # of the drafts
    s["draft_logits"] = None
    if case["draft"]:
        # the draft model is some way from the target, and draws under the same settings
        z = z[rows]
        z += torch.randn(z.shape, generator=g, device="cuda").mul_(0.7)
        s["draft_logits"] = _matrix(rows.numel(), V, case["dtype"])
        s["draft_logits"].copy_(z)
        s["draft_ids"] = torch.zeros(rows.numel(), dtype=torch.int64, device="cuda")
        if rows.numel():
            q = _kept_weights(s, s["draft_logits"].float(), seq[rows])
            at = torch.rand(rows.numel(), generator=g, device="cuda")
            s["draft_ids"] = _drawn(q, at)[:, 0]
    else:
        likely = z[rows].argmax(dim=1) if rows.numel() else rows
        other = torch.randint(0, V, (rows.numel(),), generator=g, device="cuda")
        s["draft_ids"] = torch.where(
            torch.rand(rows.numel(), generator=g, device="cuda") < 0.7, likely, other)


def _prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=case)
    if case["kind"] == "verify":
        _prepare_verify(case, s, g)
        return s
    T, H = case["T"], case["H"]
    s["weight"] = _weight(H, case["w"], g)
    if case["kind"] == "norm":
        s["x"] = _activations(T, H, case["x"], g, 1.0)
        s["residual"] = _activations(T, H, case["stream"], g, 3.0) if case["residual"] else None
        return s
    s["x"] = _activations(T, H, case["stream"], g, 3.0)
    s["dy"] = _activations(T, H, case["dy"], g, 1e-3)
    s["dresidual"] = _activations(T, H, case["dx"], g, 1e-3) if case["residual"] else None
    return s


def prepare(case, seed):
    s = _prepare(case, seed)
    if own:  # the handle that a decoding or training loop keeps over its buffers
        import paper_2609_32444_amd as cis
        if case["kind"] == "norm":
            s["call"] = cis.RmsNormCall(s["x"], s["weight"], s["residual"], eps=case["eps"],
                                        out_dtype=getattr(torch, case["out"]), group=case["group"])
        elif case["kind"] == "grad":
            s["call"] = cis.RmsNormGradCall(s["dy"], s["x"], s["weight"], s["dresidual"],
                                            eps=case["eps"], dx_dtype=getattr(torch, case["dx"]))
        else:
            s["call"] = cis.VerifyCall(s["logits"], s["draft_ids"], s["u"], s["offsets"],
                                       s["draft_logits"], temperature=s["temperature"],
                                       top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return s


# ------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------

NAMES = {"norm": ("y", "scale", "residual"), "grad": ("dx", "dweight"),
         "verify": ("ids", "accepted", "logp", "logp_kept")}


def run(state):
    case = state["case"]
    if own:
        out = state["call"].run()
        return {k: out[k] for k in NAMES[case["kind"]] if k in out}
    return {"norm": _plain_norm, "grad": _plain_grad, "verify": _plain_verify}[case["kind"]](
        case, state)


def _plain_norm(case, s):
    x, out = s["x"].float(), {}
    if s["residual"] is not None:
        # the sum is kept in the stream's type, and what is kept is normalised
        out["residual"] = (x + s["residual"].float()).to(s["residual"].dtype)
        x = out["residual"].float()
    rstd = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + case["eps"])
    y = x * rstd * s["weight"].float()
    if case["out"] != "float8_e4m3fn":
        return out | {"y": y.to(getattr(torch, case["out"]))}
    T, H = y.shape
    n = case["group"] or H
    blocks = torch.nn.functional.pad(y, (0, -H % n)).view(T, -1, n)
    scale = (blocks.abs().amax(dim=2) / E4M3_MAX).clamp(min=E4M3_LEAST)
    q = (blocks / scale[:, :, None]).view(T, -1)[:, :H]
    return out | {"y": q.to(torch.float8_e4m3fn), "scale": scale if case["group"] else scale[:, 0]}


def _plain_grad(case, s):
    x, dy = s["x"].float(), s["dy"].float()
    rstd = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + case["eps"])
    xh = x * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - xh * (g * xh).mean(dim=1, keepdim=True))
    if s["dresidual"] is not None:
        dx = dx + s["dresidual"].float()
    return {"dx": dx.to(getattr(torch, case["dx"])), "dweight": (dy * xh).sum(dim=0)}


def _of_rows(s, name, seq, dtype):
    x = s[name]
    if isinstance(x, torch.Tensor):
        return x.to(dtype)[seq][:, None]
    return torch.full((seq.numel(), 1), x, dtype=torch.float32, device="cuda").to(dtype)


def _kept_weights(s, z, seq):
    """Weights of the rows' tokens under their sequences' settings, as whole multiples of 2^-28 of the
    largest one (their sums are exact in any order); 0 for tokens that a cut leaves out."""
    V = z.shape[1]
    tau = _of_rows(s, "temperature", seq, torch.float32)
    k = _of_rows(s, "top_k", seq, torch.int64)
    top_p = _of_rows(s, "top_p", seq, torch.float32).double()
    min_p = _of_rows(s, "min_p", seq, torch.float32).double()
    x = z - z.amax(dim=1, keepdim=True)
    c = torch.div(torch.full_like(tau, LOG2E), torch.where(tau == 0, 1.0, tau))
    q = (torch.exp2(x * c) * ONE).to(torch.int64)
    # in order of the logits, the lowest id first among equals, every cut keeps a first part
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    cum = q.gather(1, order).cumsum(1)
    n = torch.where((k == 0) | (k > V), V, k)
    enough = cum.double() >= top_p * cum.gather(1, n - 1).double()
    n_p = torch.where(top_p >= 1, V, 1 + (~enough).sum(1, keepdim=True))
    n_m = (q.double() >= min_p * ONE).sum(1, keepdim=True)
    n = torch.where(tau == 0, 1, torch.minimum(torch.minimum(n, n_p), n_m))
    kept = torch.zeros_like(q, dtype=torch.bool).scatter_(
        1, order, torch.arange(V, device="cuda") < n)
    return torch.where(kept, q, 0)


def _drawn(w, u):
    """[n, 1] the ids that the random numbers u fall on, by whole weights in order of the ids."""
    cdf = w.cumsum(1)
    total = cdf[:, -1:]
    at = (u[:, None].double() * total.double()).long()
    return (cdf <= torch.minimum(at, total - 1)).sum(1, keepdim=True)


def _plain_verify(case, s):
    offsets, u = s["offsets"], s["u"]
    T, B, D = u.numel(), offsets.numel() - 1, s["draft_ids"].numel()
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(offsets, t, right=True) - 1
    first, last = offsets[seq], offsets[seq + 1] - 1
    z = s["logits"].float()
    P = _kept_weights(s, z, seq)
    N = P.sum(1)
    drafted = t != last
    at = (t - seq).clamp(max=max(D - 1, 0))     # a row's place among the drafts
    ids = s["draft_ids"][at] if D else torch.zeros_like(t)
    Pd = P.gather(1, ids[:, None])[:, 0]
    if s["draft_logits"] is None:
        share = N.double()
    else:
        Q = _kept_weights(s, s["draft_logits"].float(), seq[drafted])
        rho = N[drafted].double() / Q.sum(1).double()
        share = torch.zeros(T, dtype=torch.float64, device="cuda")
        share[drafted] = Q.gather(1, ids[drafted][:, None])[:, 0].double() * rho
    accept = drafted & (u.double() * share < Pd.double())
    # drafts count up to the first that is turned down
    accepted = torch.full((B,), T, dtype=torch.int64, device="cuda").scatter_reduce_(
        0, seq, torch.where(accept, T, t - first), "amin")
    stop = offsets[:-1] + accepted              # each sequence's last token is drawn at this row
    R = P[stop]
    if s["draft_logits"] is None:
        R.scatter_(1, ids[stop][:, None],
                   torch.where(drafted[stop][:, None], 0, R.gather(1, ids[stop][:, None])))
    elif D:
        place = (drafted.cumsum(0) - 1).clamp(min=0)[stop]
        full = torch.zeros(T, dtype=torch.float64, device="cuda")
        full[drafted] = rho
        less = (Q[place].double() * full[stop][:, None]).long()
        R = torch.where(drafted[stop][:, None], (R - less).clamp(min=0), R)
    R = torch.where(R.sum(1, keepdim=True) > 0, R, P[stop])
    out = torch.where(t < stop[seq], ids, -1)
    out[stop] = _drawn(R, u[offsets[1:] - 1])[:, 0]
    there = out >= 0
    y = out.clamp(min=0)[:, None]
    x = z - z.amax(dim=1, keepdim=True)
    logp = (x.gather(1, y) - torch.log(torch.exp(x).sum(1, keepdim=True)))[:, 0]
    kept = torch.log(P.gather(1, y)[:, 0].double() / N.double()).float()
    return {"ids": out, "accepted": accepted.to(torch.int32),
            "logp": torch.where(there, logp, 0.0), "logp_kept": torch.where(there, kept, 0.0)}


# ------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------

def _size(dtype):
    return getattr(torch, dtype).itemsize


def work(case):
    if case["kind"] == "verify":
        B, V = case["B"], case["V"]
        drafts = sum(_lengths(case)) - B
        rows = B + drafts + (drafts if case["draft"] else 0)
        small = drafts * 8 + (B + drafts) * (4 + 8 + 4 + 4) + B * (8 + 4 + (16 if case["per_seq"] else 0))
        return {"bytes": int(rows * V * _size(case["dtype"]) + small), "flops": int(3 * rows * V)}
    T, H = case["T"], case["H"]
    n = H * _size(case["w"])
    if case["kind"] == "norm":
        n += T * H * (_size(case["x"]) + _size(case["out"]))
        n += 2 * T * H * _size(case["stream"]) if case["residual"] else 0
        if case["out"] == "float8_e4m3fn":
            n += 4 * T * (-(-H // case["group"]) if case["group"] else 1)
        return {"bytes": n, "flops": 5 * T * H}
    n += T * H * (_size(case["dy"]) + _size(case["stream"]) + _size(case["dx"])) + 4 * H
    n += T * H * _size(case["dx"]) if case["residual"] else 0
    return {"bytes": n, "flops": 10 * T * H}


# ------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# ------------------------------------------------------------------------------------------

def _exact_norm(case, s, r):
    x = s["x"][r].double()
    out = {}
    if s["residual"] is not None:
        total = x + s["residual"][r].double()
        out["residual"] = total
        x = total.to(s["residual"].dtype).double()
    y = x / torch.sqrt(x.square().sum(1, keepdim=True) / x.shape[1] + case["eps"])
    y = y * s["weight"].double()
    out["y"] = y
    if case["out"] == "float8_e4m3fn":
        n = case["group"] or y.shape[1]
        top = torch.stack([b.abs().amax(dim=1) for b in y.split(n, dim=1)], dim=1)
        scale = torch.clamp(top / E4M3_MAX, min=E4M3_LEAST)
        out["y"] = y / scale.repeat_interleave(n, dim=1)[:, :y.shape[1]]
        out["scale"] = scale if case["group"] else scale[:, 0]
    return out


def _exact_grad(case, s, r):
    x, dy, w = s["x"][r].double(), s["dy"][r].double(), s["weight"].double()
    H = x.shape[1]
    v = x.square().sum(1, keepdim=True) / H + case["eps"]
    dot = (dy * w * x).sum(1, keepdim=True)
    dx = dy * w / v.sqrt() - x * dot / (H * v * v.sqrt())
    if s["dresidual"] is not None:
        dx = dx + s["dresidual"][r].double()
    return {"dx": dx, "dweight": (dy * x / v.sqrt()).sum(0)}


def _exact_weights(z, tau, k, p, m):
    """One row's weights (whole numbers in float64), 0 for what is cut."""
    v, order = torch.sort(z, descending=True, stable=True)
    c = torch.tensor(LOG2E, dtype=torch.float32) / torch.tensor(tau, dtype=torch.float32)
    if not bool(torch.isfinite(c)):
        q = torch.zeros_like(z)
        q[order[0]] = ONE
        return q
    # a weight's exponent is a float32 product by definition
    w = torch.floor(torch.exp2(((v - v[0]).float() * c.to(z.device)).double()) * ONE)
    rank = torch.arange(z.numel(), device=z.device)
    in_k = torch.where(rank < k, w, 0.0) if 0 < k < z.numel() else w
    keep = (in_k > 0) & (w >= m * ONE)
    if p < 1.0:
        keep &= in_k.cumsum(0) - in_k < p * in_k.sum()
    return torch.zeros_like(z).scatter_(0, order, torch.where(keep, w, 0.0))


def _exact_verify(case, s):
    offsets, u = s["offsets"].tolist(), s["u"].double().tolist()
    drafts = s["draft_ids"].tolist()
    as_list = lambda n: (s[n].double().tolist() if isinstance(s[n], torch.Tensor)  # noqa: E731
                         else [float(torch.tensor(s[n], dtype=torch.float32))] * case["B"])
    sets = list(zip(*(as_list(n) for n in ("temperature", "top_k", "top_p", "min_p"))))
    logp = torch.zeros(offsets[-1], dtype=torch.float64, device="cuda")
    kept = torch.zeros_like(logp)
    for b in range(case["B"]):
        for t in range(offsets[b], offsets[b + 1]):
            z = s["logits"][t].double()
            P = _exact_weights(z, *sets[b])
            N, y = float(P.sum()), None
            W = P
            if t + 1 < offsets[b + 1]:
                d = drafts[t - b]
                if s["draft_logits"] is None:
                    share, W = N, P.clone()
                    W[d] = 0.0
                else:
                    Q = _exact_weights(s["draft_logits"][t - b].double(), *sets[b])
                    x = Q * (N / float(Q.sum()))
                    share, W = float(x[d]), torch.clamp(P - torch.floor(x), min=0.0)
                if u[t] * share < float(P[d]):
                    y = d
            stop = y is None
            if stop:
                W = W if float(W.sum()) > 0 else P
                cdf = W.cumsum(0)
                at = math.floor(u[offsets[b + 1] - 1] * float(cdf[-1]))
                y = int(torch.searchsorted(cdf, torch.tensor([float(at)], dtype=torch.float64,
                                                             device="cuda"), right=True))
            logp[t] = torch.log_softmax(z, dim=0)[y]
            kept[t] = torch.log(P[y] / N)
            if stop:
                break
    return {"ids": None, "accepted": None, "logp": logp, "logp_kept": kept}


def exact(case, seed):
    s = _prepare(case, seed)
    if case["kind"] == "verify":
        return _exact_verify(case, s)
    one = _exact_norm if case["kind"] == "norm" else _exact_grad
    step = max(1, (1 << 26) // case["H"])
    parts = [one(case, s, slice(r, min(case["T"], r + step))) for r in range(0, case["T"], step)]
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0] if k != "dweight"}
    if "dweight" in parts[0]:
        out["dweight"] = sum(p["dweight"] for p in parts)
    return out
