"""The verification of drafted tokens on the GPU against the oracle (oracle/verify.py).

Ids and counts are compared exactly: weights come from the definition's float32 exponents through
torch.exp2 on the same device (whose result equals the hardware's wherever a weight is not 0), and
all that follows is whole numbers, or double rounded as the definition says.

Tolerances of the log-probabilities are those of the draws (tests/test_gpu_tokens.py): logp_kept is
rounded once; logp is the difference of two logits and the log of a sum, whose exponents round once each
below 128 in base 2: 2^-24 (128 + 2 * 32) ln 2 and less than 2e-6 for exp2 and the sums, under 1e-5.
"""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2609_32444_amd as cis
from oracle import tokens, verify as orc
from paper_2609_32444_amd import _tokens, _verify

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOL = 1e-5
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _store(z, dtype, pad=0):
    T, V = z.shape
    epv = 16 // dtype.itemsize
    ld = (V + epv - 1) // epv * epv + pad * epv
    s = torch.full((max(T, 1), ld), math.nan, dtype=dtype, device=DEV)
    s[:T, :V] = z.to(dtype)
    return s[:T, :V]


def _logits(T, V, seed, kind="normal"):
    g = _gen(seed)
    z = torch.randn(T, V, generator=g, device=DEV) * 3
    if kind == "ties":
        z = z.round()
    if kind == "banned":
        z[torch.rand(T, V, generator=g, device=DEV) < 0.6] = -math.inf
        z[:, V // 2] = 1.0
    if kind == "peaked":
        z[torch.arange(T), torch.randint(0, V, (T,), generator=g, device=DEV)] += 25
    if kind == "lowest":
        z[torch.rand(T, V, generator=g, device=DEV) < 0.6] = torch.finfo(BF).min
    return z


def _row_weights(logits, s):
    """(kept weights, logits) of a row, or None where it cannot be drawn from."""
    z = logits.float().cpu().numpy()
    if not tokens.drawable(z):
        return None
    t = tokens.draw_exponents(z, s.get("temperature", 1.0))
    greedy = t is None
    if greedy:
        q = np.where(z == z.max(), tokens.ONE, 0).astype(np.int64)
    else:
        q = (torch.exp2(torch.from_numpy(t).to(DEV)) * tokens.ONE).long().cpu().numpy()
    return orc.kept_weights(z, q, int(s.get("top_k", 0)), s.get("top_p", 1.0), s.get("min_p", 0.0),
                            greedy)


def _setting(settings, b):
    return {k: (v[b].item() if isinstance(v, torch.Tensor) else v) for k, v in settings.items()}


def _check(logits, draft_ids, u, offsets, draft_logits, out, settings, only=None):
    """Every sequence (or those of `only`) against the oracle."""
    T = logits.shape[0]
    ids, lp, lk = (out[k].cpu().numpy() for k in ("ids", "logp", "logp_kept"))
    acc, us, drafts = out["accepted"].cpu().numpy(), u.double().cpu().numpy(), draft_ids.tolist()
    seen = np.zeros(T, bool)
    for b in range(len(offsets) - 1):
        o0, o1 = offsets[b], offsets[b + 1]
        seen[o0:o1] = True
        if only is not None and b not in only:
            continue
        s = _setting(settings, b)
        P = [_row_weights(logits[t], s) for t in range(o0, o1)]
        Q = None
        if draft_logits is not None:
            Q = [_row_weights(draft_logits[t - b], s) for t in range(o0, o1 - 1)]
        want, n = orc.sequence(P, drafts[o0 - b:o1 - b - 1] if o1 > o0 else [], us[o0:o1], Q)
        assert ids[o0:o1].tolist() == want + [-1] * (o1 - o0 - len(want)), (b, acc[b], n)
        assert acc[b] == n, b
        for i, y in enumerate(want):
            ref = tokens.log_softmax_at(logits[o0 + i].float().cpu().numpy(), y)
            assert abs(lp[o0 + i] - ref) <= TOL * min(1.0, abs(ref)) + 2.0 ** -22 * abs(ref)
            ref = orc.kept_logp(P[i], y)
            assert abs(lk[o0 + i] - ref) <= 2.0 ** -23 * abs(ref)
    none = ids == -1
    assert none[~seen].all() and not lp[none].any() and not lk[none].any()


def _batch(lengths, V, seed, dtype, kind="normal", near=0.7, certain=False, settings=None, pad=0):
    """Logits of sequences with `lengths` rows each, drafts drawn from a draft model near the target."""
    B, T = len(lengths), sum(lengths)
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    g = _gen(seed + 1000)
    z = _logits(T, V, seed, kind)
    rows = [t for b in range(B) for t in range(offsets[b], offsets[b + 1] - 1)]
    logits = _store(z, dtype, pad)
    u = torch.rand(T, generator=g, device=DEV)
    draft_logits, D = None, len(rows)
    draft_ids = torch.zeros(D, dtype=torch.int64, device=DEV)
    if D and not certain:
        q = z[rows] + near * torch.randn(D, V, generator=g, device=DEV)
        draft_logits = _store(q, dtype, pad + 1)
        seq = torch.tensor([b for b in range(B) for _ in range(max(lengths[b] - 1, 0))], device=DEV)
        s = {k: (v[seq].contiguous() if isinstance(v, torch.Tensor) else v)
             for k, v in (settings or {}).items()}
        draft_ids = cis.sample(draft_logits, torch.rand(D, generator=g, device=DEV), **s)["ids"]
    elif D:
        best = z[rows].argmax(1)
        other = torch.randint(0, V, (D,), generator=g, device=DEV)
        draft_ids = torch.where(torch.rand(D, generator=g, device=DEV) < 0.7, best, other)
    return logits, draft_ids, u, offsets, draft_logits


def _run(logits, draft_ids, u, offsets, draft_logits, settings, **kw):
    return cis.verify(logits, draft_ids, u, torch.tensor(offsets, device=DEV), draft_logits,
                      **settings, **kw)


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.6), dict(temperature=7.5),
            dict(top_k=1), dict(top_k=5), dict(top_k=40), dict(top_k=1 << 30), dict(top_p=0.3),
            dict(top_p=0.9), dict(top_p=0.999999), dict(min_p=0.1), dict(min_p=1.0),
            dict(top_k=30, top_p=0.8, min_p=0.01, temperature=1.3),
            dict(temperature=1e-3, top_p=0.5), dict(temperature=1e-42), dict(temperature=1e30)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["normal", "ties", "banned", "peaked", "lowest"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 1000, 4097])
def test_verify(V, kind, dtype):
    lengths = [3, 1, 5, 2, 1, 4]
    for i, s in enumerate(SETTINGS):
        batch = _batch(lengths, V, V + i, dtype, kind, certain=i % 3 == 2, settings=s, pad=i % 2)
        _check(*batch, _run(*batch, s), s)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [50257, 151936, 262144, 300001])
def test_long_rows(V, dtype):
    for i, s in enumerate((dict(), dict(top_k=50, top_p=0.9, temperature=0.7), dict(top_p=0.95),
                           dict(top_k=1500), dict(top_k=3000, top_p=0.7), dict(min_p=0.02),
                           dict(temperature=0.0), dict(temperature=4.0))):
        for kind in ("normal", "ties", "peaked"):
            batch = _batch([2, 1, 3], V, 7 + i, dtype, kind, settings=s, certain=i % 4 == 3)
            _check(*batch, _run(*batch, s), s)


@pytest.mark.parametrize("order", ["equal", "two values", "one block", "rising"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_cuts_among_equal_logits(order, dtype):
    """Where a cut falls among many tokens of one logit, the lowest ids are kept."""
    V = 20000
    j = torch.arange(V, device=DEV, dtype=F32)
    z = {"rising": j / 2000, "equal": 0 * j + 1.5, "two values": (j % 3 == 1).float(),
         "one block": torch.where((j >= 7000) & (j < 9000), j % 17 / 8 + 4, -j / V)}[order]
    logits = _store(z.expand(6, V), dtype)
    offsets = [0, 3, 6]
    shift = _store(z.roll(5).expand(4, V), dtype)
    u = torch.tensor([0.1, 0.9, 0.3, 0.7, 0.999, 0.6], device=DEV)
    for s in (dict(), dict(top_k=7), dict(top_k=700), dict(top_k=1024), dict(top_k=5000),
              dict(top_p=0.5), dict(top_p=0.01), dict(top_k=900, top_p=0.6), dict(min_p=0.9),
              dict(top_k=6000, top_p=0.9), dict(top_k=3000, min_p=0.5)):
        for q in (shift, None, logits[:4]):
            ids = cis.sample(shift if q is None else q, u[:4], **s)["ids"]
            _check(logits, ids, u, offsets, q, _run(logits, ids, u, offsets, q, s), s)


@pytest.mark.parametrize("n", [63, 64, 65, 128, 129, 200])
def test_long_drafts(n):
    """More drafts than a wave has lanes, all accepted, or turned down at either side of the 64th."""
    V = 300
    logits, ids, u, offsets, q = _batch([n, 2, n + 1], V, n, F32, near=0.0)
    out = _run(logits, ids, u, offsets, q, {})
    assert out["accepted"].tolist() == [n - 1, 1, n]      # the draft is the target
    _check(logits, ids, u, offsets, q, out, {})
    for at in (61, 62, 63, 64, 65, n - 2):
        if at < n - 1:
            turned = ids.clone()
            turned[at] = int(logits[at].argmin())
            q2 = q.clone()
            q2[at] = 0.0
            q2[at, turned[at]] = 30.0
            u2 = u.clone()
            u2[at] = 0.9
            out = _run(logits, turned, u2, offsets, q2, {})
            assert out["accepted"][0] == at
            _check(logits, turned, u2, offsets, q2, out, {})


def test_many_sequences_and_settings_of_their_own():
    g = _gen(3)
    B, V = 500, 700
    lengths = torch.randint(1, 7, (B,), generator=g, device=DEV).tolist() + [0, 0]
    choose = lambda v, dt: torch.tensor(v, dtype=dt, device=DEV)[  # noqa: E731
        torch.randint(0, len(v), (B + 2,), generator=g, device=DEV)]
    s = dict(temperature=choose([0.0, 0.5, 1.0, 1.5], F32), top_k=choose([0, 1, 20, 600], torch.int32),
             top_p=choose([0.5, 0.9, 1.0], F32), min_p=choose([0.0, 0.0, 0.05], F32))
    for certain in (False, True):
        batch = _batch(lengths, V, 11, BF, certain=certain, settings=s)
        _check(*batch, _run(*batch, s), s)
    one = dict(s, top_k=0, min_p=0.0)
    batch = _batch(lengths, V, 12, F32, settings=one)
    _check(*batch, _run(*batch, one), one)
    # out of range for some: their rows cannot be drawn from
    s["temperature"][3], s["top_p"][10], s["min_p"][20], s["top_k"][30] = -1.0, 0.0, 2.0, -5
    batch = _batch(lengths, V, 13, BF, certain=True)
    out = _run(*batch, s)
    bad = [3, 10, 20, 30]
    off = batch[3]
    for b in bad:
        assert out["accepted"][b] == 0 and torch.all(out["ids"][off[b]:off[b + 1]] == -1)
    _check(*batch, out, s, only=[b for b in range(B) if b not in bad])


def _same_as_settings_of_their_own(batch):
    """A temperature of 1 per sequence takes the kernels that weigh every row; one for all, over as many
    logits as here, those that look at what the scan's sums decide first. Every output is the same."""
    ones = torch.ones(len(batch[3]) - 1, device=DEV)
    a, b = _run(*batch, {}), _run(*batch, dict(temperature=ones))
    for k in ("ids", "accepted", "logp", "logp_kept"):
        assert torch.equal(a[k], b[k]), k
    return a


@pytest.mark.parametrize("kind", ["normal", "peaked", "banned"])
@pytest.mark.parametrize("near", [0.0, 0.02, 0.7, 4.0])
def test_drafts_that_the_sums_decide(near, kind):
    """At temperature 1 with nothing cut, over more than 80 MiB of logits: drafts from the target itself, from close
    to it (where many a random number is near its border) and from far away."""
    batch = _batch([5, 7, 1, 4, 2, 9, 3, 70, 6], 300001, int(10 * near), F32, kind, near=near)
    out = _same_as_settings_of_their_own(batch)
    if near == 0.0:
        assert out["accepted"].tolist() == [4, 6, 0, 3, 1, 8, 2, 69, 5]
    _check(*batch, out, {}, only=[0, 3, 4])
    # random numbers at the very border of the first draft's acceptance, and one step beside it
    logits, ids, u, offsets, q = batch
    P, Q = _row_weights(logits[0], {}), _row_weights(q[0], {})
    share = float(Q[ids[0]]) * (float(int(P.sum())) / float(int(Q.sum())))
    edge = np.float32(min(float(P[ids[0]]) / share, 1 - 2.0 ** -24))
    for x in (edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(1))):
        u[0] = float(min(x, np.float32(1 - 2.0 ** -24)))
        _check(*batch, _same_as_settings_of_their_own(batch), {}, only=[0])


@pytest.mark.parametrize("dtype,V,n", [(BF, 151936, 64), (F32, 32768, 200), (BF, 50257, 300)])
def test_decided_batches(dtype, V, n):
    for certain in (False, True):
        g = _gen(V + certain)
        lengths = torch.randint(1, 8 if not certain else 14, (n,), generator=g, device=DEV).tolist()
        _same_as_settings_of_their_own(_batch(lengths, V, n, dtype, "peaked", certain=certain))


def test_unusable_rows_among_decided_ones():
    V = 300001
    lengths = [5] * 9
    logits, ids, u, offsets, q = _batch(lengths, V, 2, F32, near=0.0)
    logits[offsets[1] + 1, 7] = math.nan
    logits[offsets[2] + 4, 8] = math.inf
    q[offsets[3] - 3 + 2, V - 1] = math.nan
    q[offsets[4] - 4] = -math.inf
    ids[offsets[5] - 5 + 1], ids[offsets[6] - 6] = V, -1
    u[offsets[7] + 1], u[offsets[8] + 4] = math.nan, 1.0
    batch = (logits, ids, u, offsets, q)
    out = _same_as_settings_of_their_own(batch)
    assert out["accepted"].tolist() == [4, 1, 4, 2, 0, 1, 0, 1, 4]
    _check(*batch, out, {}, only=[1, 3, 4, 5, 7, 8])
    # a draft that is surely turned down ahead of rows that cannot be used, which nobody looks at
    for b in (1, 3, 5):
        ids[offsets[b] - b] = int(logits[offsets[b]].argmin())
        u[offsets[b]] = 0.999
        q[offsets[b] - b, ids[offsets[b] - b]] = 40.0
    out = _same_as_settings_of_their_own(batch)
    assert out["accepted"].tolist() == [4, 0, 4, 0, 0, 0, 0, 1, 4]
    _check(*batch, out, {}, only=[1, 3, 5])


def test_a_sequence_of_one_row_is_a_draw():
    V, T = 5000, 40
    logits = _store(_logits(T, V, 1), BF)
    u = torch.rand(T, generator=_gen(2), device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    for s in SETTINGS:
        want = cis.sample(logits, u, **s)
        for q in (None, torch.empty(0, V, dtype=BF, device=DEV)):
            out = _run(logits, none, u, list(range(T + 1)), q, s)
            assert not out["accepted"].any()
            for k in ("ids", "logp", "logp_kept"):
                assert torch.equal(out[k], want[k]), k


def test_rows_that_cannot_be_drawn_from():
    V = 900
    lengths = [4, 4, 4, 4, 4, 4, 4, 4, 4, 4, 4]
    logits, ids, u, offsets, q = _batch(lengths, V, 5, F32, near=0.0)
    logits[offsets[1] + 1, 7] = math.nan              # a target row
    logits[offsets[2] + 3, 8] = math.inf              # the row after the last draft
    q[offsets[3] - 3 + 2, 9] = math.nan               # a draft's row
    q[offsets[4] - 4] = -math.inf
    ids[offsets[5] - 5 + 1] = V                       # drafts that are no ids
    ids[offsets[6] - 6] = -1
    ids[offsets[7] - 7 + 2] = 1 << 40
    u[offsets[8] + 1], u[offsets[9] + 3], u[offsets[10]] = math.nan, 1.0, -0.5
    us = u.clone()
    out = _run(logits, ids, u, offsets, q, {})
    assert out["accepted"].tolist() == [3, 1, 3, 2, 0, 1, 0, 2, 1, 3, 0]
    _check(logits, ids, us, offsets, q, out, {})
    # certain drafts at the same places, and a turned-down draft whose draw has no number
    ids[offsets[9] - 9] = int(logits[offsets[9]].argmin())
    u[offsets[9]] = 0.99
    for draft in (q, None):
        out = _run(logits, ids, u, offsets, draft, {})
        _check(logits, ids, u, offsets, draft, out, {})
    assert out["accepted"][9] == 0 and out["ids"][offsets[9]] == -1


def test_nothing_left_of_equal_distributions():
    """A draft without weight on either side is turned down; what is left of equal weights is nothing, and the
    draw is from all of them."""
    V = 3000
    z = _logits(2, V, 1)
    z[0, 5] = -math.inf
    logits = _store(z, BF)
    ids = torch.tensor([5], device=DEV)
    for k in range(8):
        u = torch.tensor([0.5, k / 8], device=DEV)
        out = _run(logits, ids, u, [0, 2], logits[:1], {})
        _check(logits, ids, u, [0, 2], logits[:1], out, {})
        assert out["ids"][0] == cis.sample(logits[:1], u[1:].clone())["ids"][0]


def test_offsets_out_of_range():
    """Offsets that rise beyond the rows, fall, or ask for drafts that are not there: -1, and no token."""
    V = 64
    logits, ids, u, offsets, q = _batch([3, 3, 3], V, 1, BF, near=0.0)
    for offs, bad in (([0, 3, 6, 99], [2]), ([0, 3, 2, 9], [1]), ([-4, 3, 6, 9], [0]),
                      ([0, 1 << 40, 6, 9], [0, 1]), ([0, -(1 << 62), 6, 9], [0, 1])):
        for draft in (q, None):
            out = _run(logits, ids, u, offs, draft, {})
            for b in range(3):
                assert (out["accepted"][b] == -1) == (b in bad), (offs, b, out["accepted"])
    # too few drafts for the last sequence; empty sequences in front leave no place for a draft
    out = _run(logits, ids[:5].clone(), u, offsets, q[:5], {})
    assert out["accepted"].tolist() == [2, 2, -1] and torch.all(out["ids"][6:] == -1)
    out = _run(logits, ids, u, [0, 0, 3, 9], q, {})
    assert out["accepted"].tolist()[:2] == [0, -1]
    # rows that no sequence has, whatever they hold
    logits[6:] = math.nan
    u[6:] = math.nan
    out = _run(logits, ids, u, [0, 3, 6, 6], q, {})
    assert out["accepted"].tolist() == [2, 2, 0] and torch.all(out["ids"][6:] == -1)
    _check(logits, ids, u, [0, 3, 6, 6], q, out, {})
    # no rows at all
    empty = _run(logits[:0], ids[:0], u[:0], [0, 0, 0], None, {})
    assert empty["accepted"].tolist() == [0, 0] and empty["ids"].numel() == 0


def test_offsets_beyond_32_bits():
    V = 262144
    T = (1 << 32) // (V * 2) + 6
    logits = torch.zeros(T, V, dtype=BF, device=DEV)
    D = T - 2
    q = torch.zeros(D, V, dtype=BF, device=DEV)
    tail = _logits(6, V, 1)
    logits[-6:] = tail.to(BF)
    q[-5:] = (tail[:5] + 0.5 * _logits(5, V, 2) / 3).to(BF)
    ids = torch.zeros(D, dtype=torch.int64, device=DEV)
    u = torch.rand(T, generator=_gen(1), device=DEV)
    ids[-5:] = cis.sample(q[-5:], u[:5].clone())["ids"]
    u[:T - 6] = 0.999
    offsets = [0, T - 6, T]
    out = _run(logits, ids, u, offsets, q, {})
    _check(logits, ids, u, offsets, q, out, {}, only=[1])
    assert out["accepted"][0] == T - 7     # equal logits: every draft is accepted


def test_more_rows_than_a_launch_takes():
    """Rows in several launches of the sampling kernels, with and without a nucleus (2048 rows of it each)."""
    V = 32
    lengths = [3] * 2000
    for s in (dict(top_p=0.9), dict()):
        batch = _batch(lengths, V, 3, F32, settings=s)
        _check(*batch, _run(*batch, s), s, only=list(range(0, 2000, 97)) + [1365, 1366, 1999])


def test_streams_graphs_and_repeats():
    V = 50257
    s = dict(top_p=0.95, temperature=0.9)
    a = _batch([4, 1, 6, 3], V, 1, BF, settings=s)
    b = _batch([4, 1, 6, 3], V, 2, BF, settings=s)
    offs = torch.tensor(a[3], device=DEV)
    make = lambda x: cis.VerifyCall(x[0], x[1], x[2], offs, x[4], **s)  # noqa: E731
    call, other = make(a), make(b)
    want_a = {k: v.clone() for k, v in call.run().items() if k != "workspace"}
    want_b = {k: v.clone() for k, v in other.run().items() if k != "workspace"}
    same = lambda out, want: all(torch.equal(out[k], want[k]) for k in want)  # noqa: E731
    assert not same(call.out, want_b)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        for st, c in zip(streams, (call, other)):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                c.run()
        for st in streams:
            torch.cuda.current_stream().wait_stream(st)
        assert same(call.out, want_a) and same(other.out, want_b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    keep = [t.clone() for t in (a[0], a[1], a[2], a[4])]
    for rep in range(4):
        src = keep if rep % 2 else (b[0], b[1], b[2], b[4])
        for dst, t in zip((a[0], a[1], a[2], a[4]), src):
            dst.copy_(t)
        call.workspace.fill_(255 if rep < 2 else 0)
        for k in want_a:
            call.out[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(call.out, want_a if rep % 2 else want_b)
        torch.randn(1000, 1000, device=DEV).sum().item()


def _placed(n=2, T=6, D=4, V=64):
    """The arguments of cis_verify in one buffer, apart from each other: (buffer, {name: (offset, bytes)})."""
    need = cis.verify_workspace_bytes(T, D, n, V, F32)
    sizes = dict(logits=T * V * 4, q=D * V * 4, ids=D * 8, u=T * 4, offs=(n + 1) * 8, temps=n * 4, ks=n * 4,
                 ps=n * 4, ms=n * 4, out=T * 8, acc=n * 4, lp=T * 4, lk=T * 4, ws=need)
    at, end = {}, 256
    for name, size in sizes.items():
        at[name] = (end, size)
        end = (end + size + 255) // 256 * 256
    buf = torch.zeros(end + 256, dtype=torch.uint8, device=DEV)
    put = lambda name, t: buf[at[name][0]:][:at[name][1]].copy_(t.view(torch.uint8).view(-1))  # noqa: E731
    logits, ids, u, offsets, q = _batch([3, 3], V, 1, F32)
    for name, t in (("logits", logits), ("q", q), ("ids", ids), ("u", u),
                    ("offs", torch.tensor(offsets, device=DEV)), ("temps", torch.ones(n, device=DEV)),
                    ("ks", torch.zeros(n, dtype=torch.int32, device=DEV)), ("ps", torch.ones(n, device=DEV)),
                    ("ms", torch.zeros(n, device=DEV))):
        put(name, t.contiguous())
    want = cis.verify(logits, ids, u, torch.tensor(offsets, device=DEV), q)
    return buf, at, want


def _call_placed(base, at, n=2, T=6, D=4, V=64, **moved):
    p = {k: base + v[0] for k, v in at.items()}
    p.update(moved)
    prm = _tokens._SampleParams(1.0, 0, 1.0, 0.0)
    return _verify._lib().cis_verify(
        p["logits"], 1, T, V, V, p["q"], D, V, p["ids"], p["u"], p["offs"], n, ctypes.byref(prm), p["temps"],
        p["ks"], p["ps"], p["ms"], p["out"], p["acc"], p["lp"], p["lk"], p["ws"], at["ws"][1],
        torch.cuda.current_stream().cuda_stream)


def test_overlapping_arguments_are_refused():
    """Each output, and the workspace, on each other argument: at its first bytes and at its last ones."""
    buf, at, want = _placed()
    base = buf.data_ptr()
    assert base % 256 == 0
    keep = buf.clone()
    outs = ("out", "acc", "lp", "lk", "ws")
    for o in outs:
        for a in at:
            if a == o:
                continue
            first, last = base + at[a][0], base + at[a][0] + at[a][1]
            step = 256 if o == "ws" else 8 if o == "out" else 4
            for place in (first, (last - 1) // step * step):
                assert _call_placed(base, at, **{o: place}) == -8, (o, a)
            # and up to the first byte of it
            place = first - at[o][1] + step
            assert place % step or _call_placed(base, at, **{o: place}) == -8, (o, a)
    torch.cuda.synchronize()
    assert torch.equal(buf, keep)      # nothing was launched
    assert _call_placed(base, at) == 0
    got = lambda name, dt: buf[at[name][0]:][:at[name][1]].view(dt)  # noqa: E731
    assert torch.equal(got("out", torch.int64), want["ids"])
    assert torch.equal(got("acc", torch.int32), want["accepted"])
    assert torch.equal(got("lp", F32), want["logp"]) and torch.equal(got("lk", F32), want["logp_kept"])
    # side by side is no overlap
    assert _call_placed(base, at, lp=base + at["out"][0] + at["out"][1]) == 0
    torch.cuda.synchronize()


def test_binding_refuses():
    V = 64
    logits, ids, u, offsets, q = _batch([3, 3], V, 1, BF)
    offs = torch.tensor(offsets, device=DEV)
    bad = [
        lambda: cis.verify(logits.half(), ids, u, offs, q), lambda: cis.verify(logits, ids.int(), u, offs, q),
        lambda: cis.verify(logits, ids, u[:4], offs, q), lambda: cis.verify(logits, ids, u, offs, q.float()),
        lambda: cis.verify(logits, ids, u, offs, q[:3]), lambda: cis.verify(logits, ids, u, offs.int(), q),
        lambda: cis.verify(logits, ids, u, None, q), lambda: cis.verify(logits, ids, u, offs[:1], q),
        lambda: cis.verify(logits, ids, u, offs.cpu(), q), lambda: cis.verify(logits, ids[::2], u, offs, q),
        lambda: cis.verify(logits, ids, u, offs, q[:, :32]), lambda: cis.verify(logits, None, u, offs, q),
        lambda: cis.verify(logits, ids, u, offs, q, temperature=torch.ones(6, device=DEV)),
        lambda: cis.verify(logits, ids, u, offs, q, V=65),
        lambda: cis.verify(logits, ids, u, offs, q, workspace=torch.empty(9, device=DEV)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for kw in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=0.0), dict(min_p=1.5)):
        with pytest.raises(cis.CisError):
            cis.verify(logits, ids, u, offs, q, **kw)
