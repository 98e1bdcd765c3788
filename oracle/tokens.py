"""CPU oracle of the token operators (include/cis_tokens.h): plain numpy, one row at a time, written
from their definitions. Test infrastructure only; shares no code with the HIP path.

Draws and ranks are whole numbers and exact; everything else is float64.
"""

from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np

ONE = 1 << 28   # a draw's weight of the largest logit


def draw_exponents(z, temperature):
    """Exponents (base 2) of a draw's weights, with the definition's float32 roundings; None for
    a greedy row. z float32 with a finite maximum."""
    f = np.float32
    with np.errstate(divide="ignore", over="ignore"):
        c = f(1.4426950408889634) / f(temperature)
    if not np.isfinite(c):
        return None
    with np.errstate(over="ignore"):
        return (z.astype(f) - z.max().astype(f)) * c


def draw_weights(t):
    """floor(2^28 2^t) for exact powers of two (an implementation's exp2 may differ by its own
    rounding: pass its weights to draw() to check the rest exactly)."""
    return np.floor(np.exp2(t.astype(np.float64)) * ONE).astype(np.int64)


def order(z):
    """Ids by (logit descending, id ascending), tokens (z > -inf) only."""
    z = z.astype(np.float64) + 0.0
    ids = np.lexsort((np.arange(z.size), -z))
    return ids[z[ids] > -np.inf]


def kept_tokens(z, q, top_k=0, top_p=1.0, min_p=0.0, greedy=False):
    """Mask of the tokens that the cuts keep, for weights q."""
    ids = order(z)
    n = 1 if greedy else ids.size if top_k == 0 else min(int(top_k), ids.size)
    if not greedy:
        cum = [int(c) for c in np.cumsum(q[ids[:n]], dtype=object)]
        first = n
        p = float(np.float32(top_p))
        if p < 1.0:
            want = math.ceil(p * float(cum[-1]))
            first = 1 + next(i for i, c in enumerate(cum) if c >= want)
        least = math.ceil(float(np.float32(min_p)) * ONE)
        n = min(n, first, int((q[ids] >= least).sum()))
    kept = np.zeros(z.size, bool)
    kept[ids[:n]] = True
    return kept


def draw(z, q, u, top_k=0, top_p=1.0, min_p=0.0, greedy=False):
    """(id, log q_id / N) of a row that can be drawn from."""
    kept = kept_tokens(z, q, top_k, top_p, min_p, greedy)
    w = np.where(kept, q, 0)
    total = int(w.sum())
    at = min(int(float(np.float32(u)) * float(total)), total - 1)
    y = int(np.searchsorted(np.cumsum(w), at, side="right"))
    return y, math.log(int(w[y]) / total)


def drawable(z):
    return bool(not np.isnan(z).any() and not np.isposinf(z).any() and np.isfinite(z.max()))


def log_softmax_at(z, y):
    z = z.astype(np.float64)
    rest = np.exp(z - z[y])
    rest[y] = 0.0
    return -math.log1p(rest.sum())


@dataclass
class TopList:
    ids: np.ndarray       # [K] int64, -1 past the last token
    values: np.ndarray    # [K] float64, -inf past it
    tail: float


def top_list(z, K, temperature=1.0):
    ids = np.full(K, -1, np.int64)
    values = np.full(K, -np.inf)
    if np.isnan(z).any() or np.isposinf(z).any():
        return TopList(ids, values, math.nan)
    best = order(z)
    n = min(K, best.size)
    ids[:n] = best[:n]
    values[:n] = z[best[:n]].astype(np.float64) + 0.0
    rest = z[best[n:]].astype(np.float64) / temperature
    tail = -math.inf
    if rest.size:
        tail = float(rest[0] + math.log(np.exp(rest - rest[0]).sum()))
    return TopList(ids, values, tail)


@dataclass
class Distilled:
    valid: bool
    bad: bool
    term: float
    grad: np.ndarray      # [V]
    p: np.ndarray         # [V] student probabilities
    q: np.ndarray         # [V] teacher's, 0 where not listed
    p_rest: float
    q_rest: float
    kl: float


def _kl(a, b):
    """sum a log(a/b) over classes, 0 log 0 = 0."""
    total = 0.0
    for x, y in zip(a, b):
        if x > 0:
            total += x * (math.log(x) - math.log(y)) if y > 0 else math.inf
    return total


def distill_row(z, ids, values, tail, reverse=False, temperature=1.0, weight=1.0, scale=1.0,
                on=True):
    """One row of the distillation loss; tail None: the teacher is its list alone."""
    V = z.size
    zero = np.zeros(V)
    got = ids[ids != -1]
    bad = bool(((got < 0) | (got >= V)).any() or np.unique(got).size != got.size)
    if not on or bad or got.size == 0:
        return Distilled(False, on and bad, 0.0, zero, zero, zero, 0.0, 0.0, 0.0)
    t = np.concatenate([values[ids != -1].astype(np.float64) / temperature,
                        [-math.inf if tail is None else float(tail)]])
    share = np.exp(t - t.max())
    share /= share.sum()
    x = z.astype(np.float64) / temperature
    p = np.exp(x - x.max())
    listed = np.zeros(V, bool)
    listed[got] = True
    rest = p[~listed].sum()
    total = p[listed].sum() + rest
    p, p_rest = p / total, rest / total
    q = np.zeros(V)
    q[got] = share[:-1]
    q_rest = float(share[-1])
    a, b = np.append(p[got], p_rest), share
    kl = _kl(a, b) if reverse else _kl(b, a)
    with np.errstate(divide="ignore", invalid="ignore"):
        if reverse:
            d = np.where(listed, np.log(p) - np.log(q),
                         np.log(p_rest) - np.log(q_rest) if p_rest > 0 else 0.0)
            grad = np.where(p > 0, p * (d - kl), 0.0)
        else:
            grad = np.where(listed, p - q, p * (1 - q_rest / p_rest) if p_rest > 0 else 0.0)
    w = float(weight) * float(scale)
    if w == 0.0:
        return Distilled(True, False, 0.0, zero, p, q, p_rest, q_rest, kl)
    return Distilled(True, False, w * kl, grad * (w / temperature), p, q, p_rest, q_rest, kl)
