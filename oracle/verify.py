"""CPU oracle of the verification of drafted tokens (include/cis_verify.h): plain numpy, a sequence at a
time, written from its definition on the weights of oracle.tokens. Test infrastructure only; shares
no code with the HIP path. Weights and sums are whole numbers; what is compared with them is in double,
rounded at each step, as the definition has it."""

from __future__ import annotations

import math

import numpy as np

from . import tokens


def accepts(P, d, u, Q=None):
    """Whether draft d is accepted with the random number u. P and Q: int64 weights of kept tokens."""
    N = float(int(P.sum()))
    share = N if Q is None else float(Q[d]) * (N / float(int(Q.sum())))
    return u * share < float(P[d])


def leftover(P, d, Q=None):
    """Weights of the draw in place of a draft that was turned down."""
    if Q is None:
        left = P.copy()
        left[d] = 0
    else:
        rho = float(int(P.sum())) / float(int(Q.sum()))
        left = np.maximum(P - np.floor(Q.astype(np.float64) * rho).astype(np.int64), 0)
    return left if left.sum() > 0 else P


def pick(w, u):
    total = int(w.sum())
    at = min(int(u * float(total)), total - 1)
    return int(np.searchsorted(np.cumsum(w), at, side="right"))


def sequence(P, drafts, us, Q=None):
    """([ids], drafts accepted) of one sequence: P a list of a row's weights each (None: it cannot be drawn
    from), one more than drafts; Q the drafts' or None; us one number per row, a bad one NaN."""
    ids = []
    for i, p in enumerate(P):
        if p is None or not 0 <= us[i] < 1:
            return ids, len(ids)
        if i == len(P) - 1:
            return ids + [pick(p, us[i])], len(ids)
        q = None if Q is None else Q[i]
        if (Q is not None and q is None) or not 0 <= drafts[i] < p.size:
            return ids, len(ids)
        if not accepts(p, drafts[i], us[i], q):
            n = len(ids)
            if 0 <= us[-1] < 1:
                ids = ids + [pick(leftover(p, drafts[i], q), us[-1])]
            return ids, n
        ids.append(int(drafts[i]))
    return ids, 0


def kept_weights(z, q, top_k=0, top_p=1.0, min_p=0.0, greedy=False):
    return np.where(tokens.kept_tokens(z, q, top_k, top_p, min_p, greedy), q, 0)


def kept_logp(P, y):
    return math.log(int(P[y]) / int(P.sum()))
