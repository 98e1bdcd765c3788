"""Pins of the verification's oracle: what comes out is distributed as the target's own draws."""

import numpy as np
import pytest

from oracle import tokens, verify as orc


def _weights(rng, V, sharp=1.0, banned=0):
    z = (rng.normal(size=V) * sharp).astype(np.float32)
    z[rng.permutation(V)[:banned]] = -np.inf
    return tokens.draw_weights(tokens.draw_exponents(z, 1.0))


@pytest.mark.parametrize("V,sharp,banned,certain", [
    (2, 1.0, 0, False), (5, 3.0, 2, False), (17, 0.1, 0, False), (40, 6.0, 25, False),
    (5, 2.0, 1, True), (17, 1.0, 0, True)])
def test_one_draft_leaves_the_targets_distribution(V, sharp, banned, certain):
    """Over all drafts and random numbers: an accepted one has probability min(1, P_d N' / (Q_d N)), and the
    draw in its place the leftover weights'. Off by the floors, 1 of 2^28 a token."""
    rng = np.random.default_rng(V + banned)
    P, Q = _weights(rng, V, sharp, banned), _weights(rng, V, sharp, banned // 2)
    N, Nq = float(P.sum()), float(Q.sum())
    if certain:
        Q = np.zeros(V, np.int64)
        Q[rng.integers(V)] = Nq = 1
    out = np.zeros(V)
    for d in range(V):
        if Q[d] == 0:
            continue
        share = Q[d] * (N / Nq) if not certain else N
        take = min(1.0, P[d] / share)
        assert orc.accepts(P, d, 0.999 * take, None if certain else Q) == (P[d] > 0)
        assert not orc.accepts(P, d, min(1.001 * take, 1.0), None if certain else Q) or take == 1
        left = orc.leftover(P, d, None if certain else Q).astype(float)
        out += Q[d] / Nq * (take * (np.arange(V) == d) + (1 - take) * left / left.sum())
    assert np.abs(out - P / N).max() < 1e-6 if not certain else np.abs(out - P / N).max() < 1e-12


def test_ends_of_a_sequence():
    P = [np.array([3, 1], np.int64)] * 3
    assert orc.sequence(P, [0, 0], [0.5, 0.5, 0.9]) == ([0, 0, 1], 2)
    assert orc.sequence(P, [1, 0], [0.5, 0.5, 0.0]) == ([0], 0)       # turned down: only 0 is left
    assert orc.sequence(P, [0, 7], [0.5, 0.5, 0.9]) == ([0], 1)       # no such id
    assert orc.sequence([P[0], None, P[0]], [0, 0], [0.5, 0.5, 0.9]) == ([0], 1)
    assert orc.sequence(P[:1], [], [0.8]) == ([1], 0)
    assert orc.sequence(P[:1], [], [float("nan")]) == ([], 0)
    assert orc.sequence([], [], []) == ([], 0)
    # nothing is left of equal weights: the draw is from all of them
    assert orc.leftover(P[0], 0, P[0]).tolist() == [3, 1]


def test_pick_is_the_samplers_rule():
    rng = np.random.default_rng(0)
    z = rng.normal(size=50).astype(np.float32)
    q = tokens.draw_weights(tokens.draw_exponents(z, 1.0))
    for u in rng.random(50).astype(np.float32):
        assert orc.pick(q, float(u)) == tokens.draw(z, q, u)[0]
