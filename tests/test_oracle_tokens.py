"""The oracle of the token operators against closed forms, enumerations and differences, and its
mistakes: each planted one fails a pin."""

import math

import numpy as np
import pytest

from oracle import tokens as orc

RNG = np.random.default_rng


def _q(z, temperature=1.0):
    return orc.draw_weights(orc.draw_exponents(z, temperature))


def test_draw_covers_each_token_by_its_weight():
    """Random numbers on a grid finer than the weights hit each token exactly as often."""
    z = np.log(np.array([4.0, 1.0, 2.0, 1.0], np.float32))
    q = np.array([4, 1, 2, 1]) * (orc.ONE // 4)
    ys = [orc.draw(z, q, (i + 0.5) / 64)[0] for i in range(64)]
    assert [ys.count(j) for j in range(4)] == [32, 8, 16, 8]
    assert ys == sorted(ys)
    assert orc.draw(z, q, 0.0)[0] == 0 and orc.draw(z, q, 1 - 2.0 ** -24)[0] == 3


def test_weights_are_the_softmax():
    z = RNG(1).normal(size=500).astype(np.float32) * 3
    for temp in (0.5, 1.0, 2.0):
        q = _q(z, temp).astype(np.float64)
        p = np.exp((z.astype(np.float64) - z.max()) / temp)
        assert np.abs(q / q.sum() - p / p.sum()).max() < 500 * 2.0 ** -28


@pytest.mark.parametrize("k", [1, 2, 3, 10])
def test_top_k_keeps_the_first_of_equals(k):
    z = np.array([1, 3, 3, 2, 3, -np.inf], np.float32)
    kept = orc.kept_tokens(z, _q(z), top_k=k)
    assert sorted(np.flatnonzero(kept)) == sorted([1, 2, 4, 3, 0][:k])


def test_top_p_is_the_shortest_part_that_reaches_it():
    z = np.log(np.array([1, 5, 2, 2], np.float32) / 5)
    q = np.array([1, 5, 2, 2]) * (orc.ONE // 5)
    want = {0.2: [1], 0.499: [1], 0.55: [1, 2], 0.7: [1, 2], 0.85: [1, 2, 3], 0.95: [0, 1, 2, 3],
            1.0: [0, 1, 2, 3]}
    for p, ids in want.items():
        assert list(np.flatnonzero(orc.kept_tokens(z, q, top_p=p))) == ids, p
    # of the tokens that top-k leaves: 5 of 7 shares are more than 0.7
    assert list(np.flatnonzero(orc.kept_tokens(z, q, top_k=2, top_p=0.7))) == [1]


def test_min_p_is_relative_to_the_largest():
    z = np.log(np.array([8, 4, 2, 1], np.float32))
    q = np.array([8, 4, 2, 1]) * (orc.ONE // 8)
    for p, n in ((0.0, 4), (0.125, 4), (0.13, 3), (0.5, 2), (0.51, 1), (1.0, 1)):
        assert orc.kept_tokens(z, q, min_p=p).sum() == n


def test_greedy_is_the_lowest_of_the_largest():
    z = np.array([0, 7, 7, 1], np.float32)
    assert orc.draw_exponents(z, 0.0) is None and orc.draw_exponents(z, 1e-45) is None
    assert orc.draw(z, _q(z), 0.99, greedy=True) == (1, 0.0)


def test_top_list_and_tail_hold_the_softmax():
    z = RNG(2).normal(size=300).astype(np.float32) * 2
    z[::7] = -np.inf
    for K in (1, 5, 299, 400):
        t = orc.top_list(z, K, 2.0)
        n = (t.ids >= 0).sum()
        assert (np.diff(t.values[:n]) <= 0).all() and np.array_equal(z[t.ids[:n]], t.values[:n])
        whole = np.exp(t.values[:n] / 2.0).sum() + math.exp(t.tail)
        assert abs(whole / np.exp(z.astype(np.float64) / 2.0).sum() - 1) < 1e-12


def _case(seed, V=40, K=6, temp=1.3):
    r = RNG(seed)
    teacher, z = r.normal(size=V) * 2, r.normal(size=V) * 2
    t = orc.top_list(teacher, K, temp)
    return z, t


@pytest.mark.parametrize("reverse,with_tail", [(False, True), (False, False), (True, True)])
def test_distill_gradient_is_the_difference_quotient(reverse, with_tail):
    for seed in range(3):
        z, t = _case(seed)
        kw = dict(reverse=reverse, temperature=1.3, weight=0.7, scale=2.5)
        tail = t.tail if with_tail else None
        out = orc.distill_row(z, t.ids, t.values, tail, **kw)
        for j in range(z.size):
            h = 1e-5
            up, dn = z.copy(), z.copy()
            up[j] += h
            dn[j] -= h
            d = (orc.distill_row(up, t.ids, t.values, tail, **kw).term
                 - orc.distill_row(dn, t.ids, t.values, tail, **kw).term) / (2 * h)
            assert abs(d - out.grad[j]) < 1e-8
        assert abs(out.grad.sum()) < 1e-12   # a softmax does not see a common shift


def test_distill_of_a_teacher_against_itself_is_zero():
    r = RNG(5)
    z = r.normal(size=64) * 3
    t = orc.top_list(z, 8, 2.0)
    for reverse in (False, True):
        out = orc.distill_row(z, t.ids, t.values, t.tail, reverse=reverse, temperature=2.0)
        assert abs(out.term) < 1e-14 and np.abs(out.grad).max() < 1e-14


def test_distill_is_the_full_kl_when_everything_is_listed():
    r = RNG(6)
    z, teacher = r.normal(size=20), r.normal(size=20)
    t = orc.top_list(teacher, 20)
    p, q = np.exp(z) / np.exp(z).sum(), np.exp(teacher) / np.exp(teacher).sum()
    got = orc.distill_row(z, t.ids, t.values, t.tail)
    assert t.tail == -math.inf and abs(got.term - (q * np.log(q / p)).sum()) < 1e-13
    assert np.abs(got.grad - (p - q)).max() < 1e-14


def test_distill_rows_that_do_not_count():
    z, t = _case(9)
    base = (z, t.ids, t.values, t.tail)
    assert not orc.distill_row(*base, on=False).valid
    for ids in ([40, 1, 2, 3, 4, 5], [-2, 1, 2, 3, 4, 5], [3, 1, 2, 3, 4, 5]):
        out = orc.distill_row(z, np.array(ids), t.values, t.tail)
        assert not out.valid and out.bad and not out.grad.any()
    out = orc.distill_row(z, np.full(6, -1), t.values, t.tail)
    assert not out.valid and not out.bad
    out = orc.distill_row(*base, weight=0.0)
    assert out.valid and out.term == 0.0 and not out.grad.any()


MUTANTS = {
    "tail ignored": lambda z, t, kw: orc.distill_row(z, t.ids, t.values, None, **kw),
    "temperature on one side": lambda z, t, kw: orc.distill_row(
        z, t.ids, t.values, t.tail, **dict(kw, temperature=1.0)),
    "directions swapped": lambda z, t, kw: orc.distill_row(
        z, t.ids, t.values, t.tail, **dict(kw, reverse=not kw["reverse"])),
    "weight dropped": lambda z, t, kw: orc.distill_row(
        z, t.ids, t.values, t.tail, **dict(kw, weight=1.0)),
}


@pytest.mark.parametrize("name", sorted(MUTANTS))
def test_planted_mistakes_move_the_loss(name):
    z, t = _case(11)
    for reverse in (False, True):
        kw = dict(reverse=reverse, temperature=1.3, weight=0.7, scale=2.5)
        right = orc.distill_row(z, t.ids, t.values, t.tail, **kw)
        wrong = MUTANTS[name](z, t, kw)
        # (a teacher without its tail makes the reverse KL infinite)
        assert not abs(wrong.term - right.term) <= 1e-3 * abs(right.term)
        assert not np.abs(wrong.grad - right.grad).max() <= 1e-3 * np.abs(right.grad).max()
