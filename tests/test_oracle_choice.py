"""Pins of the row-wise choices' oracle against things other than itself: the exponential, counted
probabilities, brute-force filters, closed forms and differences."""
import math

import numpy as np
import pytest

from oracle import choice_oracle as C


def test_weights_are_the_exponential_within_their_stated_error():
    x = np.linspace(-27.7, 0, 40001).astype(np.float32)  # t from -40 to 0
    w = C.fixed_weights(x, C.LOG2E)
    assert w[-1] == 2**40  # the maximum, exactly
    real = np.exp(x.astype(np.float64)) * 2.0**40
    # 2^t: the polynomial (1.9e-7); the constant log2(e) and the product's rounding move t by
    # |t| (2^-25 + 2^-24), t = x log2(e); half a unit of the integer
    bound = real * (1.9e-7 + np.abs(x) * (2.0**-24 + 2.0**-25)) + 0.5
    assert np.all(np.abs(w - real) <= bound)


def test_weights_vanish_far_below_the_maximum_and_where_masked():
    assert C.fixed_weights(np.array([0, -28.5, -29, -1e30, -np.inf], np.float32), C.LOG2E)[2:].tolist() == [0, 0, 0]
    assert C.fixed_weights(C.clean([np.nan, -np.inf]), C.LOG2E).tolist() == [0, 0]
    assert C.fixed_weights(C.clean([np.inf, 3.0, np.inf]), C.LOG2E).tolist() == [2**40, 0, 2**40]
    low = np.finfo(np.float32).min
    assert C.fixed_weights(C.clean([low, low]), C.LOG2E).tolist() == [2**40, 2**40]


def test_every_entry_owns_a_share_of_the_words_that_is_its_probability():
    x = np.random.default_rng(1).normal(size=12).astype(np.float32)
    q = C.sample_probs(x, 0.7, np.arange(12))
    edge = 0.0
    for i in range(12):  # just inside both ends of entry i's interval of words
        for u in (edge + 1e-6, edge + q[i] - 1e-6):
            got, logp, _ = C.sample_row(x, int(u * 2.0**64), 0.7)
            assert got == i
            assert abs(logp - math.log(q[i])) < 1e-6
        edge += q[i]


@pytest.mark.parametrize("k,p,mp", [(3, 1.0, 0.0), (0, 0.6, 0.0), (0, 1.0, 0.2), (5, 0.8, 0.05), (1, 0.1, 1.0)])
def test_filters_keep_what_the_textbook_keeps(k, p, mp):
    rng = np.random.default_rng(7)
    for _ in range(20):
        x = rng.normal(size=30, scale=2).astype(np.float32)
        q = C.sample_probs(x, 1.0, np.arange(30))
        by = np.argsort(-q, kind="stable")
        by = by[q[by] >= mp * q.max() * (1 - 1e-6)]
        if k:
            by = by[:k]
        mass = np.cumsum(q[by]) / q[by].sum()
        if np.min(np.abs(mass - p)) < 1e-5:
            continue
        if p < 1:
            by = by[: int(np.searchsorted(mass, p)) + 1]
        assert C.sample_row(x, 5, 1.0, k, p, mp)[2] == sorted(by.tolist())


def test_ties_go_to_the_lowest_index_and_greedy_takes_the_first_best():
    x = np.array([1, 2, 2, -0.0, 0.0, 2], np.float32)
    assert C.sample_row(x, 3, 1.0, 2)[2] == [1, 2]
    assert C.sample_row(x, 2**63, 0.0)[:2] == (1, 0.0)
    assert C.sample_row(np.array([-0.0, 0.0], np.float32), 2**64 - 1, 1.0, 1)[0] == 0
    assert C.sample_row(np.full(4, -np.inf, np.float32), 9) == (-1, -math.inf, [])


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_scores_are_the_function_within_rounding(kind):
    x = np.random.default_rng(3).normal(size=(20, 33), scale=3).astype(np.float32)
    s, _ = C.route_scores(x, kind)
    real = C.scores64(x, kind)
    # |t| <= 40 here: t's rounding moves 2^t by 40 (2^-24 + 2^-24 + 2^-25) ln 2, the rest by < 1e-6
    assert np.all(np.abs(s - real) <= real * 6e-6 + 2.0**-40)


def test_route_by_hand():
    x = np.log(np.array([[1.0, 4.0, 2.0, 3.0]])).astype(np.float32)
    e, w = C.route(x, 2, "softmax", renorm=False)
    assert e.tolist() == [[1, 3]]
    np.testing.assert_allclose(w, [[0.4, 0.3]], rtol=1e-6)
    e, w = C.route(x, 2, "softmax", bias=[1, 0, 0, 0], renorm=True, scale=2.0)
    assert e.tolist() == [[0, 1]]
    np.testing.assert_allclose(w, [[0.4, 1.6]], rtol=1e-6)
    # groups {0, 1} and {2, 3}: sums 5 and 5 of 10 tie in exact arithmetic; by the best alone the first wins
    e, _ = C.route(x, 2, "softmax", groups=2, top_groups=1, group_best=1)
    assert e.tolist() == [[1, 0]]
    e, w = C.route(np.full((1, 4), -np.inf, np.float32), 3, "sigmoid")
    assert e.tolist() == [[-1, -1, -1]] and not w.any()


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_gradient_against_differences(kind, renorm):
    rng = np.random.default_rng(11)
    x = rng.normal(size=(4, 9))
    e, _ = C.route(x, 3, kind, renorm=renorm)
    e[1, 2] = -1
    g = rng.normal(size=e.shape)
    got = C.route_gradient(x.astype(np.float32), e, g, kind, renorm, 1.7)
    x = x.astype(np.float32).astype(np.float64)
    h = 2.0**-7
    for i in range(9):
        up, down = x.copy(), x.copy()
        up[:, i] += h
        down[:, i] -= h  # scores64 rounds to float32: h and x are kept representable
        up, down = up.astype(np.float32), down.astype(np.float32)
        step = up[:, i].astype(np.float64) - down[:, i]
        d = ((C.weights64(up, e, kind, renorm, 1.7) - C.weights64(down, e, kind, renorm, 1.7)) * g).sum(1) / step
        # the central difference's own error: h^2/6 times a third derivative of order sum|g| 1.7 / D^3
        assert np.max(np.abs(d - got[:, i])) < 2e-3


def test_plan_and_combine_by_hand():
    offsets, order, slot = C.plan(np.array([[2, 0], [-1, 2], [0, 7]]), 3)
    assert offsets.tolist() == [0, 2, 2, 4]
    assert order.tolist() == [1, 4, 0, 3, -1, -1]
    assert slot.tolist() == [[2, 0], [-1, 3], [1, -1]]
    y = np.arange(12.0).reshape(6, 2)
    w = np.array([[0.5, 2.0], [9.0, 1.0], [3.0, 9.0]])
    out = C.combine(y, slot, w)
    assert out.tolist() == [[2.0, 4.5], [6.0, 7.0], [6.0, 9.0]]
    dout = np.ones((3, 2))
    dy, dw = C.combine_gradient(dout, y, slot, w)
    h = 1e-3
    for s in range(6):  # linear in y and in w: differences are exact up to rounding
        up = y.copy()
        up[s, 1] += h
        assert abs((C.combine(up, slot, w) - out).sum() / h - dy[s, 1]) < 1e-9
    for t, j in np.ndindex(slot.shape):
        up = w.copy()
        up[t, j] += h
        assert abs((C.combine(y, slot, up) - out).sum() / h - dw[t, j]) < 1e-9
