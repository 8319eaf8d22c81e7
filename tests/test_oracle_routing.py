"""Pins of the oracle of the routing operators: distributions enumerated by hand, gradients against differences."""
import math

import numpy as np
import pytest

from oracle import routing as R
from oracle.train import mixture_logp


def test_route_weights_and_density():
    rng = np.random.default_rng(0)
    t, a = rng.normal(0, 3, (7, 20)), np.log(rng.dirichlet(np.ones(7)))
    ids, w, logp, p = R.route(t, a, 3)
    np.testing.assert_allclose(logp, mixture_logp(t, a), rtol=1e-13)
    np.testing.assert_allclose(p.sum(0), 1.0, rtol=1e-13)
    assert (np.diff(w, axis=1) <= 0).all()
    np.testing.assert_allclose(w, np.sort(p, axis=0)[::-1][:3].T, rtol=1e-13)
    np.testing.assert_allclose(R.route(t, a, 3, True)[1].sum(1), 1.0, rtol=1e-13)


def test_route_ties_and_closed_components():
    ids, w, logp, _ = R.route(np.array([[0.0], [np.nan], [0.0], [-np.inf]]), None, 3)
    assert ids.tolist() == [[0, 2, -1]] and w.tolist() == [[0.5, 0.5, 0.0]]
    assert logp[0] == pytest.approx(math.log(2))
    ids, w, logp, _ = R.route(np.full((3, 1), -np.inf), None, 2, True)
    assert ids.tolist() == [[-1, -1]] and w.tolist() == [[0.0, 0.0]] and logp[0] == -np.inf
    ids, w, logp, _ = R.route(np.array([[1.0], [np.inf], [np.inf]]), None, 2)
    assert ids.tolist() == [[1, 2]] and w.tolist() == [[0.5, 0.5]] and logp[0] == np.inf


@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient_against_differences(renormalise):
    rng = np.random.default_rng(1)
    M, N, top = 5, 4, 2
    t, a = rng.normal(0, 1, (M, N)), rng.normal(0, 1, M)
    dw, dl = rng.normal(size=(N, top)), rng.normal(size=N)
    ids = R.route(t, a, top, renormalise)[0]

    def value(t, a):
        _, w, logp, _ = R.route(t, a, top, renormalise)
        return (w * dw).sum() + (logp * dl).sum()

    g, ga = R.route_backward(t, a, ids, dw, dl, renormalise)
    h = 1e-6
    for c in range(M):
        for n in range(N):
            e = np.zeros((M, N))
            e[c, n] = h
            assert (value(t + e, a) - value(t - e, a)) / (2 * h) == pytest.approx(g[c, n], abs=1e-8)
        e = np.zeros(M)
        e[c] = h
        assert (value(t, a + e) - value(t, a - e)) / (2 * h) == pytest.approx(ga[c], abs=1e-8)


def test_exchange_and_its_gradient():
    ids = np.array([[2, 0], [2, -1], [0, 5], [1, 2]], np.int32)
    first, place = R.sort(ids, 3)
    assert first.tolist() == [0, 2, 3, 6] and place.tolist() == [[3, 0], [4, -1], [1, -1], [2, 5]]
    rng = np.random.default_rng(2)
    x, w = rng.normal(size=(4, 3)), rng.random((4, 2))
    xs = R.dispatch(x, place, np.full((8, 3), 7.0))
    assert (xs[6:] == 7.0).all() and (xs[5] == x[3]).all() and (xs[0] == x[0]).all()
    rows, dy = rng.normal(size=(8, 3)), rng.normal(size=(4, 3))
    drows, dw = R.combine_backward(dy, rows, place, w, np.zeros((8, 3)))
    h = 1e-6
    for i in np.ndindex(8, 3):
        e = np.zeros((8, 3))
        e[i] = h
        d = ((R.combine(rows + e, place, w) - R.combine(rows - e, place, w)) * dy).sum() / (2 * h)
        assert d == pytest.approx(drows[i], abs=1e-8)
    for i in np.ndindex(4, 2):
        e = np.zeros((4, 2))
        e[i] = h
        assert ((R.combine(rows, place, w + e) - R.combine(rows, place, w - e)) * dy).sum() / (2 * h) == pytest.approx(dw[i], abs=1e-8)
    # carrying rows out and adding them up again: every row as often as it has slots
    np.testing.assert_allclose(R.combine(xs, place), x * (place >= 0).sum(1)[:, None])


def test_choice_follows_the_kept_distribution():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    assert R.kept(x) == pytest.approx({0: 0.25, 1: 1.0, 2: 0.5, 3: 0.75})
    assert set(R.kept(x, top_k=2)) == {1, 3}
    assert set(R.kept(x, top_p=0.4)) == {1} or set(R.kept(x, top_p=0.4)) == {1, 3}   # (0.4 is a border)
    assert set(R.kept(x, top_p=0.5)) == {1, 3}
    assert set(R.kept(x, top_p=0.75)) == {1, 2, 3}
    assert set(R.kept(x, top_k=3, top_p=0.75)) == {1, 3}          # 0.4 + 0.3 of 0.9 is above three quarters
    assert set(R.kept(x, min_p=0.6)) == {1, 3}
    assert set(R.kept(x, temperature=0)) == {1}
    assert set(R.kept(x, top_p=0.0)) == {1}
    edges = np.cumsum([0.1, 0.4, 0.2, 0.3])
    for u in np.linspace(0.01, 0.99, 50):
        assert R.choose(x, u)[0] == int(np.searchsorted(edges, u))
    assert R.choose(x, 0.2)[1] == pytest.approx(math.log(0.4))
    assert R.choose([-np.inf, np.nan], 0.3) == (-1, -np.inf)
    assert R.choose([0.0, 0.0, 0.0, 0.0], 0.5) == (2, pytest.approx(math.log(0.25)))
    assert R.choose([0.0, 0.0, 0.0, 0.0], 0.5, top_k=2) == (1, pytest.approx(math.log(0.5)))
    assert R.choose([3.0, np.inf, 1.0, np.inf], 0.7) == (3, pytest.approx(math.log(0.5)))
