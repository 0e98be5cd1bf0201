"""The sampling oracle pinned: cuts worked out by hand, draws against the definition of the inverse cdf, the gradient
against differences."""
import numpy as np
import pytest

from oracle import sampling as so

Z = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))


@pytest.mark.parametrize("settings,want", [
    (dict(), [0, 1, 2, 3, 4]),
    (dict(tau=0.0), [1]),
    (dict(top_k=2), [1, 3]),
    (dict(top_k=4), [0, 1, 3, 4]),             # of the two words of 0.1, the lower index
    (dict(top_k=9), [0, 1, 2, 3, 4]),
    (dict(top_p=0.0), [1]),
    (dict(top_p=0.39), [1]),
    (dict(top_p=0.5), [1, 3]),
    (dict(top_p=0.85), [0, 1, 3, 4]),
    (dict(top_k=2, top_p=0.6), [1]),           # 0.4 of 0.65 is 0.615
    (dict(top_k=2, top_p=0.62), [1, 3]),
    (dict(min_p=0.3), [1, 3, 4]),
    (dict(min_p=1.0), [1]),
    (dict(top_k=2, min_p=0.3), [1, 3]),
    (dict(tau=0.5, top_p=0.61), [1, 3]),       # weights 0.16, 0.0625, 0.0225, 0.01, 0.01 of 0.265: 0.604 first
    (dict(tau=0.5, top_p=0.60), [1]),
])
def test_cuts(settings, want):
    assert so.kept(Z, **settings)[0].tolist() == want


def test_masked_words_and_empty_rows():
    z = np.array([-np.inf, 0.0, -1e8, -1e9, 0.0])
    assert so.kept(z)[0].tolist() == [1, 4]
    assert so.kept(z, top_k=1)[0].tolist() == [1]
    assert so.kept(z, tau=0.0)[0].tolist() == [1]
    assert so.draw(np.full(3, -np.inf), 0.5) == (-1, -np.inf, 0)


@pytest.mark.parametrize("u,want", [(0.0, 0), (0.0999, 0), (0.1001, 1), (0.4999, 1), (0.5001, 2), (0.9999, 4)])
def test_draw_is_the_inverse_cdf_in_the_order_of_the_indices(u, want):
    a, lp, n = so.draw(Z, u)
    assert a == want and n == 5 and abs(lp - Z[want]) < 1e-15


def test_draw_within_a_cut():
    a, lp, n = so.draw(Z, 0.7, top_k=2)  # 1: 0.615, 3: 0.385
    assert (a, n) == (3, 2) and abs(lp - np.log(0.25 / 0.65)) < 1e-15


@pytest.mark.parametrize("settings", [dict(), dict(tau=0.7), dict(tau=1.3, top_k=3), dict(top_p=0.7), dict(min_p=0.3)])
def test_gradient_against_differences(settings):
    lp, n, d = so.logp(Z, 3, **settings)
    h = 1e-6
    for i in range(Z.size):
        e = np.zeros(Z.size)
        e[i] = h
        num = (so.logp(Z + e, 3, **settings)[0] - so.logp(Z - e, 3, **settings)[0]) / (2 * h)
        assert abs(num - d[i]) < 1e-9
    assert so.logp(Z, 0, top_k=2)[0] == -np.inf and not so.logp(Z, 0, top_k=2)[2].any()
