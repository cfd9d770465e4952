"""Pins of the float64 oracle of routing, 8-bit rows and sampling: hand-worked cases, closed forms and properties."""
import numpy as np
import pytest

from oracle import experts as X


def test_route_hand_worked():
    # sigmoid scores 0.5, 0.7310585, 0.2689414, 0.8807971; the bias turns the order round, the weights are without it
    l = np.array([[0.0, 1.0, -1.0, 2.0]])
    ids, w = X.route(l, 2, score="sigmoid")
    assert ids.tolist() == [[3, 1]] and np.allclose(w, [[0.8807970779778823, 0.7310585786300049]], rtol=1e-15)
    ids, w = X.route(l, 2, bias=[1.0, 0.0, 1.0, 0.0], score="sigmoid", renorm=True, scale=2.0)
    assert ids.tolist() == [[0, 2]]                               # 1.5 and 1.2689 against 0.88 and 0.73
    assert np.allclose(w, [[2 * 0.5 / 0.7689414213699951, 2 * 0.2689414213699951 / 0.7689414213699951]], rtol=1e-14)
    ids, w = X.route(np.log([[1.0, 2.0, 3.0, 4.0]]), 3)           # softmax of logarithms: tenths
    assert ids.tolist() == [[3, 2, 1]] and np.allclose(w, [[0.4, 0.3, 0.2]], rtol=1e-14)


def test_route_groups_hand_worked():
    # groups (9 1)(5 5)(8 0): by the best (9, 5, 8) groups 0 and 2 take part, by the sum of two (10, 10, 8) groups 0 and 1
    l = np.log([[9.0, 1.0, 5.0, 5.0, 8.0, 0.5]])
    assert X.route(l, 3, n_groups=3, top_groups=2, group_top=1)[0].tolist() == [[0, 4, 1]]
    ids, _ = X.route(np.array([[9.0, 1.0, 5.0, 5.0, 8.0, 0.5]]), 3, score="softmax", n_groups=3, top_groups=2, group_top=1)
    assert ids.tolist() == [[0, 4, 1]]
    assert X.route(l, 3, n_groups=3, top_groups=2, group_top=2)[0].tolist() == [[0, 2, 3]]
    assert X.route(l, 4, n_groups=3, top_groups=2, group_top=2)[0].tolist() == [[0, 2, 3, 1]]


def test_route_masks_and_ties():
    inf = np.inf
    ids, w = X.route(np.array([[-inf, -inf, -inf], [0.0, -inf, 0.0], [1.0, 1.0, 1.0], [np.nan, 0.0, 0.0]]), 2, score="sigmoid", renorm=True)
    assert ids.tolist() == [[-1, -1], [0, 2], [0, 1], [-1, -1]]
    assert w[0].tolist() == [0.0, 0.0] and np.isnan(w[3]).all()
    ids, w = X.route(np.array([[0.0, 5.0, 1.0]]), 3, bias=[0.0, -inf, 0.0])
    assert ids.tolist() == [[2, 0, -1]] and w[0, 2] == 0.0


def test_group_hand_worked():
    off, rows = X.group(np.array([[2, 0], [0, 3], [-1, 2], [7, 0]]), 4, keep=[3, 3, 3, 1])
    assert off.tolist() == [0, 2, 2, 4, 5] and rows.tolist() == [1, 2, 0, 5, 3, -1, -1, -1]   # the last token's slot 1 is dropped


def test_group_is_a_permutation_of_what_stays():
    rng = np.random.default_rng(0)
    ids = rng.integers(-1, 9, size=(200, 5))
    off, rows = X.group(ids, 8)
    flat = ids.reshape(-1)
    listed = rows[:off[-1]]
    assert sorted(listed.tolist()) == np.nonzero((flat >= 0) & (flat < 8))[0].tolist()
    for e in range(8):
        mine = rows[off[e]:off[e + 1]]
        assert (flat[mine] == e).all() and (np.diff(mine) > 0).all()


def test_quant8_ties_and_marked_rows():
    # scale 1: halves go to the even code
    codes, s = X.quant8(np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 3.49, 126.5]]))
    assert s.tolist() == [1.0] and codes.tolist() == [[127, 0, 2, 2, 0, -2, 3, 126]]
    codes, s = X.quant8(np.array([[0.0, 0.0], [np.inf, 1.0], [np.nan, 1.0]]))
    assert s[0] == 0.0 and np.isnan(s[1:]).all() and (codes == 0).all()
    # a value that 64-bit division puts on the middle and exact arithmetic beside it would be decided by the fraction
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64)).astype(np.float32).astype(np.float64)
    codes, s = X.quant8(x)
    assert (np.abs(codes * s[:, None] - x) <= 0.5000001 * s[:, None]).all() and (np.abs(codes).max(axis=1) == 127).all()


def test_matmul8_is_the_product_of_the_rows_it_stands_for():
    rng = np.random.default_rng(2)
    w, x = rng.standard_normal((7, 33)), rng.standard_normal((5, 33))
    wc, ws = X.quant8(w)
    xc, xs = X.quant8(x)
    assert np.allclose(X.matmul8(wc, ws, xc, xs), (xc * xs[:, None]) @ (wc * ws[:, None]).T, rtol=1e-13)
    assert X.matmul8(np.full((1, 131072), 127), np.ones(1), np.full((1, 131072), -127), np.ones(1))[0, 0] == -127.0 ** 2 * 131072


def test_sample_hand_worked():
    l = np.log([4.0, 1.0, 3.0, 2.0])                    # tenths 4 1 3 2
    assert [X.sample(l, u)[0] for u in (0.0, 0.39, 0.41, 0.49, 0.51, 0.79, 0.81, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert X.kept(l, top_k=2)[0].tolist() == [0, 2]
    assert X.kept(l, top_p=0.65)[0].tolist() == [0, 2]   # 4 in front of the 3, 7 in front of the 2
    assert X.kept(l, top_p=0.75)[0].tolist() == [0, 2, 3]
    assert X.kept(l, min_p=0.4)[0].tolist() == [0, 2, 3]  # at least 1.6
    assert X.kept(l, top_k=3, top_p=0.75)[0].tolist() == [0, 2]   # three quarters of 9 is 6.75: 7 is in front of the 2
    token, p = X.sample(l, 0.9, top_k=2)
    assert token == 2 and abs(p - 3 / 7) < 1e-15
    assert X.sample(l, 0.9, temperature=0.0) == (0, 1.0)
    assert abs(X.sample(l, 0.0, temperature=0.5)[1] - 16 / 30) < 1e-14


def test_sample_masks():
    inf = np.inf
    assert X.sample([-inf, -inf], 0.3)[0] == -1 and X.sample([0.0, np.nan], 0.3)[0] == -1
    assert X.sample([0.0, inf, 1.0, inf], 0.4)[0] == 1 and X.sample([0.0, inf, 1.0, inf], 0.6)[0] == 3
    assert X.sample([-inf, 2.0, -inf], 0.999)[0] == 1


@pytest.mark.parametrize("kw", [{}, dict(top_k=5), dict(top_p=0.7), dict(min_p=0.2), dict(top_k=6, top_p=0.9, min_p=0.05, temperature=0.6)])
def test_sample_frequencies_are_the_probabilities(kw):
    """Evenly spread numbers draw a token as often as its probability says, to within one draw."""
    rng = np.random.default_rng(3)
    l = rng.standard_normal(12)
    stay, p = X.kept(l, **kw)
    p = p / p.sum()
    n = 2000
    count = np.bincount([X.sample(l, (i + 0.5) / n, **kw)[0] for i in range(n)], minlength=12)
    assert set(np.nonzero(count)[0]) <= set(stay) and (np.abs(count[stay] - n * p) <= 1.0 + 1e-9).all()
