"""Pins of the oracle of the routing by scores and of the orthogonal update (CPU only)."""
import numpy as np
import pytest

from oracle import router_oracle as ro


def test_worked_examples():
    # sigmoid(0) = 1/2, sigmoid(ln 3) = 3/4, sigmoid(-ln 3) = 1/4
    l = np.array([[0.0, np.log(3.0), -np.log(3.0), 0.0]])
    np.testing.assert_allclose(ro.scores(l, "sigmoid"), [[0.5, 0.75, 0.25, 0.5]], rtol=1e-15)
    idx, s = ro.select(l, "sigmoid", 3)
    assert idx.tolist() == [[1, 0, 3]]                              # the tie goes to the lower expert
    np.testing.assert_allclose(ro.weights(s, idx, True, 3.5), [[1.5, 1.0, 1.0]], rtol=1e-15)
    # a bias decides the selection, not the weights
    idx, s = ro.select(l, "sigmoid", 2, bias=[0.0, -1.0, 1.0, 0.1])
    assert idx.tolist() == [[2, 3]]
    np.testing.assert_allclose(ro.weights(s, idx, False, 2.0), [[0.5, 1.0]], rtol=1e-15)
    # groups (0, 1) and (2, 3): 1/2 + 3/4 against 1/4 + 1/2
    assert ro.select(l, "sigmoid", 2, n_group=2, topk_group=1)[0].tolist() == [[1, 0]]
    # groups of one: their only key
    assert ro.select(l, "sigmoid", 2, n_group=4, topk_group=2)[0].tolist() == [[1, 0]]
    # softmax of ln 1, ln 3, ln 4
    l = np.log([[1.0, 3.0, 4.0]])
    idx, s = ro.select(l, "softmax", 2)
    assert idx.tolist() == [[2, 1]]
    np.testing.assert_allclose(ro.weights(s, idx, False, 1.0), [[0.5, 0.375]], rtol=1e-15)


def test_rows_with_holes():
    inf, nan = np.inf, np.nan
    l = np.array([[-inf, 1.0, nan, 0.0], [-inf] * 4, [inf, inf, 0.0, -inf]])
    for kind in ("sigmoid", "softmax"):
        idx, s = ro.select(l, kind, 3, bias=[5.0, 0.0, 0.0, 0.0])
        assert idx[0].tolist() == [1, 3, 0] and idx[1].tolist() == [0, 1, 2]
        w = ro.weights(s, idx, True, 1.0)
        assert w[0, 2] == 0 and (w[1] == 0).all() and np.isfinite(w).all()
        np.testing.assert_allclose(w[0].sum(), 1.0)
    assert ro.scores(l, "softmax")[2].tolist() == [0.5, 0.5, 0.0, 0.0]
    # one living expert to a group counts by itself: -0.2 + nothing against -0.1 - 0.2
    l = np.zeros((1, 4))
    l[0, 1] = -inf
    assert ro.select(l, "sigmoid", 1, bias=[-0.7, 0.0, -0.6, -0.7], n_group=2)[0].tolist() == [[0]]


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_is_that_of_the_weights(kind, renormalize):
    r = np.random.default_rng(3)
    l = r.normal(size=(5, 12))
    idx, _ = ro.select(l, kind, 4, bias=0.3 * r.normal(size=12))
    dw = r.normal(size=(5, 4))
    got = ro.weights_backward(l, kind, idx, dw, renormalize, 1.75)
    h = 1e-6
    for t in range(5):
        for e in range(12):
            d = np.zeros_like(l)
            d[t, e] = h
            up, down = (ro.weights(ro.scores(l + s * d, kind), idx, renormalize, 1.75) for s in (1, -1))
            assert abs(((up - down) * dw).sum() / (2 * h) - got[t, e]) < 1e-8


def test_bias_step():
    assert ro.bias_step([0.0, 1.0, 2.0], [4, 2, 3], 0.5).tolist() == [-0.5, 1.5, 2.0]
    big = 2 ** 31 - 1                                              # a mean that no fp32 can tell from its neighbours
    assert ro.bias_step([0.0, 0.0], [big, big - 1], 1.0).tolist() == [-1.0, 1.0]


@pytest.mark.parametrize("M,N", [(6, 9), (9, 6), (7, 7), (1, 5)])
def test_orthogonalize_takes_singular_values_through_the_polynomial(M, N):
    r = np.random.default_rng(M + N)
    u = r.normal(size=(M, N))
    got = ro.orthogonalize(u, steps=3, coefs=[(3.0, -3.2, 1.2), ro.USUAL, (2.0, -1.5, 0.5)], eps=1e-9)
    U, s, V = np.linalg.svd(u, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-9)
    for a, b, c in ((3.0, -3.2, 1.2), ro.USUAL, (2.0, -1.5, 0.5)):
        s = a * s + b * s ** 3 + c * s ** 5
    np.testing.assert_allclose(got, (U * s) @ V, atol=1e-12)


def test_muon_step():
    g, m, w = (np.random.default_rng(i).normal(size=(4, 3)) for i in range(3))
    m1, w1 = ro.muon_step(g, m, w, 0.1, 0.9, False, 0.5, 2.0, steps=2)
    np.testing.assert_allclose(m1, 0.9 * m + g)
    np.testing.assert_allclose(w1, 0.95 * w - 0.2 * ro.orthogonalize(m1, steps=2))
    _, w2 = ro.muon_step(g, m, w, 0.1, 0.9, True, 0.0, 1.0)
    np.testing.assert_allclose(w2, w - 0.1 * ro.orthogonalize(g + 0.9 * m1))
