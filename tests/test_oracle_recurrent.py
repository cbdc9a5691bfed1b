"""The oracle of the recurrent block: the recurrence against its closed form and
finite differences, the group norm against finite differences and known
moments, the orthogonalised update against the singular values that the
iteration's polynomial gives."""
import numpy as np
import pytest

from oracle import recurrent as rec


def normal(seed, *shape):
    return np.random.default_rng(seed).normal(size=shape)


def slope(f, x, v, h=1e-6):
    """Central difference of the number f along v at x."""
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


def test_recurrence_is_the_weighted_sum_of_its_inputs():
    b, t, w = 2, 7, 3
    x, r, i = (normal(s, b, t, w) for s in (1, 2, 3))
    decay, state = normal(4, w), normal(5, b, w)
    h, last = rec.recur_fwd(x, r, i, decay, 8.0, state=state)
    L = np.cumsum(-8.0 * np.log1p(np.exp(decay)) / (1 + np.exp(-r)), 1)
    a = np.exp(np.diff(L, axis=1, prepend=0))
    u = np.sqrt(1 - a * a) / (1 + np.exp(-i)) * x
    for k in range(t):
        want = np.exp(L[:, k]) * state + sum(np.exp(L[:, k] - L[:, j]) * u[:, j] for j in range(k + 1))
        assert np.allclose(h[:, k], want, rtol=1e-12)
    assert np.array_equal(last, h[:, -1])


def test_recurrence_keeps_a_unit_variance():
    # a^2 + (1 - a^2) = 1: white inputs with open gates give white states
    x, r, i = normal(6, 1, 300, 1), np.zeros((1, 300, 1)), np.full((1, 300, 1), 50.0)
    a = np.exp(-8 * np.log(2) / 2)
    h, _ = rec.recur_fwd(x, r, i, np.zeros(1), 8.0)
    assert np.allclose(h[0, 1:, 0], a * h[0, :-1, 0] + np.sqrt(1 - a * a) * x[0, 1:, 0])


def test_recurrence_lengths():
    x, r, i = (normal(s, 3, 5, 2) for s in (1, 2, 3))
    state = normal(4, 3, 2)
    h, last = rec.recur_fwd(x, r, i, np.zeros(2), 4.0, lens=[0, 3, 9], state=state)
    assert not h[0].any() and np.array_equal(last[0], state[0]) and not h[1, 3:].any()
    assert np.array_equal(last[1], h[1, 2]) and np.array_equal(last[2], h[2, 4])


def test_recurrence_backward_by_differences():
    b, t, w, rate = 2, 6, 3, 3.0
    x, r, i, dh = (normal(s, b, t, w) for s in (1, 2, 3, 4))
    decay, state, ds = normal(5, w), normal(6, b, w), normal(7, b, w)
    lens = [6, 4]

    def loss(x=x, r=r, i=i, decay=decay, state=state):
        h, last = rec.recur_fwd(x, r, i, decay, rate, lens, state)
        return (h * dh).sum() + (last * ds).sum()

    h, _ = rec.recur_fwd(x, r, i, decay, rate, lens, state)
    got = dict(zip(("x", "r", "i", "decay", "state"), rec.recur_bwd(x, r, i, decay, rate, h, dh, lens, state, ds)))
    for name, at in (("x", x), ("r", r), ("i", i), ("decay", decay), ("state", state)):
        v = normal(9, *at.shape)
        assert np.isclose(slope(lambda y: loss(**{name: y}), at, v), (got[name] * v).sum(), rtol=1e-6), name


def test_recurrence_step_is_one_token():
    x, r, i = (normal(s, 3, 1, 4) for s in (1, 2, 3))
    states, decay = normal(4, 5, 4), normal(5, 4)
    h, after = rec.recur_step(x[:, 0], r[:, 0], i[:, 0], decay, 8.0, states, [4, -1, 1])
    want, last = rec.recur_fwd(x, r, i, decay, 8.0, state=states[[4, 0, 1]])
    assert np.array_equal(h[[0, 2]], want[[0, 2], 0]) and not h[1].any()
    assert np.array_equal(after[[4, 1]], last[[0, 2]]) and np.array_equal(after[[0, 2, 3]], states[[0, 2, 3]])


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_group_norm_by_differences(act):
    b, t, w, g = 2, 5, 6, 3
    x, dy = normal(1, b, t, w), normal(2, b, t, w)
    wt, bias = 1 + 0.1 * normal(3, w), normal(4, w)
    lens = [5, 3]
    y, stats = rec.group_norm_fwd(x, g, wt, bias, act, 1e-3, lens)
    assert not y[1, 3:].any()
    z, _ = rec.group_norm_fwd(x, g, lens=lens, eps=1e-12)
    for s in range(b):
        v = z[s, :lens[s]].reshape(lens[s], g, -1)
        assert np.allclose(v.mean((0, 2)), 0) and np.allclose((v ** 2).mean((0, 2)), 1)
    got = dict(zip("xwb", rec.group_norm_bwd(x, g, wt, bias, stats, dy, act, lens)))

    def loss(x=x, w=wt, b=bias):
        return (rec.group_norm_fwd(x, g, w, b, act, 1e-3, lens)[0] * dy).sum()

    for name, at in (("x", x), ("w", wt), ("b", bias)):
        v = normal(9, *at.shape)
        assert np.isclose(slope(lambda y: loss(**{name: y}), at, v), (got[name] * v).sum(), rtol=1e-5), name


@pytest.mark.parametrize("shape", [(4, 9), (9, 4), (5, 5), (1, 7), (7, 1), (1, 1)])
def test_orthogonal_maps_the_singular_values(shape):
    U = normal(3, *shape)
    left, s, right = np.linalg.svd(U / np.linalg.norm(U), full_matrices=False)
    p, q, c = rec.COEF
    for _ in range(5):
        s = s * (p + q * s ** 2 + c * s ** 4)
    assert np.allclose(rec.orthogonal(U), (left * s) @ right, atol=1e-12)
    assert not rec.orthogonal(np.zeros(shape)).any()


def test_the_polynomial_keeps_its_range():
    """[0, 1.21] goes into itself, with the bounds on X, A and B that the stored parts rely on."""
    p, q, c = rec.COEF
    x = np.linspace(0, 1.21, 200_001)
    y = x * (p + q * x ** 2 + c * x ** 4)
    assert 0 <= y.min() and y.max() < 1.21
    lam = x * x
    assert lam.max() < 1.4642 and np.abs(q * lam + c * lam ** 2).max() < 2.81


def test_muon_step():
    W, G, M = (normal(s, 3, 4) for s in (1, 2, 3))
    w, m = rec.muon_step(W, G, M, 0.1, 0.9, 0.2, True, 5, 2.0)
    assert np.allclose(m, 0.9 * M + G)
    assert np.allclose(w, 0.98 * W - 0.2 * rec.orthogonal(G + 0.9 * m))
    w0, _ = rec.muon_step(W, G, M, 0.1, 0.9, 0.0, False, 0, 1.0)
    assert np.allclose(w0, W - 0.1 * m / np.linalg.norm(m))
