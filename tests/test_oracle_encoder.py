"""The encoder oracle on the CPU: linear attention against its closed form (a
lower-triangular matrix of decays), the rotation's invariants, and every
gradient against central differences."""
import numpy as np
import pytest

from oracle import encoder


def diff(f, x, e=1e-6):
    """Central differences of the scalar f over every element of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += e
        b[i] -= e
        g[i] = (f(a) - f(b)) / (2 * e)
    return g


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_linear_and_glu_gradients(act):
    r = np.random.default_rng(1)
    x, W, b, R = r.normal(size=(4, 3)), r.normal(size=(3, 6)), r.normal(size=6), r.normal(size=(4, 6))
    for fwd, bwd, up in ((lambda x, W, b: encoder.linear(x, W, b, R, act), encoder.linear_bwd, r.normal(size=(4, 6))),
                         (lambda x, W, b: encoder.glu(x, W, b, act), encoder.glu_bwd, r.normal(size=(4, 3)))):
        dx, dW, db = bwd(x, W, b, up, act)
        assert np.allclose(dx, diff(lambda v: (fwd(v, W, b) * up).sum(), x), atol=1e-7)
        assert np.allclose(dW, diff(lambda v: (fwd(x, v, b) * up).sum(), W), atol=1e-7)
        assert np.allclose(db, diff(lambda v: (fwd(x, W, v) * up).sum(), b), atol=1e-7)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 4, 8])
def test_norm_rope(interleaved, rot):
    r = np.random.default_rng(2)
    x, w, up = r.normal(size=(5, 2, 8)), r.normal(size=8), r.normal(size=(5, 2, 8))
    pos = np.array([0, 3, 9, 1, 3])
    tab = encoder.rope_table(10, rot)
    y = encoder.norm_rope(x, None, tab, pos, 0.0, interleaved)
    assert np.allclose((y ** 2).mean(-1), 1)              # turning keeps the norm
    # the product of a turned query and key depends on the distance alone
    z = encoder.norm_rope(np.broadcast_to(x[:1], x.shape), None, tab, pos, 0.0, interleaved)
    s = np.einsum("ihd,jhd->ijh", z, z)
    assert np.allclose(s[1, 4], s[0, 0]) and np.allclose(s[1, 1], s[2, 2])
    dx, dw = encoder.norm_rope_bwd(x, w, tab, pos, up, 1e-3, interleaved)
    assert np.allclose(dx, diff(lambda v: (encoder.norm_rope(v, w, tab, pos, 1e-3, interleaved) * up).sum(), x), atol=1e-7)
    assert np.allclose(dw, diff(lambda v: (encoder.norm_rope(x, v, tab, pos, 1e-3, interleaved) * up).sum(), w), atol=1e-7)
    bad = encoder.norm_rope(x, w, tab, np.array([0, -1, 9, 10, 3]), 1e-3, interleaved)
    assert np.isnan(bad[[1, 3]]).all() and np.isfinite(bad[[0, 2, 4]]).all()


def test_linattn_closed_form_and_gradients():
    r = np.random.default_rng(3)
    b, t, h, hk, d = 2, 5, 4, 2, 3
    q, k, v = r.normal(size=(b, t, h, d)), r.normal(size=(b, t, hk, d)), r.normal(size=(b, t, hk, d))
    g, S0 = -np.array([0.0, 0.1, 1.0, 4.0]), r.normal(size=(b, h, d, d))
    lens = np.array([5, 3])
    o, S = encoder.linattn(q, k, v, g, 0.7, lens, S0)
    for i in range(b):
        n = lens[i]
        for j in range(h):
            x = np.arange(n)
            M = np.where(x[:, None] >= x[None], np.exp(g[j] * np.maximum(x[:, None] - x[None], 0)), 0)
            kk, vv = k[i, :n, j // 2], v[i, :n, j // 2]
            ref = 0.7 * ((q[i, :n, j] @ kk.T * M) @ vv + np.exp(g[j] * (x + 1))[:, None] * (q[i, :n, j] @ S0[i, j]))
            assert np.allclose(o[i, :n, j], ref) and not o[i, n:, j].any()
            end = (kk * np.exp(g[j] * (n - 1 - x))[:, None]).T @ vv + np.exp(g[j] * n) * S0[i, j]
            assert np.allclose(S[i, j], end)
    do, dS = r.normal(size=o.shape), r.normal(size=S.shape)

    def loss(q, k, v, S0):
        o, S = encoder.linattn(q, k, v, g, 0.7, lens, S0)
        return (o * do).sum() + (S * dS).sum()

    dq, dk, dv, dS0 = encoder.linattn_bwd(q, k, v, g, do, 0.7, lens, S0, dS)
    assert np.allclose(dq, diff(lambda x: loss(x, k, v, S0), q), atol=1e-6)
    assert np.allclose(dk, diff(lambda x: loss(q, x, v, S0), k), atol=1e-6)
    assert np.allclose(dv, diff(lambda x: loss(q, k, x, S0), v), atol=1e-6)
    assert np.allclose(dS0, diff(lambda x: loss(q, k, v, x), S0), atol=1e-6)


def test_linattn_steps_are_the_sequence():
    r = np.random.default_rng(4)
    b, t, h, hk, d = 3, 6, 2, 1, 4
    q, k, v = r.normal(size=(b, t, h, d)), r.normal(size=(b, t, hk, d)), r.normal(size=(b, t, hk, d))
    g, S = np.array([-0.2, -0.01]), np.zeros((5, h, d, d))
    o, end = encoder.linattn(q, k, v, g, 0.5)
    slots = np.array([4, 0, 2])
    for i in range(t):
        y, S = encoder.linattn_step(q[:, i], k[:, i], v[:, i], g, S, slots, 0.5)
        assert np.allclose(y, o[:, i])
    assert np.allclose(S[slots], end) and not S[[1, 3]].any()
    y, S2 = encoder.linattn_step(q[:, 0], k[:, 0], v[:, 0], g, S, np.array([5, -1, 2]), 0.5)
    assert not y[:2].any() and np.array_equal(S2[[0, 1, 3, 4]], S[[0, 1, 3, 4]])
