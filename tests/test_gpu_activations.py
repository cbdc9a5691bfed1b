"""The activations of the linear map and the gated product far from zero, where
exponentials overflow and vanish: z on a dense grid over -200 .. 200, at +-1e4 and
at +-infinity, forward and backward, on every path (few rows, tiles, tiles with k
split, narrow rows in one pass), against the oracle in float64.

z is set by the bias: X W adds exact zeros to it, since X is one in its first
column, where W is zero, and zero elsewhere.  So dW's first row and dbias are
the sums of dz over the rows, and dX is dz W^T.

Bounds.  SiLU is z s(z): the exponential, 1 + e, the reciprocal and the product
are each off by at most 2^-22 relative, 2^-20 together; where s falls below the
smallest normal number 2^-126 it may be zero.  GELU is z Phi(z), with Phi formed
to 2^-22 (the last test holds negative z to their own size).  bfloat16 results add
one rounding: 8 bits, 2^-8 of a value just above a power of two."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder
from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ACT = {"silu": api.HG_ACT_SILU, "gelu": api.HG_ACT_GELU}
SPECIAL = [-89.0, -95.0, -101.0, -110.0, -128.0, -149.0, -1e4, 1e4, -88.75, 88.75, -0.0, -1e-30, 1e-30, 150.0, -150.0]


def grid(kind):
    """z of the columns, float32; `kind`: with the infinities, or a part of them for 128 columns."""
    z = np.concatenate([np.linspace(-200, 200, 785), SPECIAL]).astype(np.float32)
    if kind == "narrow":
        z = np.concatenate([z[785:], z[:785:7]])[:128]
    return np.concatenate([z, np.array([np.inf, -np.inf] * 4, np.float32)]) if kind == "infinite" else z


def problem(n, d, z, dtype, gated):
    """x, W and the bias that give z in every row (gated: beside u = 1.5)."""
    f = len(z)
    g = torch.Generator().manual_seed(3)
    x = torch.zeros(n, d, dtype=dtype)
    x[:, 0] = 1
    W = (torch.randn(d, 2 * f if gated else f, generator=g) * d ** -0.5).to(dtype)
    W[0] = 0
    b = torch.from_numpy(np.concatenate([z, np.full(f, 1.5, np.float32)]) if gated else z)
    up = torch.randn(n, f, generator=g).to(dtype)
    return x.cuda(), W.cuda(), b.cuda(), up.cuda()


def host(t):
    return t.double().cpu().numpy()


def close(got, z, act, dtype, factor=1.0):
    z = z.astype(np.float64)
    with np.errstate(over="ignore"):
        ref = encoder.act(act, z) * factor
    rel, low = 2.0 ** -20 + (2.0 ** -8 if dtype == BF16 else 0), np.abs(z) * factor * 2.0 ** -125
    if act == "gelu":
        low = np.abs(z) * factor * 2.0 ** -22
    err = np.abs(got - ref)
    assert np.all(np.isfinite(got)), z[~np.isfinite(got).all(0)]
    assert np.all(err <= rel * np.abs(ref) + low), (z[(err > rel * np.abs(ref) + low).any(0)][:5], err.max())


# rows and k: few rows, tiles, k split over blocks
ROWS = [(1, 64), (2, 24), (4, 40), (100, 64), (100, 2048), (333, 24)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,d", ROWS)
def test_forward(n, d, act, dtype):
    z = grid("all")
    x, W, b, _ = problem(n, d, z, dtype, False)
    close(host(api.hg_linear_fwd(x, W, bias=b, act=ACT[act])), z, act, dtype)
    x, W, b, _ = problem(n, d, z, dtype, True)
    close(host(api.hg_glu_fwd(x, W, bias=b, act=ACT[act])), z, act, dtype, 1.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n,d", ROWS)
def test_backward(n, d, gated, act, dtype):
    check_backward(n, d, grid("all"), gated, act, dtype)


def check_backward(n, d, z, gated, act, dtype):
    """A gradient is a sum of products of dz = up * (a factor formed from z).  The
    factor is off by at most 2^-18 of max(1, |z|) (SiLU's slope adds s and f (1 - s)),
    and the sums add less than that.  bfloat16 calls round dz and the result, 2^-8 each."""
    x, W, b, up = problem(n, d, z, dtype, gated)
    got = (api.hg_glu_bwd if gated else api.hg_linear_bwd)(x, W, b, up, act=ACT[act])
    X, V, U, z = host(x), host(W), host(up), z.astype(np.float64)
    with np.errstate(over="ignore"):
        f, s = encoder.act(act, z), encoder.act_slope(act, z)
    dz, size = (np.concatenate(p, 1) if gated else p[0] for p in
                (([U * 1.5 * s, U * f] if gated else [U * s]), [np.abs(U) * 1.5, np.abs(U) * np.maximum(1, np.abs(z))]))
    u = 2.0 ** -8 if dtype == BF16 else 0.0
    off = u * np.abs(dz) + 2.0 ** -17 * size
    refs = (("dx", dz @ V.T, off @ np.abs(V).T, u), ("dW", X.T @ dz, np.abs(X).T @ off, u),
            ("db", dz.sum(0), 2.0 ** -17 * size.sum(0), 0.0))
    for (name, r, e, round_), g in zip(refs, got):
        assert torch.isfinite(g).all(), name
        err = np.abs(host(g) - r)
        assert np.all(err <= e + round_ * (np.abs(r) + e) + 2.0 ** -22 * np.abs(r)), (name, (err / (e + 1e-300)).max())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n", [16384, 16411])
def test_narrow_rows(n, act):
    """The rows past the end of the last tile have z = bias too and stay out of every sum."""
    check_backward(n, 128, grid("narrow"), False, act, F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,d", ROWS)
def test_infinities_stay_in_their_column(n, d, act, dtype):
    z = grid("infinite")
    x, W, b, up = problem(n, d, z, dtype, False)
    fin = np.isfinite(z)
    y = host(api.hg_linear_fwd(x, W, bias=b, act=ACT[act]))
    close(y[:, fin], z[fin], act, dtype)
    assert np.all(y[:, z == np.inf] == np.inf)
    _, dW, db = api.hg_linear_bwd(x, W, b, up, act=ACT[act], want=(False, True, True))
    clean = torch.where(torch.isfinite(b), b, torch.zeros_like(b))
    _, cW, cb = api.hg_linear_bwd(x, W, clean, up, act=ACT[act], want=(False, True, True))
    keep = torch.from_numpy(fin).cuda()
    assert torch.equal(dW[:, keep], cW[:, keep]) and torch.equal(db[keep], cb[keep])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", ROWS)
def test_gelu_keeps_its_digits_below_zero(n, d, dtype):
    """z Phi(z) for z = -13 .. 0 to its own size: the tail and the products to 2^-20, exp(-z^2 / 2) to z^2 2^-24 for
    the rounding of z^2, one rounding of the result."""
    z = np.linspace(-13, 0, 800).astype(np.float32)
    z64 = z.astype(np.float64)
    ref = z64 * 0.5 * np.vectorize(math.erfc)(-z64 / math.sqrt(2))
    rel = 2.0 ** -20 + z64 ** 2 * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0)
    x, W, b, _ = problem(n, d, z, dtype, False)
    err = np.abs(host(api.hg_linear_fwd(x, W, bias=b, act=api.HG_ACT_GELU)) - ref)
    assert np.all(err <= rel * np.abs(ref) + 13 * 2.0 ** -125)
    x, W, b, _ = problem(n, d, z, dtype, True)
    err = np.abs(host(api.hg_glu_fwd(x, W, bias=b, act=api.HG_ACT_GELU)) - 1.5 * ref)
    assert np.all(err <= (rel * np.abs(ref) + 13 * 2.0 ** -125) * 1.5)
