"""GPU parity of the linear map and the gated product (hg_linear_*, hg_glu_*)
against the oracle (oracle/encoder.py, float64): every output, for widths that
fill no tile, strided rows, one row and many, all activations, the k range
split over blocks, accumulation, partial gradients, values that are not finite,
and the argument checks.

Bars (max over elements of |error| / max(|value|, rms)): float32 1e-4, the bar
of the library's float32 products; bfloat16 2e-2: the result's rounding (2^-9
relative) and, in the backward, the rounding of dz (2^-9 a term, at most 4e-3 of
the rms for the 200 terms and more of these sums)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
BAR = {torch.float32: 1e-4, torch.bfloat16: 2e-2}
ACT = {"none": api.HG_ACT_NONE, "relu": api.HG_ACT_RELU, "silu": api.HG_ACT_SILU, "gelu": api.HG_ACT_GELU}
F32, BF16 = torch.float32, torch.bfloat16


def draw(seed, *shape, dtype=F32, scale=1.0, pad=0):
    """A device tensor; with pad its rows lie in wider ones filled with NaN."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(*shape, generator=g) * scale).to(dtype)
    if pad:
        wide = torch.full((*shape[:-1], shape[-1] + pad), float("nan"), dtype=dtype, device="cuda")
        wide[..., :shape[-1]] = x.cuda()
        return wide[..., :shape[-1]]
    return x.cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def problem(n, d, cols, dtype, bias, pad, seed=1):
    x = draw(seed, n, d, dtype=dtype, pad=pad)
    W = draw(seed + 1, d, cols, dtype=dtype, scale=d ** -0.5)
    b = draw(seed + 2, cols, scale=0.5) if bias else None
    return x, W, b


# rows: the single-token kernel (1, 2, 3, 8), the tiles (9, 130, 1000), many tiles
SHAPES = [(1, 64, 64), (2, 200, 136), (3, 37, 51), (8, 512, 72), (9, 16, 8), (130, 200, 136), (65, 37, 51),
          (1000, 72, 264), (257, 1, 1), (64, 2048, 64), (4100, 256, 512)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,m", SHAPES)
@pytest.mark.parametrize("act,bias,pad", [("none", True, 0), ("silu", False, 3), ("gelu", True, 8), ("relu", True, 0)])
def test_linear_forward(n, d, m, dtype, act, bias, pad):
    x, W, b = problem(n, d, m, dtype, bias, pad)
    r = draw(7, n, m, dtype=dtype, pad=pad) if bias else None
    y = torch.full((n, m + 5), 9.0, dtype=dtype, device="cuda")[:, :m]
    api.hg_linear_fwd(x, W, bias=b, residual=r, act=ACT[act], y=y)
    ref = encoder.linear(host(x), host(W), host(b), host(r), act)
    assert parity_err(host(y), ref) <= BAR[dtype]
    if n > 1:  # the columns between the rows are untouched
        assert torch.all(y.as_strided((n - 1, 5), (m + 5, 1), m) == 9.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", SHAPES)
@pytest.mark.parametrize("act,bias,pad", [("silu", False, 0), ("gelu", True, 8), ("none", True, 5)])
def test_glu_forward(n, d, f, dtype, act, bias, pad):
    x, W, b = problem(n, d, 2 * f, dtype, bias, pad)
    h = api.hg_glu_fwd(x, W, bias=b, act=ACT[act])
    assert parity_err(host(h), encoder.glu(host(x), host(W), host(b), act)) <= BAR[dtype]


def check_grads(got, ref, dtype, what):
    for name, g, r in zip(("dx", "dW", "db"), got, ref):
        if g is not None:
            bar = 1e-4 if name == "db" else BAR[dtype]
            err = parity_err(host(g), r)
            assert err <= bar, (what, name, err)


BWD = [(1, 64, 64), (5, 37, 51), (130, 200, 136), (1000, 72, 264), (2500, 128, 128), (3, 8, 520), (700, 33, 7)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,m", BWD)
@pytest.mark.parametrize("act,bias,pad", [("none", True, 0), ("none", False, 5), ("silu", True, 0), ("gelu", False, 8)])
def test_linear_backward(n, d, m, dtype, act, bias, pad):
    x, W, b = problem(n, d, m, dtype, bias, pad)
    dy = draw(9, n, m, dtype=dtype, pad=pad)
    got = api.hg_linear_bwd(x, W, b, dy, act=ACT[act])
    check_grads(got, encoder.linear_bwd(host(x), host(W), host(b), host(dy), act), dtype, (n, d, m, act))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", BWD)
@pytest.mark.parametrize("act,bias,pad", [("silu", True, 0), ("gelu", False, 8), ("none", True, 3)])
def test_glu_backward(n, d, f, dtype, act, bias, pad):
    x, W, b = problem(n, d, 2 * f, dtype, bias, pad)
    dh = draw(9, n, f, dtype=dtype, pad=pad)
    got = api.hg_glu_bwd(x, W, b, dh, act=ACT[act])
    check_grads(got, encoder.glu_bwd(host(x), host(W), host(b), host(dh), act), dtype, (n, d, f, act))


@pytest.mark.parametrize("n,d,f,pad", [(20003, 128, 128, 0), (16384, 64, 128, 4), (16400, 128, 64, 0), (17001, 36, 20, 8),
                                       (16385, 4, 100, 0), (30000, 100, 4, 4)])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_narrow_rows_backward(n, d, f, pad, act):
    """Very many float32 rows with both widths up to 128: one pass; the same by
    tiles where dx is not wanted; added into what is there."""
    x, W, b = problem(n, d, f, F32, True, pad)
    dy = draw(9, n, f, pad=pad)
    wide = torch.full((n, d + 4), 5.0, device="cuda")
    got = api.hg_linear_bwd(x, W, b, dy, act=ACT[act], dx=wide[:, :d])
    ref = encoder.linear_bwd(host(x), host(W), host(b), host(dy), act)
    check_grads(got, ref, F32, (n, d, f, act))
    assert torch.all(wide[:, d:] == 5.0)
    again = api.hg_linear_bwd(x, W, b, dy, act=ACT[act], want=(False, True, True))
    check_grads(again, ref, F32, "by tiles")
    dW, db = torch.full_like(W, 2.0), torch.full_like(b, 3.0)
    api.hg_linear_bwd(x, W, b, dy, act=ACT[act], dW=dW, dbias=db, accumulate=True)
    assert torch.equal(dW, 2.0 + got[1]) and torch.equal(db, 3.0 + got[2])


def test_relu_backward_away_from_the_kink():
    # z = x W + b with b far from every kink: half of the columns all positive, half all negative
    n, d, m = 300, 40, 64
    x, W, _ = problem(n, d, m, F32, False, 0)
    b = torch.where(torch.arange(m, device="cuda") % 2 == 0, 30.0, -30.0)
    dy = draw(9, n, m)
    got = api.hg_linear_bwd(x, W, b, dy, act=api.HG_ACT_RELU)
    check_grads(got, encoder.linear_bwd(host(x), host(W), host(b), host(dy), "relu"), F32, "relu")
    assert torch.all(got[1][:, 1::2] == 0)


def test_backward_against_differences():
    """The float32 gradients against central differences of the oracle's loss."""
    n, d, f = 12, 9, 7
    x, W, b = problem(n, d, 2 * f, F32, True, 0)
    dh = draw(9, n, f)
    dx, dW, db = (host(t) for t in api.hg_glu_bwd(x, W, b, dh, act=api.HG_ACT_GELU))
    X, V, B, G = host(x), host(W), host(b), host(dh)

    def loss(X, V, B):
        return float((encoder.glu(X, V, B, "gelu") * G).sum())

    e = 1e-6
    for at in ((0, 0), (5, 3), (11, 8)):
        p, q = X.copy(), X.copy()
        p[at] += e
        q[at] -= e
        assert abs((loss(p, V, B) - loss(q, V, B)) / (2 * e) - dx[at]) < 1e-4
    for at in ((0, 0), (4, 6), (8, 7), (2, 13)):
        p, q = V.copy(), V.copy()
        p[at] += e
        q[at] -= e
        assert abs((loss(X, p, B) - loss(X, q, B)) / (2 * e) - dW[at]) < 2e-4
    for at in (0, 6, 7, 13):
        p, q = B.copy(), B.copy()
        p[at] += e
        q[at] -= e
        assert abs((loss(X, V, p) - loss(X, V, q)) / (2 * e) - db[at]) < 1e-4


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_accumulate_and_partial_gradients(dtype):
    n, d, m = 200, 72, 40
    x, W, b = problem(n, d, m, dtype, True, 0)
    dy = draw(9, n, m, dtype=dtype)
    ref = encoder.linear_bwd(host(x), host(W), host(b), host(dy), "silu")
    dW, db = draw(20, d, m, dtype=dtype, scale=3.0), draw(21, m)
    w0, b0 = host(dW), host(db)
    dx, dW, db = api.hg_linear_bwd(x, W, b, dy, act=api.HG_ACT_SILU, dW=dW, dbias=db, accumulate=True)
    check_grads((dx, dW, db), (ref[0], w0 + ref[1], b0 + ref[2]), dtype, "accumulate")
    only = api.hg_linear_bwd(x, W, b, dy, act=api.HG_ACT_SILU, want=(False, True, False))
    assert only[0] is None and only[2] is None
    check_grads(only, (None, ref[1], None), dtype, "dW alone")
    only = api.hg_linear_bwd(x, W, b, dy, act=api.HG_ACT_SILU, want=(True, False, False))
    check_grads(only, ref, dtype, "dx alone")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows(dtype):
    x, W, b = problem(0, 24, 10, dtype, True, 0)
    assert api.hg_linear_fwd(x, W, bias=b).shape == (0, 10)
    assert api.hg_glu_fwd(x, W, bias=b).shape == (0, 5)
    dx, dW, db = api.hg_linear_bwd(x, W, b, x.new_zeros(0, 10))
    assert dx.shape == (0, 24) and not dW.any() and not db.any()
    dW, db = torch.ones_like(W), torch.ones_like(b)
    api.hg_glu_bwd(x, W, b, x.new_zeros(0, 5), dW=dW, dbias=db, accumulate=True)
    assert torch.all(dW == 1) and torch.all(db == 1)


def test_residual_in_place():
    for dtype in (F32, BF16):
        for n in (3, 300):
            x, W, _ = problem(n, 64, 64, dtype, False, 0)
            y = draw(5, n, 64, dtype=dtype)
            ref = encoder.linear(host(x), host(W), None, host(y), "silu")
            api.hg_linear_fwd(x, W, residual=y, act=api.HG_ACT_SILU, y=y)
            assert parity_err(host(y), ref) <= BAR[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [5, 200])
def test_values_that_are_not_finite_stay_in_their_row(dtype, n):
    x, W, b = problem(n, 72, 40, dtype, True, 0)
    clean = api.hg_linear_fwd(x, W, bias=b)
    for bad in (float("inf"), float("nan")):
        y = x.clone()
        y[3, 17] = bad
        got = api.hg_linear_fwd(y, W, bias=b)
        assert not torch.isfinite(got[3]).any()
        keep = torch.arange(n, device="cuda") != 3
        assert torch.equal(got[keep], clean[keep])


def test_rows_of_very_different_size():
    """float32 rows scaled by 1e-25 .. 1e25 keep their own relative accuracy."""
    n = 200
    x, W, _ = problem(n, 96, 64, F32, False, 0)
    s = 10.0 ** torch.linspace(-25, 25, n, device="cuda")[:, None]
    y = host(api.hg_linear_fwd(x * s, W))
    ref = encoder.linear(host(x * s), host(W))
    rms = np.sqrt((ref ** 2).mean(1, keepdims=True))
    assert np.max(np.abs(y - ref) / rms) < 1e-5


def test_deterministic_and_graph():
    """Two runs give equal bits, and a captured call replays to them."""
    n, d, f = 500, 264, 136
    x, W, b = problem(n, d, 2 * f, BF16, True, 0)
    dh = draw(9, n, f, dtype=BF16)
    ws = torch.empty(api.hg_glu_bwd_workspace_size(n, d, f, BF16), dtype=torch.uint8, device="cuda")
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)

    def call():
        api.hg_glu_bwd(x, W, b, dh, dx=dx, dW=dW, dbias=db, ws=ws)

    call()
    torch.cuda.synchronize()
    first = [t.clone() for t in (dx, dW, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        for t in (dx, dW, db):
            t.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        for t, u in zip((dx, dW, db), first):
            assert torch.equal(t, u)


def test_refusals():
    x, W, b = problem(20, 24, 32, BF16, True, 0)

    def refused(code, f, *a, **k):
        with pytest.raises(api.HgError) as e:
            f(*a, **k)
        assert e.value.status == code

    refused(api.HG_ERR_ARG, api.hg_linear_fwd, x, W, act=9)
    refused(api.HG_ERR_ARG, api.hg_linear_fwd, x, W, y=torch.empty(0, dtype=BF16, device="cuda").set_(
        W.untyped_storage(), 0, (20, 32), (32, 1)))
    wide = draw(1, 20, 40, dtype=BF16)
    refused(api.HG_ERR_ARG, api.hg_linear_fwd, wide[:, 1:25], W)  # not 16-byte aligned
    odd = draw(1, 20, 23, dtype=BF16)
    refused(api.HG_ERR_CAPACITY, api.hg_linear_fwd, odd, W[:23].contiguous(),
            ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        api.hg_linear_fwd(x, W.float())
    with pytest.raises(TypeError):
        api.hg_linear_fwd(x.half(), W.half())
    with pytest.raises(ValueError):
        api.hg_linear_fwd(x, W.t())
    with pytest.raises(ValueError):
        api.hg_linear_fwd(x, W, bias=b[:8])
    with pytest.raises(ValueError):
        api.hg_linear_fwd(x, W, bias=b.bfloat16())
    with pytest.raises(ValueError):
        api.hg_linear_fwd(x, W, y=torch.empty(20, 31, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        api.hg_glu_fwd(x, W[:, :31].contiguous())
    with pytest.raises(ValueError):
        api.hg_linear_bwd(x, W, b, torch.empty(20, 32, dtype=BF16, device="cuda"), accumulate=True)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n,d,f", [(10, 24, 1448), (1, 100, 37), (300, 13, 260)])
def test_small_bf16_gradients_keep_their_precision(n, d, f, gated):
    """Where a result has few values, dz enters the products with 16 bits: the
    gradients are off by their own rounding, at most 2^-9 of each value and so of the
    norm, and 1% more for dz and the sums."""
    x, w = draw(1, n, d, dtype=BF16), draw(2, d, 2 * f if gated else f, dtype=BF16, scale=d ** -0.5)
    b, up = draw(3, w.shape[1]), draw(4, n, f, dtype=BF16)
    if gated:
        got = api.hg_glu_bwd(x, w, b, up, act=api.HG_ACT_SILU)
    else:
        got = api.hg_linear_bwd(x, w, b, up, act=api.HG_ACT_SILU)
    X, W = x.double().requires_grad_(), w.double().requires_grad_()
    z = X @ W + b.double()
    y = torch.nn.functional.silu(z[:, :f]) * z[:, f:] if gated else torch.nn.functional.silu(z)
    for g, r in zip(got, torch.autograd.grad(y, (X, W), up.double())):
        assert float((g.double() - r).norm() / r.norm()) <= 1.01 * 2.0 ** -9
