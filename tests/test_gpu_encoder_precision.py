"""What the bfloat16 calls of the sequence encoder promise about precision, held by
the norm of the error over the norm of the result (float64).

Rounding normal values to 8 bits is off by 0.85 x 2^-9 of their norm (an error
uniform over a unit in the last place, 2^-7 / sqrt(12) of the power of two below
a value), up to 0.9 x 2^-9 with some thousand values; roundings of independent
values add in squares.  So a result that is rounded once, from float32 or from
16-bit factors (2^-17), is within 2^-9; one whose dz was rounded to 8 bits before
within sqrt(2) 2^-9; 1% for the rest."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder
from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ONE, TWO = 1.01 * 2.0 ** -9, 1.01 * math.sqrt(2) * 2.0 ** -9  # roundings


def normal(seed, *shape, dtype=BF16, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def off(got, ref):
    got, ref = (torch.as_tensor(v).double().cpu() for v in (got, ref))
    return float((got - ref).norm() / ref.norm())


def product_grads(n, d, f, gated, act, want):
    """(the call's dx, dw; those in float64)"""
    x, w = normal(1, n, d), normal(2, d, 2 * f if gated else f, scale=d ** -0.5)
    b, up = normal(3, w.shape[1], dtype=torch.float32), normal(4, n, f)
    code = {"none": api.HG_ACT_NONE, "silu": api.HG_ACT_SILU, "gelu": api.HG_ACT_GELU}[act]
    got = (api.hg_glu_bwd if gated else api.hg_linear_bwd)(x, w, b, up, act=code, want=want)
    fun = {"none": lambda v: v, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act]
    X, W = x.double(), w.double()
    z = (X @ W + b.double()).requires_grad_()
    y = fun(z[:, :f]) * z[:, f:] if gated else fun(z)
    (dz,) = torch.autograd.grad(y, z, up.double())
    ref = (dz @ W.T if want[0] else None, X.T @ dz if want[1] else None)
    return [(a, r) for a, r in zip(got, ref) if r is not None]


# n d_in d_out (gated 2 f): dX or dW of fewer than 4096 values, up to 2^28 products
@pytest.mark.parametrize("n,d,f,gated", [(70000, 60, 60, False), (74000, 60, 30, True), (511, 8, 4000, False),
                                         (40, 100, 3000, True), (3000, 7, 500, False)])
def test_gradients_of_few_values_are_rounded_once(n, d, f, gated):
    cols = 2 * f if gated else f
    assert d * min(n, cols) < 4096 and n * d * cols <= 1 << 28
    for got, ref in product_grads(n, d, f, gated, "silu", (True, True, False)):
        assert off(got, ref) <= ONE


@pytest.mark.parametrize("n,d,f,gated,want", [
    (75000, 60, 60, False, (True, True, False)), (80000, 60, 30, True, (True, True, False)),  # past 2^28 products
    (1, 2048, 131080, False, (True, False, False)),
    (64, 64, 4000, False, (True, True, False)), (4096, 64, 64, False, (True, True, False)),  # 4096 values
    (1000, 72, 264, False, (True, True, False)), (2500, 130, 129, True, (True, True, False)),
    (4100, 520, 768, False, (True, True, False)), (2050, 512, 1536, True, (True, True, False))])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_other_gradients_round_dz_and_the_result(n, d, f, gated, want, act):
    for got, ref in product_grads(n, d, f, gated, act, want):
        assert off(got, ref) <= TWO


@pytest.mark.parametrize("n,d,f", [(1000, 72, 264), (5, 370, 515), (4100, 520, 768)])
def test_gradients_without_an_activation_are_rounded_once(n, d, f):
    for got, ref in product_grads(n, d, f, False, "none", (True, True, False)):
        assert off(got, ref) <= ONE


@pytest.mark.parametrize("n,d,f", [(1, 512, 2064), (6, 40, 515), (300, 72, 136), (2000, 512, 384), (64, 2048, 64)])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_products_are_rounded_once(n, d, f, act):
    code = {"none": api.HG_ACT_NONE, "silu": api.HG_ACT_SILU, "gelu": api.HG_ACT_GELU}[act]
    x, w, v = normal(1, n, d), normal(2, d, f, scale=d ** -0.5), normal(3, d, 2 * f, scale=d ** -0.5)
    r = normal(4, n, f)
    h = [t.double().cpu().numpy() for t in (x, w, v, r)]
    assert off(api.hg_linear_fwd(x, w, residual=r, act=code), encoder.linear(h[0], h[1], None, h[3], act)) <= ONE
    assert off(api.hg_glu_fwd(x, v, act=code), encoder.glu(h[0], h[2], None, act)) <= ONE


# one chunk, several, several segments; the heads of a key head apart, two in a block, and three with a sum of gradients
ATTN = [(2, 33, 2, 2, 64), (3, 130, 4, 2, 96), (2, 257, 3, 1, 24), (1, 1500, 2, 2, 64), (1, 1200, 2, 1, 128),
        (700, 40, 4, 2, 16), (350, 70, 6, 2, 32)]


@pytest.mark.parametrize("b,t,h,hk,d", ATTN)
def test_linear_attention_is_rounded_once(b, t, h, hk, d):
    """P and the copy of S at 16 bits do not show beside the rounding of o and of the
    gradients: either at 8 bits would, as one more rounding."""
    q, kv, do = normal(1, b, t, h, d), normal(2, b, t, 2 * hk, d), normal(3, b, t, h, d)
    k, v = kv[:, :, :hk], kv[:, :, hk:]
    g = -torch.logspace(-2.5, -0.5, h, device="cuda")
    S, dS = normal(4, b, h, d, d, dtype=torch.float32), normal(5, b, h, d, d, dtype=torch.float32)
    Q, K, V, O, G, S0, D0 = (x.double().cpu().numpy() for x in (q, k, v, do, g, S, dS))
    o, end = api.hg_linattn_fwd(q, k, v, g, scale=0.3, state=S, want_state=True)
    ro, rend = encoder.linattn(Q, K, V, G, 0.3, None, S0)
    assert off(o, ro) <= ONE and off(end, rend) <= 1e-5
    got = api.hg_linattn_bwd(q, k, v, g, do, scale=0.3, state=S, dstate_out=dS)
    ref = encoder.linattn_bwd(Q, K, V, G, O, 0.3, None, S0, D0)
    for a, r in zip(got[:3], ref[:3]):
        assert off(a, r) <= ONE
    assert off(got[3], ref[3]) <= 1e-5
