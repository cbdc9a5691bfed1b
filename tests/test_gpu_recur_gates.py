"""Gradients of the gated linear recurrence (hg_recur_bwd) where its gates are
nearly open or shut, each channel by its own size: a channel's dr and di are as
small as sigmoid' there, far below those of the others.

Bars (max over a channel's elements of |error| / max(|value|, its rms)): float32
as everywhere, (16 + min(t, 1 / (1 - a))) 2^-23 with the exponentials' own error
beside it, |z| log2 e roundings of 2^-24 for a gate at z: 64 2^-24 up to z = 40.
bfloat16: half a step of the written row, 2^-8, beside that."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
EXPS = 64 * 2.0 ** -24


def bar(dtype, t):
    return (16 + min(t, 2000)) * 2.0 ** -23 + EXPS + (2.0 ** -8 if dtype is BF16 else 0.0)


def normal(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def host(t):
    return t.double().cpu().numpy()


def decays(w, rate=8.0):
    """Factors at r = 0 from 0.2 to 0.9995."""
    a = 1 - torch.logspace(np.log10(0.8), np.log10(5e-4), w, dtype=torch.float64)
    return torch.log(torch.expm1(-2 * torch.log(a) / rate)).float().cuda()


def backward(x, r, i, g, dh, s0):
    h, _ = api.hg_recur_fwd(x, r, i, g, state=s0)
    got = api.hg_recur_bwd(x, r, i, g, h, dh, state=s0)
    return [host(v) for v in got], rec.recur_bwd(host(x), host(r), host(i), host(g), 8.0, host(h), host(dh), None, host(s0))


# a wave and a block that walk a sequence, and tiles that compose through memory
SHAPES = [(3, 20, 16), (1030, 70, 12), (2, 700, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,w", SHAPES)
def test_open_and_shut_gates(b, t, w, dtype):
    """Both gates of channel c near the same value, from -16 to 40."""
    at = torch.linspace(-16.0, 40.0, w).cuda()
    x, dh, s0 = normal(1, b, t, w, dtype=dtype), normal(4, b, t, w, dtype=dtype), normal(5, b, w)
    r, i = ((normal(k, b, t, w) * 0.25 + at).to(dtype) for k in (2, 3))
    got, want = backward(x, r, i, decays(w), dh, s0)
    for k, name in enumerate(("dx", "dr", "di")):
        for c in range(w):
            assert parity_err(got[k][..., c], want[k][..., c]) < bar(dtype, t), (name, float(at[c]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,w", SHAPES)
def test_infinite_gates(b, t, w, dtype):
    """Gates at their ends have finite gradients: zero, like sigmoid' there."""
    x, dh, s0 = normal(1, b, t, w, dtype=dtype), normal(4, b, t, w, dtype=dtype), normal(5, b, w)
    r, i = normal(2, b, t, w, dtype=dtype), normal(3, b, t, w, dtype=dtype)
    inf = float("inf")
    r[:, 2], r[:, 3], i[:, 4], i[:, 5], r[:, 6], i[:, 7] = inf, -inf, inf, -inf, 200.0, -200.0
    got, want = backward(x, r, i, decays(w), dh, s0)
    assert all(np.isfinite(v).all() for v in got)
    assert not got[1][:, [2, 3, 6]].any() and not got[2][:, [4, 5, 7]].any()
    for k in range(5):
        assert parity_err(got[k], want[k]) < bar(dtype if k < 3 else F32, t), k
