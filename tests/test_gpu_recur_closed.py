"""Gradients of the gated linear recurrence (hg_recur_bwd) where almost nothing
passes its gates: 1 - a^2 is exact, by its own size, down to 2^-126, the smallest
normal number, and is taken as zero below; no product of large rows and small
gates overflows on the way to a gradient of zero.

Bars (max over a channel's elements of |error| / max(|value|, its rms)): those of
every recurrence, (16 + t) 2^-23 and 2^-8 for bfloat16 rows, with |z| log2 e
roundings of 2^-24 of an exponential for a gate at z: 128 2^-24 to z = -88."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bar(dtype, t):
    return (16 + t) * 2.0 ** -23 + 128 * 2.0 ** -24 + (2.0 ** -8 if dtype is BF16 else 0.0)


def normal(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def host(t):
    return t.double().cpu().numpy()


def slopes(*rho, rate=8.0):
    """decay for which rate softplus(decay) is as given."""
    return torch.log(torch.expm1(torch.tensor(rho, dtype=torch.float64) / rate)).float().cuda()


def backward(x, r, i, g, dh):
    h, _ = api.hg_recur_fwd(x, r, i, g)
    got = api.hg_recur_bwd(x, r, i, g, h, dh)
    return [host(v) for v in got[:4]], rec.recur_bwd(host(x), host(r), host(i), host(g), 8.0, host(h), host(dh))


SHAPES = [(3, 20), (1030, 70), (2, 400)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t", SHAPES)
def test_small_gates(b, t, dtype):
    """r near -84.5 (1 - a^2 from 2^-121 on) and from there to -100."""
    w = 8
    at = torch.tensor([-20.0, -60.0, -84.5, -84.5, -84.5, -88.0, -92.0, -100.0]).cuda()
    g = slopes(1.0, 1.0, 1.0, 2.0, 3.0, 1.0, 1.0, 1.0)
    x, i, dh = (normal(k, b, t, w, dtype=dtype) for k in (1, 2, 3))
    r = (at + 0.5 * torch.sin(normal(4, b, t, w))).to(dtype)
    got, want = backward(x, r, i, g, dh)
    for k, name in enumerate(("dx", "dr", "di")):
        for c in range(5):
            assert parity_err(got[k][..., c], want[k][..., c]) < bar(dtype, t), (name, c)
    for k in (0, 2):  # right or nothing
        d, v = got[k][..., 5:], want[k][..., 5:]
        assert ((np.abs(d - v) <= bar(dtype, t) * np.abs(v)) | (d == 0)).all()


@pytest.mark.parametrize("b,t", SHAPES)
def test_large_rows_behind_closed_gates(b, t):
    """x and dh of 1e15 where sigmoid(r) = 0 or the decay lets nothing in: gradients of zero, as finite ones."""
    w = 8
    x, i = (normal(k, b, t, w) for k in (1, 2))
    r, dh = normal(3, b, t, w), normal(4, b, t, w)
    g = slopes(*[1.0] * w)
    g[1] = -120.0
    r[:, 5] = float("-inf")
    x[:, 5], dh[:, 5] = x[:, 5] * 1e15, dh[:, 5] * 1e15
    x[..., 1] *= 1e15
    dh[..., 1] *= 1e15
    got, _ = backward(x, r, i, g, dh)
    assert all(np.isfinite(v).all() for v in got)
    for k in (0, 1, 2):
        assert not got[k][:, 5].any() and not got[k][..., 1].any()
    assert got[3][1] == 0
