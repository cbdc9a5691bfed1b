"""Group norms of more items than a launch has blocks, so that each block takes
several in turn: small items, many to a block, items of a block of 256 and of 1024
threads, single channels, ragged lengths; forward and backward against the same
formulas by torch in float64 on the device.

Bars as everywhere in the group norm: float32 2e-5 of the larger of a value and the
rms, half a step of the written row, 2^-8, beside it in bfloat16."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# items, tokens, groups, channels of a group
SHAPES = [(40000, 1, 4, 16), (70001, 1, 1, 8), (2900, 1, 2, 1024), (1300, 1, 1, 4096), (9001, 1, 7, 25), (5003, 9, 3, 24),
          (3001, 70, 1, 40), (1100, 600, 1, 16), (2500, 1, 1, 1000)]


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def off(got, want):
    rms = want.square().mean().sqrt()
    return float(((got.double() - want).abs() / torch.maximum(want.abs(), rms)).max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,g,cg", SHAPES)
def test_many_items(b, t, g, cg, dtype):
    bar, w = 2e-5 + (2.0 ** -8 if dtype is BF16 else 0.0), g * cg
    x = (0.7 * normal(1, b, t, w) + normal(2, w)).to(dtype)
    weight, bias, dy = 1 + 0.2 * normal(3, w), 0.5 * normal(4, w), normal(5, b, t, w).to(dtype)
    lens = torch.randint(0, t + 1, (b,), generator=torch.Generator().manual_seed(6)).int().cuda() if t > 1 else None
    y, stats = api.hg_group_norm_fwd(x, g, weight, bias, act=api.HG_ACT_SILU, lens=lens, want_stats=True)
    dx, dw, db = api.hg_group_norm_bwd(x, g, weight, bias, stats, dy, act=api.HG_ACT_SILU, lens=lens)
    n = torch.full((b,), t, device="cuda") if lens is None else lens.long()
    live = (torch.arange(t, device="cuda") < n[:, None])[:, :, None, None]
    count = (n * cg).clamp(min=1).view(b, 1, 1, 1)
    v = x.double().view(b, t, g, cg) * live
    mean = v.sum((1, 3), keepdim=True) / count
    rstd = 1 / (((v - mean) * live).square().sum((1, 3), keepdim=True) / count + 1e-5).sqrt()
    u = (v - mean) * rstd * live
    z = u * weight.double().view(g, cg) + bias.double().view(g, cg)
    s = torch.sigmoid(z)
    assert off(y, (z * s * live).view(b, t, w)) < bar
    assert off(stats[..., 0], mean.view(b, g)) < 2e-5
    assert off(stats[..., 1], (rstd * (n > 0).view(b, 1, 1, 1)).view(b, g)) < 2e-5
    dz = dy.double().view(b, t, g, cg) * s * (1 + z * (1 - s)) * live
    e = dz * weight.double().view(g, cg)
    want = rstd * (e - e.sum((1, 3), keepdim=True) / count - u * ((e * u).sum((1, 3), keepdim=True) / count)) * live
    assert off(dx, want.view(b, t, w)) < bar
    assert off(dw, (dz * u).sum((0, 1)).view(w)) < 2e-5 and off(db, dz.sum((0, 1)).view(w)) < 2e-5
