"""Outputs of the recurrence and the group norm as views of one packed buffer, in
every order of its dimensions: the same values as in buffers of their own, and
nothing beside them written."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
B, T, W = 3, 90, 24
# the order in memory of sequences, tokens and the three gradients (a row's channels lie together)
ORDERS = ["btg", "tbg", "bgt", "tgb", "gbt", "gtb"]


def normal(seed, *shape, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def views(order, dtype):
    """Three [B, T, W] views of a buffer whose rows have two values more than W, and that buffer."""
    mem = torch.full([{"b": B, "t": T, "g": 3}[k] for k in order] + [W + 2], 7.0, dtype=dtype, device="cuda")
    at = mem.permute(*[order.index(k) for k in "gbt"], 3)
    return [at[k, ..., 1:W + 1] for k in range(3)], mem


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ORDERS)
def test_packed_outputs(order, dtype):
    x, r, i, dh = (normal(k, B, T, W, dtype=dtype) for k in range(4))
    decay, s0 = torch.linspace(-6.0, 1.0, W).cuda(), normal(5, B, W, dtype=torch.float32)
    h, _ = api.hg_recur_fwd(x, r, i, decay, state=s0)
    want = api.hg_recur_bwd(x, r, i, decay, h, dh, state=s0)
    (dx, dr, di), mem = views(order, dtype)
    got = api.hg_recur_bwd(x, r, i, decay, h, dh, state=s0, dx=dx, dr=dr, di=di)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert (mem[..., 0] == 7.0).all() and (mem[..., -1] == 7.0).all()
    # the norm and its gradient beside its input
    (u, y, du), mem = views(order, dtype)
    u.copy_(x)
    want, stats = api.hg_group_norm_fwd(x, 3, act=api.HG_ACT_SILU, want_stats=True)
    api.hg_group_norm_fwd(u, 3, act=api.HG_ACT_SILU, y=y)
    api.hg_group_norm_bwd(u, 3, None, None, stats, dh, act=api.HG_ACT_SILU, dx=du)
    assert torch.equal(y, want) and torch.equal(u, x)
    assert torch.equal(du, api.hg_group_norm_bwd(x, 3, None, None, stats, dh, act=api.HG_ACT_SILU)[0])
    assert (mem[..., 0] == 7.0).all() and (mem[..., -1] == 7.0).all()
