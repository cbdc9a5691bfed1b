"""GPU parity of the group norm with an activation (hg_group_norm_*) against the
oracle (float64): rows, histories and whole node sets, ragged lengths, groups
that fill no vector or wave, strided and unaligned rows, the backward, replayed
graphs.

Bars (max over elements of |error| / max(|value|, rms)).  Float32: the mean is
off by sqrt(n) 2^-24 of the values' size at most (n terms, joined in a tree), u
by that and some 2^-22, the activation by 2^-20: 2e-5 with the inputs' mean of up
to four deviations.  bfloat16 half a step of the written row, 2^-8, beside it.
Statistics and the weights' gradients (float32 sums of n terms of either sign,
whose size is sqrt(n)): 2e-5."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
BAR = {F32: 2e-5, BF16: 2e-5 + 2.0 ** -8}
ACTS = ["none", "relu", "silu", "gelu"]


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def lens_of(kind, b, t):
    if kind is None:
        return None
    x = np.random.default_rng(3).integers(0, t + 1, b)
    x[0] = {"ragged": t, "empty": 0, "wild": t + 5}[kind]
    if kind == "wild" and b > 1:
        x[1] = -3
    return torch.from_numpy(x.astype(np.int32)).cuda()


def inputs(b, t, w, dtype):
    x = (normal(1, b, t, w) * 0.7 + normal(2, w)).to(dtype)
    return x, 1 + 0.2 * normal(3, w), 0.5 * normal(4, w)


# b, t, width, groups, lens: rows (t = 1), groups of one channel, of odd widths, of a wave and more, histories,
# items of a block, chunks
CASES = [(1, 1, 1, 1, None), (7, 1, 64, 4, None), (300, 1, 96, 12, None), (5, 1, 75, 3, None), (33, 1, 1024, 16, None),
         (3, 1, 2048, 1, None), (2, 1, 8192, 2, None), (9, 1, 40, 40, None), (4, 1, 1000, 1, None), (17, 1, 60, 5, "ragged"),
         (6, 5, 32, 4, "ragged"), (64, 24, 64, 4, "ragged"), (5, 96, 200, 5, "wild"), (2, 100, 24, 3, "empty"),
         (3, 333, 48, 2, "ragged"), (40, 700, 16, 2, None), (1, 5000, 128, 8, None), (2, 9001, 40, 5, "ragged"),
         (1, 4000, 25, 1, None), (2, 3000, 1100, 11, "wild"), (1, 70000, 16, 16, None), (2, 20, 512, 2, "ragged"), (3, 7, 2048, 1, None),
         (2, 60, 300, 3, "wild"), (9, 3, 1000, 1, None), (1, 300, 1024, 1, None)]


def clear_of_kinks(x, w, b, groups, lens):
    """Channels whose z comes near 0 get another bias, so that the slopes of ReLU are the same in 32 and 64 bits."""
    z, _ = rec.group_norm_fwd(host(x), groups, host(w), host(b), "none", 1e-5, None if lens is None else lens.cpu().numpy())
    z = z.reshape(-1, z.shape[-1])
    shift = np.zeros(z.shape[1])
    for c in range(z.shape[1]):
        v = np.sort(z[:, c])
        gaps = np.diff(v)
        near = np.argmax(np.where(np.abs(v[:-1]) < 1, gaps, 0)) if len(v) > 1 else 0
        shift[c] = -(v[near] + v[near + 1]) / 2 if len(v) > 1 else 1.0
    return b + torch.from_numpy(shift).float().cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", range(len(CASES)))
def test_forward_and_backward(k, dtype):
    b, t, width, groups, lens = CASES[k]
    act = ACTS[(k + (dtype is BF16)) % 4]
    code = ACTS.index(act)
    x, w, bias = inputs(b, t, width, dtype)
    if width == groups and t == 1:
        x = x.float().round().to(dtype)  # (each value is its own mean, exactly)
    n = lens_of(lens, b, t)
    if act == "relu":
        bias = clear_of_kinks(x, w, bias, groups, n)
    lens_h = None if n is None else n.cpu().numpy()
    y, stats = api.hg_group_norm_fwd(x, groups, w, bias, act=code, lens=n, want_stats=True)
    want, want_st = rec.group_norm_fwd(host(x), groups, host(w), host(bias), act, 1e-5, lens_h)
    assert parity_err(host(y), want) < BAR[dtype]
    assert parity_err(host(stats)[..., 0], want_st[..., 0]) < BAR[F32]
    assert parity_err(host(stats)[..., 1], want_st[..., 1]) < BAR[F32]
    dy = normal(9, b, t, width, dtype=dtype)
    got = api.hg_group_norm_bwd(x, groups, w, bias, stats, dy, act=code, lens=n)
    ref = rec.group_norm_bwd(host(x), groups, host(w), host(bias), host(stats), host(dy), act, lens_h)
    # where a group is one value dx is 0, a difference of values of the size rstd dy w
    size = np.abs(host(stats)[..., 1]).max() if width // groups * t == 1 else 0.0
    if size:
        assert np.abs(host(got[0]) - ref[0]).max() < 1e-6 * size
    else:
        assert parity_err(host(got[0]), ref[0]) < BAR[dtype]
    for name, p, q in (("dw", got[1], ref[1]), ("db", got[2], ref[2])):
        assert parity_err(host(p), q) < BAR[F32], name
    if n is not None:
        for s in range(b):
            m = min(max(int(lens_h[s]), 0), t)
            assert not y[s, m:].any() and not got[0][s, m:].any()
            if not m:
                assert not stats[s].any()


def test_rows_are_sequences_of_one_token():
    x, w, b = inputs(50, 1, 48, F32)
    y, s = api.hg_group_norm_fwd(x, 4, w, b, act=api.HG_ACT_SILU, want_stats=True)
    y2, s2 = api.hg_group_norm_fwd(x[:, 0], 4, w, b, act=api.HG_ACT_SILU, want_stats=True)
    assert torch.equal(y[:, 0], y2) and torch.equal(s, s2)
    d3 = api.hg_group_norm_bwd(x, 4, w, b, s, y, act=api.HG_ACT_SILU)
    d2 = api.hg_group_norm_bwd(x[:, 0], 4, w, b, s, y2, act=api.HG_ACT_SILU)
    assert torch.equal(d3[0][:, 0], d2[0]) and torch.equal(d3[1], d2[1]) and torch.equal(d3[2], d2[2])


@pytest.mark.parametrize("t", [1, 60, 20000])
def test_large_means_keep_their_digits(t):
    """A mean of 1000 deviations: squares are taken about it.  An input's own 2^-24 of 1000 is 6e-5 of a deviation;
    the values are whole quarters, so that there is no such rounding, and the mean's is 2^-24 1000 sqrt(2)."""
    x = torch.round(normal(1, 2, t, 64) * 4) / 4 + 1000.0
    y, stats = api.hg_group_norm_fwd(x, 2, want_stats=True)
    want, st = rec.group_norm_fwd(host(x), 2)
    assert np.abs(host(y) - want).max() < 4e-4
    assert parity_err(host(stats)[..., 1], st[..., 1]) < 1e-5


@pytest.mark.parametrize("t", [1, 30, 3000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_where_they_lie(t, dtype):
    b, width, groups = 3, 40, 5
    mem = normal(1, t + 2, b, width + 9, dtype=dtype)
    x = mem[1:t + 1, :, 3:3 + width].transpose(0, 1)
    out = torch.full((2, b, t + 1, width + 4), 7.0, dtype=dtype, device="cuda")
    y, dx = (out[k, :, :t, 1:1 + width] for k in range(2))
    w, bias, dy = 1 + 0.1 * normal(2, width), normal(3, width), normal(4, b, t, width, dtype=dtype)
    want, st = api.hg_group_norm_fwd(x.contiguous(), groups, w, bias, act=2, want_stats=True)
    _, st2 = api.hg_group_norm_fwd(x, groups, w, bias, act=2, y=y, want_stats=True)
    assert torch.equal(y, want) and torch.equal(st, st2)
    ref = api.hg_group_norm_bwd(x.contiguous(), groups, w, bias, st, dy, act=2)
    got = api.hg_group_norm_bwd(x, groups, w, bias, st, dy, act=2, dx=dx)
    assert all(torch.equal(p, q) for p, q in zip(got, ref))
    mask = torch.zeros_like(out, dtype=torch.bool)
    mask[:, :, :t, 1:1 + width] = True
    assert (out[~mask] == 7.0).all()


@pytest.mark.parametrize("t", [9, 2100])
def test_offsets_beyond_32_bits(t):
    """Rows up to 8.8 GB behind the first (a row past 2^32 bytes, in the same and in chunks of a sequence)."""
    width, far = 16, 1 << (21 if t > 1000 else 29)
    mem = torch.empty((t - 1) * far + 3 * width, dtype=BF16, device="cuda")
    x, y, dx = (mem.as_strided((1, t, width), (0, far, 1), k * width) for k in range(3))
    x.copy_(normal(1, 1, t, width))
    w, b, dy = 1 + 0.1 * normal(2, width), normal(3, width), normal(4, 1, t, width, dtype=BF16)
    want, st = api.hg_group_norm_fwd(x.contiguous(), 2, w, b, act=2, want_stats=True)
    api.hg_group_norm_fwd(x, 2, w, b, act=2, y=y)
    assert torch.equal(y, want)
    ref = api.hg_group_norm_bwd(x.contiguous(), 2, w, b, st, dy, act=2)
    got = api.hg_group_norm_bwd(x, 2, w, b, st, dy, act=2, dx=dx)
    assert all(torch.equal(p, q) for p, q in zip(got, ref)) and torch.equal(y, want)


@pytest.mark.parametrize("t", [1, 40, 6000])
def test_without_weights_and_accumulated(t):
    x, w, b = inputs(2, t, 32, F32)
    dy = normal(5, 2, t, 32)
    one, zero = torch.ones(32).cuda(), torch.zeros(32).cuda()
    y, st = api.hg_group_norm_fwd(x, 4, want_stats=True)
    assert torch.equal(y, api.hg_group_norm_fwd(x, 4, one, zero)[0])
    dx, dw, db = api.hg_group_norm_bwd(x, 4, None, None, st, dy)
    ref = api.hg_group_norm_bwd(x, 4, one, zero, st, dy)
    assert dw is None and db is None and torch.equal(dx, ref[0])
    aw, ab = ref[1].clone(), ref[2].clone()
    api.hg_group_norm_bwd(x, 4, one, zero, st, dy, dw=aw, db=ab, accumulate=True)
    assert torch.equal(aw, ref[1] + ref[1]) and torch.equal(ab, ref[2] + ref[2])


@pytest.mark.parametrize("t", [1, 50, 9000])
def test_values_that_are_not_finite_stay_in_their_group(t):
    x, w, b = inputs(3, t, 24, F32)
    clean, _ = api.hg_group_norm_fwd(x, 3, w, b, act=2)
    x[1, t // 2, 9] = float("nan")
    y, _ = api.hg_group_norm_fwd(x, 3, w, b, act=2)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, :, 8:16] = True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])
    n = torch.tensor([t, t // 2, t], dtype=torch.int32).cuda()
    y, st = api.hg_group_norm_fwd(x, 3, w, b, act=2, lens=n, want_stats=True)
    got = api.hg_group_norm_bwd(x, 3, w, b, st, x, act=2, lens=n)
    assert torch.isfinite(y).all() and torch.isfinite(st).all() and all(torch.isfinite(v).all() for v in got)


def test_backward_by_differences():
    b, t, width, groups = 2, 40, 24, 3
    x, w, bias = inputs(b, t, width, F32)
    dy = normal(9, b, t, width)
    n = torch.tensor([40, 17], dtype=torch.int32).cuda()
    _, st = api.hg_group_norm_fwd(x, groups, w, bias, act=3, lens=n, want_stats=True)
    got = api.hg_group_norm_bwd(x, groups, w, bias, st, dy, act=3, lens=n)

    def loss(p):
        return float((api.hg_group_norm_fwd(*p[:1], groups, *p[1:], act=3, lens=n)[0].double() * dy.double()).sum())

    at = [x, w, bias]
    for k in range(3):
        v, e = normal(20 + k, *at[k].shape), 2.0 ** -7
        hi, lo = (loss([p + s * e * v if q == k else p for q, p in enumerate(at)]) for s in (1, -1))
        want, have = (hi - lo) / (2 * e), float((got[k].double() * v.double()).sum())
        size = float(got[k].double().norm() * v.double().norm()) / v.numel() ** 0.5
        assert abs(want - have) < 2e-2 * size + 1e-3, k


def test_nothing_to_do():
    w = torch.ones(8).cuda()
    z = torch.empty(2, 0, 8).cuda()
    y, st = api.hg_group_norm_fwd(z, 2, w, w, want_stats=True)
    dx, dw, db = api.hg_group_norm_bwd(z, 2, w, w, st, z)
    assert y.shape == z.shape and not st.any() and not dw.any() and not db.any()
    z = torch.empty(0, 8).cuda()
    y, st = api.hg_group_norm_fwd(z, 2, w, w, want_stats=True)
    dx, dw, db = api.hg_group_norm_bwd(z, 2, w, w, st, z)
    assert y.shape == z.shape and not dw.any() and not db.any()


@pytest.mark.parametrize("t", [1, 8000])
def test_replayed_graph(t):
    x, w, b = inputs(3, t, 32, BF16)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    st, dw, db = torch.empty(3, 4, 2).cuda(), torch.empty(32).cuda(), torch.empty(32).cuda()

    def both():
        api.hg_group_norm_fwd(x, 4, w, b, act=2, y=y, stats=st)
        api.hg_group_norm_bwd(x, 4, w, b, st, y, act=2, dx=dx, dw=dw, db=db)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        x.copy_(normal(10 + k, 3, t, 32))
        graph.replay()
        torch.cuda.synchronize()
        want, s = api.hg_group_norm_fwd(x, 4, w, b, act=2, want_stats=True)
        ref = api.hg_group_norm_bwd(x, 4, w, b, s, want, act=2)
        assert torch.equal(y, want) and all(torch.equal(p, q) for p, q in zip((dx, dw, db), ref))
