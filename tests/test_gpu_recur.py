"""GPU parity of the gated linear recurrence (hg_recur_*) against the oracle
(token by token, float64): lengths from zero to several segments, ragged batches,
widths that fill no vector, states in and out, strided and unaligned rows, gates
at their ends, the backward, single tokens, replayed graphs.

Bars (max over elements of |error| / max(|value|, rms)).  Float32: a factor a is
off by a few 2^-24, and what reaches a token has passed min(t, 1 / (1 - a)) of
them, so (16 + that) 2^-23; the inputs' factors end at 0.9995.  bfloat16: half a
step of the written row, 2^-8, beside that.  Sums over tokens (ddecay) and
states are float32: the float32 bar."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bar(dtype, t):
    return (16 + min(t, 2000)) * 2.0 ** -23 + (2.0 ** -8 if dtype is BF16 else 0.0)


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def decays(w, rate=8.0):
    """Factors at r = 0 from 0.2 to 0.9995."""
    a = 1 - torch.logspace(np.log10(0.8), np.log10(5e-4), w, dtype=torch.float64)
    return torch.log(torch.expm1(-2 * torch.log(a) / rate)).float().cuda()


def problem(b, t, w, dtype, seed=1, packed=True):
    if packed:
        p = normal(seed, b, t, 3 * w, dtype=dtype)
        return p[..., :w], p[..., w:2 * w], p[..., 2 * w:]
    return tuple(normal(seed + k, b, t, w, dtype=dtype) for k in range(3))


def lens_of(kind, b, t):
    if kind is None:
        return None
    x = np.random.default_rng(3).integers(0, t + 1, b)
    x[0] = {"ragged": t, "empty": 0, "wild": t + 5}[kind]
    if kind == "wild" and b > 1:
        x[1] = -3
    return torch.from_numpy(x.astype(np.int32)).cuda()


# one token, below a run, a tile and one more, several tiles, segments; widths below and above a slab, odd ones
CASES = [(2, 1, 8, None, True), (3, 3, 5, "ragged", False), (2, 9, 64, "ragged", True), (2, 64, 67, "wild", True),
         (1, 65, 4, None, False), (2, 130, 30, "empty", True), (3, 257, 64, "ragged", True), (1, 700, 129, None, True),
         (1, 2100, 66, None, False), (2, 2500, 33, "wild", True), (130, 40, 16, "ragged", False),
         (70, 70, 4200, "ragged", True), (1030, 70, 16, "ragged", True), (1, 9000, 70, None, True)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,w,lens,state", CASES)
def test_forward_and_backward(b, t, w, lens, state, dtype):
    x, r, i = problem(b, t, w, dtype)
    n = lens_of(lens, b, t)
    s0, ds = (normal(7, b, w), normal(8, b, w)) if state else (None, None)
    g = decays(w)
    h, s1 = api.hg_recur_fwd(x, r, i, g, lens=n, state=s0, want_state=True)
    dh = normal(9, b, t, w, dtype=dtype)
    got = api.hg_recur_bwd(x, r, i, g, h, dh, lens=n, state=s0, dstate_out=ds)
    if b > 64:  # the oracle on some sequences
        keep = [0, 1, b - 1]
        x, r, i, h, dh = (v[keep] for v in (x, r, i, h, dh))
        s0, ds, s1, n = (None if v is None else v[keep] for v in (s0, ds, s1, n))
        got = [v[keep] if v is not None and v.shape[0] == b else None for v in got]
    lens_h = None if n is None else n.cpu().numpy()
    want_h, want_s = rec.recur_fwd(host(x), host(r), host(i), host(g), 8.0, lens_h, host(s0))
    assert parity_err(host(h), want_h) < bar(dtype, t)
    assert parity_err(host(s1), want_s) < bar(F32, t)
    want = rec.recur_bwd(host(x), host(r), host(i), host(g), 8.0, host(h), host(dh), lens_h, host(s0), host(ds))
    for k, name in enumerate(("dx", "dr", "di", "ddecay", "dstate")):
        if got[k] is not None:
            assert parity_err(host(got[k]), want[k]) < bar(dtype if k < 3 else F32, t), name
    if n is not None:
        for k in range(x.shape[0]):
            m = min(max(int(lens_h[k]), 0), t)
            assert not h[k, m:].any() and not any(v[k, m:].any() for v in got[:3])


def test_the_paths_are_exercised():
    """The sizes above reach the paths that they are there for: waves and blocks that walk a sequence need no
    workspace forward, tiles that compose through memory do."""
    size = api.hg_recur_fwd_workspace_size
    assert size(130, 40, 16) == size(1030, 70, 16) == size(70, 70, 4200) == 0
    assert min(size(1, 65, 4), size(2, 2500, 33), size(1, 9000, 70)) > 0


def test_results_do_not_depend_on_timing():
    """Tiles that compose through memory: the same bits each time, with other work beside them too."""
    b, t, w = 2, 9000, 100
    x, r, i = problem(b, t, w, F32)
    g, dh, n = decays(w), normal(4, b, t, w), lens_of("ragged", b, t)
    first = None
    other, side = torch.randn(4096, 4096).cuda(), torch.cuda.Stream()
    for k in range(6):
        if k % 2:
            with torch.cuda.stream(side):
                other @ other
        h, s = api.hg_recur_fwd(x, r, i, g, lens=n, want_state=True)
        out = [h, s] + [v for v in api.hg_recur_bwd(x, r, i, g, h, dh, lens=n) if v is not None]
        first = first or out
        assert all(torch.equal(p, q) for p, q in zip(first, out))
    torch.cuda.synchronize()


def test_two_calls_at_once():
    b, t, w = 1, 20000, 80
    x, r, i = problem(b, t, w, BF16)
    want, _ = api.hg_recur_fwd(x, r, i, decays(w))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [api.hg_recur_fwd(x, r, i, decays(w), stream=s)[0] for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(v, want) for v in got)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward_by_differences(dtype):
    """The gradient against differences of the kernel's own forward in float32."""
    b, t, w = 2, 300, 24
    x, r, i = problem(b, t, w, F32, packed=False)
    g, s0, ds, dh = decays(w), normal(7, b, w), normal(8, b, w), normal(9, b, t, w)
    if dtype is BF16:  # exactly representable inputs
        x, r, i, dh = (v.to(BF16).float() for v in (x, r, i, dh))
    h, _ = api.hg_recur_fwd(x, r, i, g, state=s0)
    args = [v.to(dtype) for v in (x, r, i)]
    got = api.hg_recur_bwd(*args, g, h.to(dtype), dh.to(dtype), state=s0, dstate_out=ds)

    def loss(p):
        y, s1 = api.hg_recur_fwd(*p[:3], p[3], state=p[4], want_state=True)
        return float((y.double() * dh.double()).sum() + (s1.double() * ds.double()).sum())

    at = [x, r, i, g, s0]
    for k in range(5):
        v = normal(20 + k, *at[k].shape)
        e = 2.0 ** -7
        hi, lo = (loss([p + s * e * v if q == k else p for q, p in enumerate(at)]) for s in (1, -1))
        want, have = (hi - lo) / (2 * e), float((got[k].double() * v.double()).sum())
        # the difference's error: e^2 / 6 times a third derivative of the size of the sum, and the rounding of
        # 2^-23 sqrt(n) |h| / e; for bfloat16 the gradients' own rounding, 2^-8 |grad| in a random direction
        size = float(got[k].double().norm() * v.double().norm()) / v.numel() ** 0.5
        assert abs(want - have) < size * (2e-2 if dtype is F32 else 3e-2) + 1e-3, k


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gates_at_their_ends(dtype):
    """Open and closed gates: a = 1 exactly passes the state on, and the gradients' limits are finite."""
    b, t, w = 2, 12, 8
    x, r, i = (v.clone() for v in problem(b, t, w, dtype, packed=False))
    r[:, 2] = -200.0          # a = 1: nothing enters
    r[:, 3] = 200.0           # sigmoid(r) = 1
    i[:, 4] = -200.0          # the input is shut out
    r[:, 5] = float("-inf")
    i[:, 6] = float("inf")
    g = decays(w)
    g[0], g[1], g[2] = -120.0, 60.0, -60.0  # a = 1 for every token; a = 0 unless r is very low; a next to 1
    s0, dh = normal(5, b, w), normal(6, b, t, w, dtype=dtype)
    h, s1 = api.hg_recur_fwd(x, r, i, g, state=s0, want_state=True)
    want, want_s = rec.recur_fwd(host(x), host(r), host(i), host(g), 8.0, None, host(s0))
    assert parity_err(host(h), want) < bar(dtype, t) and parity_err(host(s1), want_s) < bar(F32, t)
    assert torch.equal(h[:, :, 0], s0[:, None, 0].expand(b, t).to(dtype))
    got = api.hg_recur_bwd(x, r, i, g, h, dh, state=s0)
    ref = rec.recur_bwd(host(x), host(r), host(i), host(g), 8.0, host(h), host(dh), None, host(s0))
    for k in range(5):
        assert torch.isfinite(got[k]).all()
        assert parity_err(host(got[k]), ref[k]) < bar(dtype if k < 3 else F32, t), k


@pytest.mark.parametrize("b,t", [(3, 600), (1200, 100), (3, 20)])
def test_slopes_past_the_largest_number(b, t):
    """rate softplus(decay) beyond float32: a = 0, but 1 where sigmoid(r) = 0, and nothing from rows past the end."""
    w = 8
    x, r, i = (v.clone() for v in problem(b, t, w, F32, packed=False))
    r[:, 3] = float("-inf")
    g = decays(w)
    g[1] = 3e38
    lens = torch.full((b,), t - 7, dtype=torch.int32, device="cuda")
    s0, dh = normal(5, b, w), normal(6, b, t, w)
    h, s1 = api.hg_recur_fwd(x, r, i, g, lens=lens, state=s0, want_state=True)
    gated = (torch.sigmoid(i.double()) * x.double())[:, :, 1]
    want = gated.clone()
    want[:, 3] = gated[:, 2]
    want[:, t - 7:] = 0
    assert parity_err(host(h)[..., 1], host(want)) < bar(F32, 1) and parity_err(host(s1)[:, 1], host(want[:, t - 8])) < bar(F32, 1)
    for v in api.hg_recur_bwd(x, r, i, g, h, dh, lens=lens, state=s0):
        assert torch.isfinite(v).all()


def test_factors_next_to_one():
    """1 - a^2 far below 2^-24: the input's share keeps its digits."""
    b, t, w = 1, 400, 16
    x, r, i = problem(b, t, w, F32)
    g = torch.linspace(-40.0, -6.0, w).cuda()
    h, _ = api.hg_recur_fwd(x, r, i, g)
    want, _ = rec.recur_fwd(host(x), host(r), host(i), host(g), 8.0)
    for c in range(w):  # each channel by its own size
        assert parity_err(host(h)[..., c], want[..., c]) < bar(F32, t), c


def test_values_that_are_not_finite_stay_in_their_channel():
    b, t, w = 2, 600, 12
    x, r, i = (v.clone() for v in problem(b, t, w, F32, packed=False))
    clean, _ = api.hg_recur_fwd(x, r, i, decays(w))
    x[0, 300, 3] = float("nan")
    r[1, 20, 5] = float("nan")
    h, _ = api.hg_recur_fwd(x, r, i, decays(w))
    bad = torch.zeros(b, t, w, dtype=torch.bool).cuda()
    bad[0, 300:, 3] = True
    bad[1, 20:, 5] = True
    assert torch.equal(torch.isnan(h), bad) and torch.equal(h[~bad], clean[~bad])
    # rows past a length may hold anything
    n = torch.tensor([300, 20], dtype=torch.int32).cuda()
    h, s = api.hg_recur_fwd(x, r, i, decays(w), lens=n, want_state=True)
    got = api.hg_recur_bwd(x, r, i, decays(w), h, torch.where(bad, float("nan"), 1.0), lens=n)
    assert torch.isfinite(h).all() and torch.isfinite(s).all() and all(torch.isfinite(v).all() for v in got[:4])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_where_they_lie(dtype):
    """Odd strides, addresses aligned to a value only, token-major layouts, rows beside the outputs untouched."""
    b, t, w = 3, 77, 21
    mem = normal(1, 3, t + 2, b, w + 6, dtype=dtype)
    x, r, i = (mem[k, 1:t + 1, :, 3:3 + w].transpose(0, 1) for k in range(3))   # [b, t, w], token stride the larger
    out = torch.full((4, b, t + 1, w + 4), 7.0, dtype=dtype, device="cuda")
    h, dx, dr, di = (out[k, :, :t, 1:1 + w] for k in range(4))
    g, dh = decays(w), normal(3, b, t, w, dtype=dtype)
    want, _ = api.hg_recur_fwd(*(v.contiguous() for v in (x, r, i)), g)
    api.hg_recur_fwd(x, r, i, g, h=h)
    assert torch.equal(h, want)
    ref = api.hg_recur_bwd(*(v.contiguous() for v in (x, r, i)), g, want, dh)
    got = api.hg_recur_bwd(x, r, i, g, h, dh, dx=dx, dr=dr, di=di)
    assert all(torch.equal(p, q) for p, q in zip(got[:4], ref[:4]))
    mask = torch.zeros_like(out, dtype=torch.bool)
    mask[:, :, :t, 1:1 + w] = True
    assert (out[~mask] == 7.0).all()


@pytest.mark.parametrize("b", [1, 300])
def test_offsets_beyond_32_bits(b):
    """Tokens (or sequences) up to 8.8 GB behind the first."""
    t, w, far = (2100, 16, 1 << 21) if b == 1 else (16, 16, 1 << 24)
    strides = (0, far, 1) if b == 1 else (far, 8 * w, 1)
    mem = torch.empty((2100 if b == 1 else 300) * far, dtype=BF16, device="cuda")
    x, r, i, h, dx, dr, di = (mem.as_strided((b, t, w), strides, k * w) for k in range(7))
    for k, v in enumerate((x, r, i)):
        v.copy_(normal(k, b, t, w))
    g, dh = decays(w), normal(4, b, t, w, dtype=BF16)
    near = [v.contiguous() for v in (x, r, i)]
    want, s1 = api.hg_recur_fwd(*near, g, want_state=True)
    _, s2 = api.hg_recur_fwd(x, r, i, g, h=h, want_state=True)
    assert torch.equal(h, want) and torch.equal(s1, s2)
    ref = api.hg_recur_bwd(*near, g, want, dh)
    got = api.hg_recur_bwd(x, r, i, g, h, dh, dx=dx, dr=dr, di=di)
    assert all(torch.equal(p, q) for p, q in zip(got[:4], ref[:4])) and torch.equal(h, want)


def test_accumulated_decay_gradient():
    x, r, i = problem(5, 33, 10, F32)
    h, _ = api.hg_recur_fwd(x, r, i, decays(10))
    one = api.hg_recur_bwd(x, r, i, decays(10), h, x.contiguous())[3]
    into = one.clone()
    api.hg_recur_bwd(x, r, i, decays(10), h, x.contiguous(), ddecay=into, accumulate=True)
    assert torch.equal(into, one + one)
    empty = torch.ones(10).cuda()
    z = torch.empty(0, 4, 10).cuda()
    api.hg_recur_bwd(z, z, z, decays(10), z, z, ddecay=empty)
    assert not empty.any()


def test_no_tokens():
    z, g = torch.empty(3, 0, 8).cuda(), decays(8)
    s0, ds = normal(1, 3, 8), normal(2, 3, 8)
    h, s = api.hg_recur_fwd(z, z, z, g, state=s0, want_state=True)
    got = api.hg_recur_bwd(z, z, z, g, h, z, state=s0, dstate_out=ds)
    assert h.shape == (3, 0, 8) and torch.equal(s, s0) and torch.equal(got[4], ds) and not got[3].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,w", [(1, 4), (5, 67), (70, 130)])
def test_single_tokens(b, w, dtype):
    p = normal(1, b, 3 * w, dtype=dtype)
    x, r, i = p[:, :w], p[:, w:2 * w], p[:, 2 * w:]
    states, g = normal(2, b + 3, w), decays(w)
    slots = torch.randperm(b + 3, generator=torch.Generator().manual_seed(4))[:b].int().cuda()
    if b > 2:
        slots[1], slots[2] = -1, b + 3
    before = states.clone()
    h = api.hg_recur_step(x, r, i, g, states, slots=slots)
    want, after = rec.recur_step(host(x), host(r), host(i), host(g), 8.0, host(before), slots.cpu().numpy())
    assert parity_err(host(h), want) < bar(dtype, 1) and parity_err(host(states), after) < bar(F32, 1)
    idle = torch.ones(b + 3, dtype=torch.bool)
    idle[slots.long().cpu()[(slots >= 0).cpu() & (slots < b + 3).cpu()]] = False
    assert torch.equal(states[idle], before[idle])


def test_tokens_one_by_one_are_the_whole_history():
    b, t, w = 4, 50, 20
    x, r, i = problem(b, t, w, F32)
    s0 = normal(3, b, w)
    h, s1 = api.hg_recur_fwd(x, r, i, decays(w), state=s0, want_state=True)
    held = s0.clone()
    steps = [api.hg_recur_step(x[:, k], r[:, k], i[:, k], decays(w), held) for k in range(t)]
    assert parity_err(host(torch.stack(steps, 1)), host(h)) < bar(F32, t)
    assert parity_err(host(held), host(s1)) < bar(F32, t)


def test_replayed_graph_and_another_stream():
    b, t, w = 1, 3000, 40
    x, r, i = (v.clone() for v in problem(b, t, w, F32, packed=False))
    g, dh = decays(w), normal(4, b, t, w)
    h, dx, dr, di = (torch.empty_like(x) for _ in range(4))
    dg = torch.zeros_like(g)

    def both():
        api.hg_recur_fwd(x, r, i, g, h=h)
        api.hg_recur_bwd(x, r, i, g, h, dh, dx=dx, dr=dr, di=di, ddecay=dg)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        x.copy_(normal(10 + k, b, t, w))
        graph.replay()
        torch.cuda.synchronize()
        eh, _ = api.hg_recur_fwd(x, r, i, g)
        want = api.hg_recur_bwd(x, r, i, g, eh, dh)
        assert torch.equal(h, eh) and all(torch.equal(p, q) for p, q in zip((dx, dr, di, dg), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = api.hg_recur_fwd(x, r, i, g, stream=side)
    side.synchronize()
    assert torch.equal(got, eh)
