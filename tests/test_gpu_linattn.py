"""GPU parity of linear attention with a decay for each head (hg_linattn_*)
against the oracle (token by token, float64): lengths from zero to several
segments, ragged batches, shared key heads, states in and out, decays from none
to total, strided heads, the backward, and single tokens.

Bars (max over elements of |error| / max(|value|, rms)): float32 1e-4, the
library's bar for float32 products; bfloat16 2e-2: o, P and the state's copy are
each rounded to 2^-9 relative, and the largest of many thousand such errors
stays below five times their sum.  States are float32 sums of exact products
in both types: 1e-4."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
BAR = {F32: 1e-4, BF16: 2e-2}


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def decays(h):
    """No decay at all, slow ones, a fast one and one that keeps nothing, as many as there are heads."""
    g = torch.tensor([-0.02, 0.0, -0.3, -1e-3, -9.0, float("-inf"), -0.1, -0.005])
    return g[:h].cuda() if h <= 8 else -torch.logspace(-3, 0, h).cuda()


def problem(b, t, h, hk, d, dtype, seed=1):
    """Queries by themselves, keys and values in one packed buffer."""
    q = normal(seed, b, t, h, d, dtype=dtype)
    kv = normal(seed + 1, b, t, 2 * hk, d, dtype=dtype)
    return q, kv[:, :, :hk], kv[:, :, hk:], decays(h)


def lens_of(kind, b, t):
    if kind is None:
        return None
    x = np.random.default_rng(3).integers(0, t + 1, b)
    x[0] = {"ragged": t, "empty": 0, "wild": t + 5}[kind]
    if kind == "wild" and b > 1:
        x[1] = -3
    return torch.from_numpy(x.astype(np.int32)).cuda()


# t: one token, below a chunk, a chunk, one more, several chunks, several segments
CASES = [(2, 1, 4, 2, 16, None), (3, 5, 2, 2, 8, "ragged"), (2, 32, 4, 1, 32, "ragged"), (2, 33, 2, 2, 64, "empty"),
         (1, 64, 3, 3, 80, None), (2, 65, 2, 1, 128, "wild"), (2, 130, 4, 2, 96, "ragged"), (1, 700, 2, 2, 64, None),
         (2, 1100, 2, 1, 128, "ragged"), (3, 600, 8, 8, 16, "empty"), (2, 257, 3, 1, 24, "wild"),
         (1, 900, 2, 1, 40, None), (70, 20, 4, 4, 16, "ragged")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("b,t,h,hk,d,lens", CASES)
def test_forward(b, t, h, hk, d, lens, dtype, state):
    q, k, v, g = problem(b, t, h, hk, d, dtype)
    L = lens_of(lens, b, t)
    S0 = normal(5, b, h, d, d, scale=2.0) if state else None
    if L is not None:  # rows past the end are not read
        for i, n in enumerate(L.clamp(0, t).tolist()):
            q[i, n:], k[i, n:], v[i, n:] = float("nan"), float("inf"), float("nan")
    o = torch.full_like(q, 7.0)
    o, S = api.hg_linattn_fwd(q, k, v, g, scale=0.3, lens=L, state=S0, o=o, want_state=True)
    ro, rS = encoder.linattn(np.nan_to_num(host(q)), np.nan_to_num(host(k), posinf=0), np.nan_to_num(host(v)), host(g),
                             0.3, None if L is None else L.cpu().numpy(), host(S0))
    assert parity_err(host(o), ro) <= BAR[dtype]
    assert parity_err(host(S), rS) <= 1e-4
    if L is not None:
        for i, n in enumerate(L.clamp(0, t).tolist()):
            assert not o[i, n:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("b,t,h,hk,d,lens", CASES)
def test_backward(b, t, h, hk, d, lens, dtype, state):
    q, k, v, g = problem(b, t, h, hk, d, dtype)
    L = lens_of(lens, b, t)
    S0, dS = (normal(5, b, h, d, d, scale=2.0), normal(6, b, h, d, d)) if state else (None, None)
    do = normal(7, b, t, h, d, dtype=dtype)
    if L is not None:
        for i, n in enumerate(L.clamp(0, t).tolist()):
            q[i, n:], do[i, n:] = float("inf"), float("nan")
    got = api.hg_linattn_bwd(q, k, v, g, do, scale=0.3, lens=L, state=S0, dstate_out=dS)
    ref = encoder.linattn_bwd(np.nan_to_num(host(q), posinf=0), host(k), host(v), host(g), np.nan_to_num(host(do)), 0.3,
                              None if L is None else L.cpu().numpy(), host(S0), host(dS))
    for name, x, r in zip(("dq", "dk", "dv"), got, ref):
        assert parity_err(host(x), r) <= BAR[dtype], name
    if state:
        assert parity_err(host(got[3]), ref[3]) <= 1e-4
    else:
        assert got[3] is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,h,hk,d,slots", [(1, 1, 1, 8, 0), (5, 4, 2, 16, 9), (3, 2, 1, 128, 3), (64, 8, 8, 64, 0),
                                            (7, 3, 1, 80, 11), (2, 2, 2, 32, 2), (700, 2, 1, 24, 0), (1, 2, 2, 40, 0)])
def test_step(b, h, hk, d, slots, dtype):
    packed = normal(1, b, h + 2 * hk, d, dtype=dtype)
    q, k, v = packed[:, :h], packed[:, h:h + hk], packed[:, h + hk:]
    g = decays(h)
    S = normal(2, slots or b, h, d, d, scale=2.0)
    at = None
    if slots:
        at = np.random.default_rng(1).permutation(slots)[:b].astype(np.int32)
        if b > 2:
            at[1], at[2] = -1, slots  # idle rows
    ro, rS = encoder.linattn_step(host(q), host(k), host(v), host(g), host(S), at, 0.5)
    o = api.hg_linattn_step(q, k, v, g, S, None if at is None else torch.from_numpy(at).cuda(), scale=0.5)
    assert parity_err(host(o), ro) <= (1e-5 if dtype == F32 else 5e-3)
    assert parity_err(host(S), rS) <= 1e-5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_then_tokens(dtype):
    """A prompt's state carried on token by token gives the whole sequence."""
    b, t, h, hk, d = 2, 150, 4, 2, 32
    q, k, v, g = problem(b, t, h, hk, d, dtype)
    o, S = api.hg_linattn_fwd(q, k, v, g, scale=0.2, want_state=True)
    n = 140
    p, S1 = api.hg_linattn_fwd(q[:, :n], k[:, :n], v[:, :n], g, scale=0.2, want_state=True)
    out = [p]
    for i in range(n, t):
        out.append(api.hg_linattn_step(q[:, i], k[:, i], v[:, i], g, S1, scale=0.2)[:, None])
    assert parity_err(host(torch.cat(out, 1)), host(o)) <= BAR[dtype]
    assert parity_err(host(S1), host(S)) <= 1e-4


def test_gradients_against_differences():
    b, t, h, hk, d = 1, 70, 2, 1, 8
    q, k, v, g = problem(b, t, h, hk, d, F32)
    S0, dS, do = normal(5, b, h, d, d), normal(6, b, h, d, d), normal(7, b, t, h, d)
    dq, dk, dv, dS0 = (host(x) for x in api.hg_linattn_bwd(q, k, v, g, do, scale=0.4, state=S0, dstate_out=dS))
    X = [host(q), host(k), host(v), host(S0)]

    def loss(X):
        o, S = encoder.linattn(X[0], X[1], X[2], host(g), 0.4, None, X[3])
        return (o * host(do)).sum() + (S * host(dS)).sum()

    for i, (grad, at) in enumerate(((dq, (0, 69, 1, 3)), (dk, (0, 0, 0, 2)), (dv, (0, 33, 0, 7)), (dS0, (0, 0, 2, 5)))):
        e = []
        for s in (1e-5, -1e-5):
            Y = [x.copy() for x in X]
            Y[i][at] += s
            e.append(loss(Y))
        assert abs((e[0] - e[1]) / 2e-5 - grad[at]) <= 1e-4 * max(1, abs(grad[at]))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_that_are_not_finite(dtype):
    """A NaN in a key reaches its own and later tokens only, and of its head alone."""
    b, t, h, d = 1, 200, 2, 32
    q, k, v, g = problem(b, t, h, h, d, dtype)
    clean, _ = api.hg_linattn_fwd(q, k, v, g)
    k = k.clone()
    k[0, 101, 0, 3] = float("nan")
    o, _ = api.hg_linattn_fwd(q, k, v, g)
    assert torch.equal(o[:, :, 1], clean[:, :, 1]) and torch.equal(o[:, :101], clean[:, :101])
    assert o[0, 101:, 0].isnan().all()


# two heads of a key head in one block of the backward: with the key head's gradient whole in the block, as one of
# several partial ones, in segments, and an odd number of heads on a key head
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,h,hk,d,lens", [(700, 40, 4, 2, 16, "ragged"), (700, 33, 4, 1, 16, "wild"),
                                             (350, 70, 6, 2, 32, None), (20, 4500, 4, 2, 16, "ragged"),
                                             (8, 1450, 4, 2, 80, "empty"), (3, 4100, 2, 1, 128, "ragged")])
def test_backward_of_many_shared_heads(b, t, h, hk, d, lens, dtype):
    test_backward(b, t, h, hk, d, lens, dtype, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_that_are_not_finite_in_v(value, dtype):
    """A value of v that is not finite reaches its own column of its own and later tokens."""
    b, t, h, d = 1, 200, 2, 32
    q, k, v, g = problem(b, t, h, h, d, dtype)
    clean, _ = api.hg_linattn_fwd(q, k, v, g)
    v = v.clone()
    v[0, 101, 0, 3] = value
    o, _ = api.hg_linattn_fwd(q, k, v, g)
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[:, 101:, 0, 3] = True
    assert torch.equal(o[~hit], clean[~hit])
    assert not o[hit].isfinite().any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,h,hk,d", [(1, 200, 2, 2, 32), (700, 40, 4, 2, 16)])
def test_gradients_that_are_not_finite(b, t, h, hk, d, dtype):
    """A NaN in a token's upstream row, key or query reaches the gradients that depend on it and no other."""
    q, k, v, g = problem(b, t, h, hk, d, dtype)
    g = torch.full_like(g, -0.02)
    do = normal(7, b, t, h, d, dtype=dtype)
    clean = api.hg_linattn_bwd(q, k, v, g, do)[:3]
    at = 21
    for which in ("do", "q", "k", "v"):
        x = dict(q=q.clone(), k=k.clone(), v=v.clone(), do=do.clone())
        x[which][0, at, 0, 3] = float("nan")
        got = api.hg_linattn_bwd(x["q"], x["k"], x["v"], g, x["do"])[:3]
        # rows of dq, dk and dv that the value reaches, by the formulas
        one, none, before, after = (at, at + 1), (0, 0), (0, at + 1), (at, t)
        rows = dict(do=(one, before, before), q=(none, before, before), k=(after, none, one), v=(after, one, none))[which]
        heads = (h // hk if which in "kv" else 1, 1, 1)  # of dq: all that share the key head
        for a, c, (lo, hi), n in zip(got, clean, rows, heads):
            hit = torch.zeros_like(a, dtype=torch.bool)
            hit[0, lo:hi, :n] = True
            assert not a[hit].isfinite().all() or lo == hi, which
            assert torch.equal(a[~hit], c[~hit]), which


def test_deterministic_other_stream_and_graph():
    b, t, h, hk, d = 1, 2000, 4, 2, 64
    q, k, v, g = problem(b, t, h, hk, d, BF16)
    do = normal(7, b, t, h, d, dtype=BF16)
    first = api.hg_linattn_bwd(q, k, v, g, do)[:3]
    out = [torch.empty_like(x) for x in first]
    ws = torch.empty(api.hg_linattn_bwd_workspace_size(b, t, h, hk, d, BF16), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        api.hg_linattn_bwd(q, k, v, g, do, dq=out[0], dk=out[1], dv=out[2], ws=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(out, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for x in out:
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, first))


def test_no_tokens_and_no_sequences():
    q, k, v, g = problem(2, 0, 2, 2, 16, F32)
    S0 = normal(5, 2, 2, 16, 16)
    o, S = api.hg_linattn_fwd(q, k, v, g, state=S0, want_state=True)
    assert o.shape == (2, 0, 2, 16) and torch.equal(S, S0)
    q, k, v, g = problem(0, 5, 2, 2, 16, F32)
    o, S = api.hg_linattn_fwd(q, k, v, g, want_state=True)
    assert o.shape == (0, 5, 2, 16) and S.shape == (0, 2, 16, 16)


def test_refusals():
    q, k, v, g = problem(2, 20, 4, 2, 16, BF16)

    def refused(code, f, *a, **kw):
        with pytest.raises(api.HgError) as e:
            f(*a, **kw)
        assert e.value.status == code

    refused(api.HG_ERR_ARG, api.hg_linattn_fwd, q[:, :, :3], k, v, g[:3])        # 3 heads on 2
    x = normal(1, 2, 20, 4, 20, dtype=BF16)
    refused(api.HG_ERR_UNSUPPORTED, api.hg_linattn_fwd, x, x, x, g)
    x = normal(1, 2, 20, 4, 136, dtype=BF16)
    refused(api.HG_ERR_UNSUPPORTED, api.hg_linattn_fwd, x, x, x, g)
    x = normal(1, 2, 20, 4, 24, dtype=BF16)
    refused(api.HG_ERR_ARG, api.hg_linattn_fwd, x[..., 4:20], k, v, g)           # not 16-byte aligned
    refused(api.HG_ERR_ARG, api.hg_linattn_fwd, q, k, v, g, o=q)
    S = normal(5, 2, 4, 16, 16)
    refused(api.HG_ERR_ARG, api.hg_linattn_fwd, q, k, v, g, state=S, state_out=S)
    refused(api.HG_ERR_ARG, api.hg_linattn_bwd, q, k, v, g, q, dq=q)
    refused(api.HG_ERR_ARG, api.hg_linattn_step, q[:, 0], k[:, 0], v[:, 0], g, S[:1])  # two rows, one state
    y, w, z, _ = problem(1, 2000, 4, 2, 16, BF16)
    refused(api.HG_ERR_CAPACITY, api.hg_linattn_fwd, y, w, z, g, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        api.hg_linattn_fwd(q, k, v[:, :10], g)
    with pytest.raises(ValueError):
        api.hg_linattn_fwd(q, k, v, g.double())
    with pytest.raises(ValueError):
        api.hg_linattn_fwd(q, k, v, g, state=S[:1])
    with pytest.raises(ValueError):
        api.hg_linattn_step(q[:, 0], k[:, 0], v[:, 0], g, S.bfloat16())
    with pytest.raises(TypeError):
        api.hg_linattn_fwd(q, k.float(), v, g)
