"""GPU parity of the orthogonalised update (hg_muon_step) against the oracle
(float64): wide, tall and square matrices, odd sizes, single rows and columns,
batches, matrices of low rank, of zeros and of extreme sizes, replayed graphs.

With W = 0, lr scale = 1 and no momentum, W becomes -X itself.  Bars, by the norm
of the difference over the norm of X.  A rounding e of the 2 + 3 steps products'
operands (2^-22 in two parts, the float32 sums' sqrt(k / 32) 2^-24 beside it;
2^-12 in one) enters X next to entries of X's own size, where a step takes it up
by at most p = 3.4445 while it brings X's norm up by as much until its singular
values are near 1: no more than a few of the roundings' sum.  float32: 3e-5.
bfloat16: 2^-9 of the written value by norm and 1.2e-2 where strong directions
lie over noise of a thirtieth of their size, whose singular values that rounding
meets unscaled; 5e-3 for matrices of independent values."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def host(t):
    return t.double().cpu().numpy()


def off(got, want):
    return np.linalg.norm(host(got) - want) / max(np.linalg.norm(want), 1e-300)


def directions(seed, m, n, dtype):
    r = max(1, min(m, n) // 8)
    u = normal(seed, m, r) * torch.linspace(1.0, 0.1, r).cuda()
    return (u @ normal(seed + 1, r, n) * r ** -0.5 + 0.03 * normal(seed + 2, m, n)).to(dtype)


SIZES = [(1, 1), (1, 50), (50, 1), (3, 5), (16, 16), (17, 64), (64, 64), (65, 63), (63, 200), (128, 128), (129, 257), (200, 517),
         (517, 200), (256, 1000), (1030, 70), (300, 300), (640, 1111), (32, 900), (31, 33), (64, 700), (128, 350), (100, 97),
         (1100, 90), (33, 1400), (1500, 140), (64, 544), (64, 545), (32, 1184), (448, 128), (449, 128), (129, 128), (2100, 130)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n", SIZES)
def test_orthogonalised(m, n, dtype):
    for G, wide in ((normal(1, m, n, dtype=dtype), 5e-3), (directions(2, m, n, dtype), 1.2e-2)):
        W, M = torch.zeros_like(G), torch.zeros(m, n).cuda()
        api.hg_muon_step(W, G, M, lr=1.0, mu=0.0, nesterov=False, scale=1.0)
        assert off(-W, rec.orthogonal(host(G))) < (3e-5 if dtype is F32 else wide)
        assert torch.equal(M, G.float())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("steps", [0, 1, 2, 5])
def test_the_whole_update(steps, nesterov, dtype):
    m, n = 40, 72
    W, G, M = normal(1, m, n, dtype=dtype), normal(2, m, n, dtype=dtype), normal(3, m, n)
    want_w, want_m = rec.muon_step(host(W), host(G), host(M), 0.3, 0.9, 0.1, nesterov, steps, 0.7)
    api.hg_muon_step(W, G, M, lr=0.3, mu=0.9, weight_decay=0.1, nesterov=nesterov, steps=steps, scale=0.7)
    assert off(W, want_w) < (1e-5 if dtype is F32 else 2.0 ** -9 + 1e-3) and off(M, want_m) < 2.0 ** -23


def test_default_scale():
    for m, n, s in ((64, 16, 2.0), (16, 64, 1.0)):
        G = normal(1, m, n)
        W, V = torch.zeros_like(G), torch.zeros_like(G)
        api.hg_muon_step(W, G, torch.zeros_like(G), lr=1.0)
        api.hg_muon_step(V, G, torch.zeros_like(G), lr=1.0, scale=s)
        assert torch.equal(W, V)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count,m,n", [(5, 33, 70), (9, 128, 128), (3, 517, 200), (200, 8, 24)])
def test_matrices_of_a_call_are_apart(count, m, n, dtype):
    """Each as if alone, and one that holds a NaN or an infinity spoils itself only, as a whole."""
    W, G, M = normal(1, count, m, n, dtype=dtype), normal(2, count, m, n, dtype=dtype), normal(3, count, m, n)
    each = [(W[k].clone(), M[k].clone()) for k in range(count)]
    w0, m0 = W.clone(), M.clone()
    api.hg_muon_step(W, G, M, lr=0.1)
    for k, (w, mom) in enumerate(each):
        api.hg_muon_step(w, G[k], mom, lr=0.1, scale=max(1.0, m / n) ** 0.5)
        assert torch.equal(W[k], w) and torch.equal(M[k], mom)
    G[0, m // 2, n // 3], G[2, 0, 0] = float("nan"), float("inf")
    W2, M2 = w0, m0
    api.hg_muon_step(W2, G, M2, lr=0.1)
    assert torch.isnan(W2[0]).all() and torch.isnan(W2[2]).all()
    good = [k for k in range(count) if k not in (0, 2)]
    assert torch.equal(W2[good], W[good]) and torch.equal(M2[good], M[good])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extreme_sizes(dtype):
    m, n = 24, 40
    zero = torch.zeros(m, n, dtype=dtype).cuda()
    W = normal(1, m, n, dtype=dtype)
    V = W.clone()
    api.hg_muon_step(W, zero, torch.zeros(m, n).cuda(), lr=1.0)
    assert torch.equal(W, V)  # no gradient, no step
    G = normal(2, m, n)
    for size in (2.0 ** -100, 2.0 ** -20, 2.0 ** 100):
        X = torch.zeros(m, n, dtype=dtype).cuda()
        api.hg_muon_step(X, (G * size).to(dtype), torch.zeros(m, n).cuda(), lr=1.0, mu=0.0, eps=1e-36)
        assert off(-X, rec.orthogonal(host((G * size).to(dtype)), eps=1e-36)) < (3e-5 if dtype is F32 else 5e-3)
    # one entry far above the rest, and a matrix of rank one
    G = G.clone()
    G[3, 4] = 1000.0
    for g in (G, normal(3, m, 1) @ normal(4, 1, n)):
        X = torch.zeros(m, n, dtype=dtype).cuda()
        api.hg_muon_step(X, g.to(dtype), torch.zeros(m, n).cuda(), lr=1.0, mu=0.0)
        # noise of 2^-22 (2^-12) of the norm is taken up by 3.4445^5 = 485 beside a few directions of size one
        assert off(-X, rec.orthogonal(host(g.to(dtype)))) < 485 * (2.0 ** -21 if dtype is F32 else 2.0 ** -11)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_steps_and_a_given_workspace(dtype):
    """Every singular value stays in the range that the stored parts rely on; a workspace's old contents do not matter."""
    m, n = 90, 150
    G = normal(1, m, n, dtype=dtype)
    ws = torch.full((api.hg_muon_workspace_size(1, m, n, dtype, 32),), 0xFF, dtype=torch.uint8).cuda()  # NaNs
    W, V = torch.zeros_like(G), torch.zeros_like(G)
    api.hg_muon_step(W, G, torch.zeros(m, n).cuda(), lr=1.0, steps=32, ws=ws)
    s = torch.linalg.svdvals(W.double().cpu())
    assert 0.6 < s.min() and s.max() < 1.25
    api.hg_muon_step(V, G, torch.zeros(m, n).cuda(), lr=1.0, steps=32)
    assert torch.equal(W, V)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n", [(48, 80), (300, 170)])
def test_replayed_graph(m, n, dtype):
    W, G, M = normal(1, m, n, dtype=dtype), normal(2, m, n, dtype=dtype), torch.zeros(m, n).cuda()
    w, mom = W.clone(), M.clone()
    api.hg_muon_step(w.clone(), G, mom.clone(), lr=0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.hg_muon_step(W, G, M, lr=0.1)
    for k in range(3):
        G.copy_(normal(5 + k, m, n))
        graph.replay()
        torch.cuda.synchronize()
        api.hg_muon_step(w, G, mom, lr=0.1)
        assert torch.equal(W, w) and torch.equal(M, mom)


# tiles of 256 x 256 and 128 x 128, symmetric products of 128 x 128 with and without parts of k, several rounds of tiles
LARGE = [(2048, 6400, BF16), (6403, 2050, BF16), (1024, 8192, F32), (8190, 1030, F32), (2100, 2100, F32), (1500, 3001, BF16),
         (520, 4100, F32), (1037, 1041, F32)]


@pytest.mark.parametrize("m,n,dtype", LARGE)
def test_large_tiles(m, n, dtype):
    """Against the same formula by torch in float64 on the device; the whole matrix and its worst 64 x 64 block, so
    that no single tile is off."""
    G = normal(1, m, n, dtype=dtype)
    W = torch.zeros_like(G)
    api.hg_muon_step(W, G, torch.zeros(m, n).cuda(), lr=1.0, mu=0.0, scale=1.0)
    p, q, s = rec.COEF
    X = G.double()
    X /= X.norm()
    for _ in range(5):
        A = X @ X.T if m <= n else X.T @ X
        B = q * A + s * (A @ A)
        X = p * X + (B @ X if m <= n else X @ B)
    bar = 3e-5 if dtype is F32 else 5e-3
    d = -W.double() - X
    assert float(d.norm() / X.norm()) < bar
    pad = torch.nn.functional.pad(d.square(), (0, -n % 64, 0, -m % 64))
    blocks = pad.view(-(-m // 64), 64, -(-n // 64), 64).sum((1, 3))
    assert float(blocks.max().sqrt()) < 4 * bar * 64 * float(X.square().mean().sqrt())
