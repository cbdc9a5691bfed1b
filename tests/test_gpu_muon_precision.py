"""The orthogonalised update (hg_muon_step) of bfloat16 matrices is as exact as
that of float32 ones: the type of W and G is that of what is read and of the last
rounding, not of X.

With W = 0, lr scale = 1 and no momentum, W becomes X + d rounded to bfloat16, d
what the products are off by.  An entry of W is then within 2^-8 of its size of
X + d (half a step), so what |W - X| exceeds 2^-8 |X| by is at most (1 + 2^-8) |d|
in the entry, and in the norm over entries.  Bars on that, of the norm of X, as
for float32 matrices: 3e-5 where noise is at least a thirtieth of the strong
directions' size; below that and for rank one, where a rounding of 2^-22 meets
empty directions, which five steps take up by 3.4445^5 = 485: 485 2^-21."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import recurrent as rec
from paper_2608_02168_amd import api

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FEW = 485 * 2.0 ** -21


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def gradient(kind, m, n, seed=1):
    """Independent values; rank one; or min / 8 strong directions over noise of the given size."""
    if kind == "independent":
        return normal(seed, m, n)
    if kind == "rank one":
        return normal(seed, m, 1) @ normal(seed + 1, 1, n)
    r = max(1, min(m, n) // 8)
    return (normal(seed, m, r) * torch.linspace(1.0, 0.1, r)) @ normal(seed + 1, r, n) * r ** -0.5 + kind * normal(seed + 2, m, n)


def excess(W, X):
    """Norm of what the entries are off by beyond their rounding."""
    return np.linalg.norm((np.abs(W - X) - 2.0 ** -8 * np.abs(X)).clip(min=0))


KINDS = [("independent", 3e-5), (0.1, 3e-5), (1 / 30, 3e-5), (0.01, FEW), (0.003, FEW), (0.001, FEW), (0.0, FEW),
         ("rank one", FEW)]


# one block (rows of 32, 64, 128), tiles of 64 x 64, tall ones
@pytest.mark.parametrize("m,n", [(24, 40), (64, 96), (128, 256), (96, 128), (200, 517), (517, 200), (300, 300)])
@pytest.mark.parametrize("kind,bar", KINDS)
def test_bfloat16_matrices(kind, bar, m, n):
    G = gradient(kind, m, n).to(BF16).cuda()
    W, M = torch.zeros_like(G), torch.zeros(m, n).cuda()
    api.hg_muon_step(W, G, M, lr=1.0, mu=0.0, nesterov=False, scale=1.0)
    X = rec.orthogonal(G.double().cpu().numpy())
    assert excess(-W.double().cpu().numpy(), X) < bar * np.linalg.norm(X)


# tiles of 128 x 128 and 256 x 256, with parts of k, tall and odd sizes
@pytest.mark.parametrize("m,n", [(1024, 4096), (2050, 6403), (6403, 2050), (4096, 8192)])
@pytest.mark.parametrize("kind,bar", [("independent", 3e-5), (1 / 30, 3e-5), ("rank one", FEW)])
def test_large_bfloat16_matrices(kind, bar, m, n):
    G = gradient(kind, m, n).to(BF16).cuda()
    W, M = torch.zeros_like(G), torch.zeros(m, n).cuda()
    api.hg_muon_step(W, G, M, lr=1.0, mu=0.0, nesterov=False, scale=1.0)
    p, q, s = rec.COEF
    X = G.double()
    X /= X.norm()
    for _ in range(5):
        A = X @ X.T if m <= n else X.T @ X
        B = q * A + s * (A @ A)
        X = p * X + (B @ X if m <= n else X @ B)
    over = ((-W.double() - X).abs() - 2.0 ** -8 * X.abs()).clamp(min=0)
    assert float(over.norm() / X.norm()) < bar


@pytest.mark.parametrize("kind,bar", [("independent", 3e-5), (0.001, FEW)])
@pytest.mark.parametrize("m,n", [(96, 128), (517, 200), (1100, 1200)])
def test_both_types_alike(kind, bar, m, n):
    """Momentum, weight decay and all: bfloat16 weights are the float32 ones of the same values, rounded."""
    G, W = gradient(kind, m, n).to(BF16).cuda(), (normal(7, m, n) * max(m, n) ** -0.5).to(BF16).cuda()
    M = (0.5 * gradient(kind, m, n, 11)).cuda()
    W32, M32 = W.float(), M.clone()
    api.hg_muon_step(W, G, M, lr=0.5, mu=0.9, weight_decay=0.1, scale=2.0)
    api.hg_muon_step(W32, G.float(), M32, lr=0.5, mu=0.9, weight_decay=0.1, scale=2.0)
    assert torch.equal(M, M32)
    # either is off by its bar of the norm of X, whose singular values are at most 1.21
    assert excess(W.double().cpu().numpy(), W32.double().cpu().numpy()) < 2 * bar * 1.21 * min(m, n) ** 0.5


# many matrices of a size between: tiles of 64, 128 and 256, tall ones, sides that fill no tile, cut tiles of several
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count,m,n", [(16, 200, 4000), (16, 1000, 200), (64, 300, 700), (6, 640, 2500), (12, 700, 600),
                                       (33, 130, 900), (4, 1100, 2050), (16, 256, 3000), (3, 1500, 1400)])
def test_batches(count, m, n, dtype):
    G = torch.stack([gradient(("independent", 0.1, 1 / 30)[k % 3], m, n, 20 + 3 * k) for k in range(count)]).to(dtype).cuda()
    W, M = torch.zeros_like(G), torch.zeros(count, m, n).cuda()
    api.hg_muon_step(W, G, M, lr=1.0, mu=0.0, nesterov=False, scale=1.0)
    p, q, s = rec.COEF
    for k in range(count):
        X = G[k].double()
        X /= X.norm()
        for _ in range(5):
            A = X @ X.T if m <= n else X.T @ X
            B = q * A + s * (A @ A)
            X = p * X + (B @ X if m <= n else X @ B)
        d = (-W[k].double() - X).abs()
        if dtype is BF16:
            d = (d - 2.0 ** -8 * X.abs()).clamp(min=0)
        assert float(d.norm() / X.norm()) < 3e-5, k
