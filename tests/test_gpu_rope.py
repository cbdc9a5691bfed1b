"""GPU parity of the norm and position rotation of queries and keys
(hg_rope_table, hg_qk_norm_rope_*) against the oracle (float64).

Bars (max over elements of |error| / max(|value|, rms)): float32 1e-5: the
norm, a product and a rotation are some ten roundings of 2^-24 on values of
the row's own size; bfloat16 5e-3: one rounding to 2^-9.  Weight gradients
sum up to 40000 float32 terms: 1e-4."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder
from paper_2608_02168_amd import api
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
BAR = {F32: 1e-5, BF16: 5e-3}


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def problem(n, hq, hk, d, rot, dtype, packed, weights=True, n_pos=300, seed=1):
    if packed:
        x = normal(seed, n, hq + 2 * hk + 1, d, dtype=dtype, scale=2.0)
        q, k = x[:, 1:1 + hq], x[:, 1 + hq:1 + hq + hk]
    else:
        q, k = normal(seed, n, hq, d, dtype=dtype, scale=2.0), normal(seed + 1, n, hk, d, dtype=dtype)
    wq, wk = (1 + 0.3 * normal(seed + 2, d), 1 + 0.3 * normal(seed + 3, d)) if weights else (None, None)
    table = api.hg_rope_table(n_pos, rot)
    pos = torch.from_numpy(np.random.default_rng(seed).integers(0, n_pos, n).astype(np.int32)).cuda()
    return q, (k if hk else None), wq, wk, table, pos


SHAPES = [(1, 1, 1, 8, 8), (7, 3, 1, 16, 8), (33, 4, 4, 64, 64), (129, 12, 3, 80, 40), (50, 5, 0, 96, 96),
          (1000, 8, 2, 128, 64), (77, 2, 2, 256, 256), (20, 33, 1, 24, 0), (300, 16, 4, 32, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("n,hq,hk,d,rot", SHAPES)
def test_forward_and_backward(n, hq, hk, d, rot, dtype, inter):
    packed = n % 2 == 1
    q, k, wq, wk, table, pos = problem(n, hq, hk, d, rot, dtype, packed, weights=n != 300)
    tab, p = encoder.rope_table(300, rot), pos.cpu().numpy()
    assert np.max(np.abs(host(table) - tab), initial=0) < 1e-7
    oq, ok = api.hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos, eps=1e-5, interleaved=inter)
    assert parity_err(host(oq), encoder.norm_rope(host(q), host(wq), tab, p, 1e-5, inter)) <= BAR[dtype]
    if hk:
        assert parity_err(host(ok), encoder.norm_rope(host(k), host(wk), tab, p, 1e-5, inter)) <= BAR[dtype]
    gq, gk = normal(8, n, hq, d, dtype=dtype), (normal(9, n, hk, d, dtype=dtype) if hk else None)
    dq, dk, dwq, dwk = api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, gq, gk, eps=1e-5, interleaved=inter)
    rx, rw = encoder.norm_rope_bwd(host(q), host(wq), tab, p, host(gq), 1e-5, inter)
    assert parity_err(host(dq), rx) <= BAR[dtype]
    if wq is not None:
        assert parity_err(host(dwq), rw) <= 1e-4
    if hk:
        rx, rw = encoder.norm_rope_bwd(host(k), host(wk), tab, p, host(gk), 1e-5, inter)
        assert parity_err(host(dk), rx) <= BAR[dtype]
        if wk is not None:
            assert parity_err(host(dwk), rw) <= 1e-4
    elif wk is not None:
        assert not dwk.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_accumulate(dtype):
    q, k, wq, wk, table, pos = problem(201, 6, 2, 64, 64, dtype, True)
    oq, ok = api.hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos)
    q1, k1 = q.clone(), k.clone()
    api.hg_qk_norm_rope_fwd(q1, k1, wq, wk, table, pos, q_out=q1, k_out=k1)
    assert torch.equal(q1, oq) and torch.equal(k1, ok)
    gq, gk = normal(8, 201, 6, 64, dtype=dtype), normal(9, 201, 2, 64, dtype=dtype)
    dq, dk, dwq, dwk = api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, gq, gk)
    a, b = torch.full_like(dwq, 2.0), torch.full_like(dwk, 3.0)
    grads = torch.zeros(201, 10, 64, dtype=dtype, device="cuda")  # a packed gradient, written in place
    grads[:, :6], grads[:, 6:8] = gq, gk
    api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, grads[:, :6], grads[:, 6:8], dq=grads[:, :6], dk=grads[:, 6:8],
                            dwq=a, dwk=b, accumulate=True)
    assert torch.equal(grads[:, :6], dq) and torch.equal(grads[:, 6:8], dk) and not grads[:, 8:].any()
    assert torch.equal(a, 2.0 + dwq) and torch.equal(b, 3.0 + dwk)


def test_positions_outside_the_table_and_zero_rows():
    q, k, wq, wk, table, pos = problem(10, 2, 1, 32, 16, F32, False)
    pos[3], pos[7] = -1, 300
    q[5] = 0
    oq, ok = api.hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos)
    bad = torch.zeros(10, dtype=torch.bool, device="cuda")
    bad[3] = bad[7] = True
    assert oq[bad].isnan().all() and ok[bad].isnan().all()
    assert oq[~bad].isfinite().all() and ok[~bad].isfinite().all() and not oq[5].any()


def test_large_positions_and_steps():
    """Angles are formed in float64: a table far from position zero keeps its accuracy."""
    table = api.hg_rope_table(200_000, 32, base=500.0, step=0.25)
    ref = encoder.rope_table(200_000, 32, 500.0, 0.25)
    assert np.max(np.abs(host(table) - ref)) < 1e-7


def test_no_tokens():
    q, k, wq, wk, table, pos = problem(0, 2, 1, 32, 16, F32, False)
    oq, ok = api.hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos)
    assert oq.shape == (0, 2, 32) and ok.shape == (0, 1, 32)
    _, _, dwq, dwk = api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, oq, ok)
    assert not dwq.any() and not dwk.any()


def test_weight_gradient_against_differences():
    q, k, wq, wk, table, pos = problem(6, 2, 1, 16, 16, F32, False)
    gq, gk = normal(8, 6, 2, 16), normal(9, 6, 1, 16)
    _, _, dwq, _ = api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, gq, gk)
    tab, p = encoder.rope_table(300, 16), pos.cpu().numpy()
    for c in (0, 7, 15):
        e = np.zeros(16)
        e[c] = 1e-6
        f = [(encoder.norm_rope(host(q), host(wq) + s * e, tab, p, 1e-6) * host(gq)).sum() for s in (1, -1)]
        assert abs((f[0] - f[1]) / 2e-6 - float(dwq[c])) < 1e-4


def test_refusals():
    q, k, wq, wk, table, pos = problem(10, 2, 1, 32, 16, BF16, False)

    def refused(code, *a, **kw):
        with pytest.raises(api.HgError) as e:
            api.hg_qk_norm_rope_fwd(*a, **kw)
        assert e.value.status == code

    refused(api.HG_ERR_ARG, q, k, wq, wk, table, pos, eps=-1.0)
    refused(api.HG_ERR_ARG, q, k, wq, wk, api.hg_rope_table(10, 40), pos)        # rot > d
    refused(api.HG_ERR_UNSUPPORTED, q, k, wq, wk, api.hg_rope_table(10, 12), pos)  # not a multiple of 8
    wide = normal(1, 10, 2, 40, dtype=BF16)
    refused(api.HG_ERR_ARG, wide[:, :, 4:36], k, wq, wk, table, pos)             # not 16-byte aligned
    z = normal(1, 10, 2, 20, dtype=BF16)
    refused(api.HG_ERR_UNSUPPORTED, z, None, None, None, api.hg_rope_table(10, 8), pos)
    with pytest.raises(api.HgError):
        api.hg_rope_table(10, 7)
    with pytest.raises(ValueError):
        api.hg_qk_norm_rope_fwd(q, k, wq, wk, table, pos.long())
    with pytest.raises(ValueError):
        api.hg_qk_norm_rope_fwd(q, k, wq[:16], wk, table, pos)
    with pytest.raises(TypeError):
        api.hg_qk_norm_rope_fwd(q, k.float(), wq, wk, table, pos)
    with pytest.raises(ValueError):
        api.hg_qk_norm_rope_bwd(q, k, wq, wk, table, pos, q, k, accumulate=True)
