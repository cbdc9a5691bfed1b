"""The sequence encoder (paper_2608_02168_amd/encoder.py), its operators
together: rows, states and every gradient of two blocks against the oracle's
operators composed the same way, token by token against whole histories, and
a short training run.

Bar (max over elements of |error| / max(|value|, rms)): 1e-4 as for every
float32 operator, times the ten operators in a row; the gradients pass ten
more: 1e-3 and 2e-3."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import encoder as ref
from paper_2608_02168_amd import api, encoder
from tests.helpers import parity_err

pytestmark = pytest.mark.gpu


def host(t):
    return t.double().cpu().numpy()


def split(cfg, qkv):
    x = qkv.reshape(qkv.shape[0], -1, cfg.d_head)
    return x[:, :cfg.heads], x[:, cfg.heads:cfg.heads + cfg.kv_heads], x[:, cfg.heads + cfg.kv_heads:]


def oracle_forward(cfg, params, plan, x, pos, lens):
    b, t, d = x.shape
    g, tab = host(plan["log_decay"]), host(plan["table"])
    x = x.reshape(-1, d)
    saved, states = [], []
    for p in params:
        p = {k: host(v) for k, v in p.items()}
        qkv = ref.linear(x, p["W_qkv"], p["b_qkv"])
        q, k, v = split(cfg, qkv)
        qr, kr = (ref.norm_rope(y, w, tab, pos.reshape(-1)) for y, w in ((q, p["w_q"]), (k, p["w_k"])))
        four = [y.reshape(b, t, *y.shape[1:]) for y in (qr, kr, v)]
        o, s = ref.linattn(*four, g, plan["scale"], lens)
        o = o.reshape(-1, d)
        y = ref.linear(o, p["W_o"], None, x)
        h = ref.glu(y, p["W_g"])
        saved.append((p, x, q, k, four, o, y, h))
        x = ref.linear(h, p["W_d"], None, y)
        states.append(s)
    return x.reshape(b, t, d), saved, states


def oracle_backward(cfg, plan, saved, dz, pos, lens):
    b, t, d = dz.shape
    gl, tab = host(plan["log_decay"]), host(plan["table"])
    g, grads = dz.reshape(-1, d), []
    for p, x, q, k, four, o, y, h in reversed(saved):
        w = {}
        dh, w["W_d"], _ = ref.linear_bwd(h, p["W_d"], None, g)
        dy, w["W_g"], _ = ref.glu_bwd(y, p["W_g"], None, dh)
        dy = dy + g
        do, w["W_o"], _ = ref.linear_bwd(o, p["W_o"], None, dy)
        dq, dk, dv, _ = ref.linattn_bwd(*four, gl, do.reshape(b, t, cfg.heads, -1), plan["scale"], lens)
        dq, dk, dv = (v.reshape(b * t, -1, cfg.d_head) for v in (dq, dk, dv))
        dq, w["w_q"] = ref.norm_rope_bwd(q, p["w_q"], tab, pos.reshape(-1), dq)
        dk, w["w_k"] = ref.norm_rope_bwd(k, p["w_k"], tab, pos.reshape(-1), dk)
        dqkv = np.concatenate([dq, dk, dv], 1).reshape(b * t, -1)
        dx, w["W_qkv"], w["b_qkv"] = ref.linear_bwd(x, p["W_qkv"], p["b_qkv"], dqkv)
        g = dx + dy
        grads.append(w)
    return g.reshape(b, t, d), grads[::-1]


def test_two_blocks_against_the_oracle():
    cfg = encoder.EncoderConfig(d=64, heads=4, kv_heads=2, f=72, blocks=2, n_pos=500)
    params, plan = encoder.make_params(cfg, 3), encoder.make_plan(cfg)
    for p in params:
        p["w_q"].uniform_(0.5, 1.5)
        p["w_k"].uniform_(0.5, 1.5)
        p["b_qkv"].normal_(std=0.3)
    x, pos, lens, _ = encoder.make_histories(1, 5, 70, cfg.d)
    z, saved, states = encoder.forward(cfg, params, plan, x, pos, lens)
    rz, rsaved, rstates = oracle_forward(cfg, params, plan, host(x), pos.cpu().numpy(), lens.cpu().numpy())
    assert parity_err(host(z), rz) <= 1e-3
    for s, r in zip(states, rstates):
        assert parity_err(host(s), r) <= 1e-3
    dz = torch.randn(z.shape, generator=torch.Generator().manual_seed(2)).cuda()
    dx, grads = encoder.backward(cfg, params, plan, saved, dz)
    rdx, rgrads = oracle_backward(cfg, plan, rsaved, host(dz), pos.cpu().numpy(), lens.cpu().numpy())
    assert parity_err(host(dx), rdx) <= 2e-3
    for g, r in zip(grads, rgrads):
        assert set(g) == set(r) == set(encoder.PARAMS)
        for n in encoder.PARAMS:
            assert parity_err(host(g[n]), r[n]) <= 2e-3, n
    twice = [{n: w.clone() for n, w in g.items()} for g in grads]
    encoder.backward(cfg, params, plan, saved, dz, grads=twice)
    for g, h in zip(grads, twice):
        for n in encoder.PARAMS:
            assert parity_err(host(h[n]), 2 * host(g[n])) <= 1e-6, n


@pytest.mark.parametrize("dtype,bar", [(torch.float32, 1e-3), (torch.bfloat16, 0.15)])
def test_tokens_one_by_one(dtype, bar):
    """bfloat16: some twenty roundings of 2^-9 a token, on other values in the two ways."""
    cfg = encoder.EncoderConfig(dtype=dtype)
    params, plan = encoder.make_params(cfg, 3), encoder.make_plan(cfg)
    x, pos, _, _ = encoder.make_histories(1, 6, 40, cfg.d)
    x = x.to(dtype)
    whole, _, states = encoder.forward(cfg, params, plan, x, pos)
    slots = torch.tensor([7, 2, 0, 5, 1, 4], dtype=torch.int32, device="cuda")
    held = [torch.zeros(8, cfg.heads, cfg.d_head, cfg.d_head, device="cuda") for _ in params]
    for i in range(40):
        z = encoder.step(cfg, params, plan, x[:, i].contiguous(), pos[:, i].contiguous(), held, slots)
        assert parity_err(host(z), host(whole[:, i])) <= bar
    for s, h in zip(states, held):
        assert parity_err(host(h[slots.long()]), host(s)) <= bar
        assert not h[[3, 6]].any()


def test_training_learns():
    losses, _, _, _ = encoder.train(encoder.EncoderConfig(), 120)
    assert all(np.isfinite(losses)) and np.mean(losses[-10:]) < 0.75 * np.mean(losses[:5])


def test_a_given_stream_owns_what_a_call_allocates(monkeypatch):
    """Workspace and outputs come from the stream that the call runs on: memory of
    the caller's current stream could be handed out again while that one still works."""
    side = torch.cuda.Stream()
    seen, empty = [], torch.empty

    def spy(*a, **k):
        seen.append(torch.cuda.current_stream())
        return empty(*a, **k)

    x, w = torch.randn(300, 203, device="cuda"), torch.randn(203, 106, device="cuda")
    q, k = torch.randn(2, 1500, 2, 16, device="cuda"), torch.randn(2, 1500, 1, 16, device="cuda")
    g, one, pos = torch.full((2,), -0.1, device="cuda"), torch.ones(16, device="cuda"), torch.arange(8, device="cuda").int()
    b, states = torch.zeros(106, device="cuda"), torch.zeros(2, 2, 16, 16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(torch, "empty", spy)
    table = api.hg_rope_table(8, 16, stream=side)
    y = api.hg_linear_fwd(x, w, act=api.HG_ACT_SILU, stream=side)
    h = api.hg_glu_fwd(x, w, stream=side)
    api.hg_linear_bwd(x, w, b, y, act=api.HG_ACT_SILU, stream=side)
    api.hg_glu_bwd(x, w, b, h, stream=side)
    qt, kt = q[0, :8], k[0, :8]
    api.hg_qk_norm_rope_fwd(qt, kt, one, one, table, pos, stream=side)
    api.hg_qk_norm_rope_bwd(qt, kt, one, one, table, pos, qt, kt, stream=side)
    api.hg_linattn_fwd(q, k, k, g, want_state=True, stream=side)
    api.hg_linattn_bwd(q, k, k, g, q, stream=side)
    api.hg_linattn_step(q[:, 0], k[:, 0], k[:, 0], g, states, stream=side)
    assert len(seen) >= 10 and all(s == side for s in seen)
    torch.cuda.synchronize()
