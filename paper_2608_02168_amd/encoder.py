"""A sequence encoder over node histories, from the library's operators: what
the temporal module does for the last few states of a node, for histories of
any length.  One block is

    qkv = x W_qkv + b_qkv                                  hg_linear
    q, k = norm and position rotation of each head         hg_qk_norm_rope
    o = linear attention with a decay for each head        hg_linattn
    y = x + o W_o                                          hg_linear
    z = y + glu(y W_g) W_d                                 hg_glu, hg_linear

or, with ``mixer="recurrence"``, a gated recurrence in place of attention,

    x', r, i = x W_in + b_in                               hg_linear
    h = gated linear recurrence                            hg_recur
    o = silu(group norm of each token's heads of h)        hg_group_norm
    y = x + o W_o                                          hg_linear
    z = y + glu(y W_g) W_d                                 hg_glu, hg_linear

It runs over whole histories (``forward``, ``backward``) or on one new token of
each node with the states that it keeps (``step``).

``python -m paper_2608_02168_amd.encoder`` trains two blocks with the prediction
head on synthetic histories and then scores the same nodes token by token;
``--mixer recurrence`` takes the recurrence, ``--optimizer muon`` updates the
blocks' matrices along their orthogonalised momentum (hg_muon_step) and the
rest by Adam.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import numpy as np
import torch

from . import api

PARAMS = ("W_qkv", "b_qkv", "w_q", "w_k", "W_o", "W_g", "W_d")  # of an attention block
RECURRENT_PARAMS = ("W_in", "b_in", "decay", "w_n", "b_n", "W_o", "W_g", "W_d")


@dataclass(frozen=True)
class EncoderConfig:
    d: int = 64             # width of a state
    heads: int = 4
    kv_heads: int = 2
    f: int = 128            # width of the gated product
    blocks: int = 2
    n_pos: int = 4096       # positions (time steps) of the rotation table
    dtype: torch.dtype = torch.float32
    mixer: str = "attention"  # or "recurrence"
    rate: float = 8.0       # of the recurrence's gates

    def __post_init__(self):
        if self.mixer not in ("attention", "recurrence"):
            raise ValueError(f"{self}: no mixer {self.mixer}")
        if min(self.heads, self.kv_heads, self.f) < 1 or min(self.blocks, self.n_pos) < 0:
            raise ValueError(f"{self}: heads and widths are at least 1")
        if self.heads % self.kv_heads:
            raise ValueError(f"{self}: {self.heads} heads on {self.kv_heads} key heads")
        if self.d % self.heads or self.d_head % 8 or not 8 <= self.d_head <= 128:
            raise ValueError(f"{self}: d is not heads of a multiple of 8 up to 128 columns")
        # (the first decays are logarithms of exponentials of 0.2 / rate)
        if not 1e-3 <= self.rate < float("inf"):
            raise ValueError(f"{self}: a rate is finite and at least 0.001")

    @property
    def params(self) -> tuple:
        """The names of a block's weights."""
        return RECURRENT_PARAMS if self.mixer == "recurrence" else PARAMS

    @property
    def d_head(self) -> int:
        return self.d // self.heads

    @property
    def d_qkv(self) -> int:
        return (self.heads + 2 * self.kv_heads) * self.d_head


def make_params(cfg: EncoderConfig, seed: int, device="cuda") -> list:
    """One dict of weights per block: matrices Xavier-uniform in cfg.dtype (the
    two that write into the rows a tenth of that, so a block starts near the
    identity), vectors float32."""
    rng = np.random.default_rng(seed)

    def mat(a, b, size=1.0):
        r = size * (6.0 / (a + b)) ** 0.5
        return torch.from_numpy(rng.uniform(-r, r, (a, b)).astype(np.float32)).to(device, cfg.dtype)

    if cfg.mixer == "recurrence":
        # factors at r = 0 from 0.9 to 0.999: from channels that forget within ten steps to ones that hold a thousand
        a = torch.linspace(0.9, 0.999, cfg.d, dtype=torch.float64)
        decay = torch.log(torch.expm1(-2 * torch.log(a) / cfg.rate)).float().to(device)
        return [dict(W_in=mat(cfg.d, 3 * cfg.d), b_in=torch.zeros(3 * cfg.d, device=device), decay=decay.clone(),
                     w_n=torch.ones(cfg.d, device=device), b_n=torch.zeros(cfg.d, device=device),
                     W_o=mat(cfg.d, cfg.d, 0.1), W_g=mat(cfg.d, 2 * cfg.f), W_d=mat(cfg.f, cfg.d, 0.1))
                for _ in range(cfg.blocks)]
    return [dict(W_qkv=mat(cfg.d, cfg.d_qkv), b_qkv=torch.zeros(cfg.d_qkv, device=device),
                 w_q=torch.ones(cfg.d_head, device=device), w_k=torch.ones(cfg.d_head, device=device),
                 W_o=mat(cfg.d, cfg.d, 0.1), W_g=mat(cfg.d, 2 * cfg.f), W_d=mat(cfg.f, cfg.d, 0.1)) for _ in range(cfg.blocks)]


def make_plan(cfg: EncoderConfig, device="cuda") -> dict:
    """The rotation table and the heads' log-decays: from heads that forget
    within some ten steps to heads that hold hundreds."""
    back = torch.linspace(3.0, 8.0, cfg.heads, dtype=torch.float64)
    return dict(table=api.hg_rope_table(cfg.n_pos, cfg.d_head, device=device),
                log_decay=torch.log1p(-(2.0 ** -back)).float().to(device), scale=1.0 / cfg.d_head)


def _split(cfg: EncoderConfig, qkv):
    """Views of the heads in a packed projection [n, d_qkv]."""
    h, k = cfg.heads, cfg.kv_heads
    x = qkv.view(qkv.shape[0], h + 2 * k, cfg.d_head)
    return x[:, :h], x[:, h:h + k], x[:, h + k:]


def _gates(cfg: EncoderConfig, rows):
    """Views of the input and its two gates in a packed projection [..., 3 d]."""
    return rows[..., :cfg.d], rows[..., cfg.d:2 * cfg.d], rows[..., 2 * cfg.d:]


def _recurrent_forward(cfg, params, x, lens):
    b, t, d = x.shape
    saved, states = [], []
    x = x.reshape(b * t, d)
    for p in params:
        xri = api.hg_linear_fwd(x, p["W_in"], bias=p["b_in"])
        h, s = api.hg_recur_fwd(*_gates(cfg, xri.view(b, t, 3 * d)), p["decay"], rate=cfg.rate, lens=lens, want_state=True)
        o, stats = api.hg_group_norm_fwd(h.view(b * t, d), cfg.heads, p["w_n"], p["b_n"], act=api.HG_ACT_SILU, want_stats=True)
        y = api.hg_linear_fwd(o, p["W_o"], residual=x)
        f = api.hg_glu_fwd(y, p["W_g"])
        z = api.hg_linear_fwd(f, p["W_d"], residual=y)
        saved.append(dict(x=x, xri=xri, h=h, stats=stats, o=o, y=y, f=f))
        states.append(s)
        x = z
    return x.view(b, t, d), dict(blocks=saved, lens=lens, shape=(b, t)), states


def _recurrent_backward(cfg, params, saved, dz, grads, add):
    (b, t), lens, d = saved["shape"], saved["lens"], cfg.d
    g = dz.reshape(b * t, d)
    for p, s, w in zip(reversed(params), reversed(saved["blocks"]), reversed(grads)):
        df, _, _ = api.hg_linear_bwd(s["f"], p["W_d"], None, g, dW=w["W_d"], accumulate=add)
        dy, _, _ = api.hg_glu_bwd(s["y"], p["W_g"], None, df, dW=w["W_g"], accumulate=add)
        dy += g
        do, _, _ = api.hg_linear_bwd(s["o"], p["W_o"], None, dy, dW=w["W_o"], accumulate=add)
        dh, _, _ = api.hg_group_norm_bwd(s["h"].view(b * t, d), cfg.heads, p["w_n"], p["b_n"], s["stats"], do,
                                         act=api.HG_ACT_SILU, dw=w["w_n"], db=w["b_n"], accumulate=add)
        dxri = torch.empty_like(s["xri"])
        xs, ds = (_gates(cfg, v.view(b, t, 3 * d)) for v in (s["xri"], dxri))
        api.hg_recur_bwd(*xs, p["decay"], s["h"], dh.view(b, t, d), rate=cfg.rate, lens=lens, dx=ds[0], dr=ds[1], di=ds[2],
                         ddecay=w["decay"], accumulate=add)
        dx, _, _ = api.hg_linear_bwd(s["x"], p["W_in"], p["b_in"], dxri, dW=w["W_in"], dbias=w["b_in"], accumulate=add)
        g = dx.add_(dy)
    return g.view(b, t, d), grads


def _recurrent_step(cfg, params, x, states, slots):
    for p, s in zip(params, states):
        xri = api.hg_linear_fwd(x, p["W_in"], bias=p["b_in"])
        h = api.hg_recur_step(*_gates(cfg, xri), p["decay"], s, slots=slots, rate=cfg.rate)
        o, _ = api.hg_group_norm_fwd(h, cfg.heads, p["w_n"], p["b_n"], act=api.HG_ACT_SILU)
        y = api.hg_linear_fwd(o, p["W_o"], residual=x)
        f = api.hg_glu_fwd(y, p["W_g"])
        x = api.hg_linear_fwd(f, p["W_d"], residual=y, y=y)
    return x


def forward(cfg: EncoderConfig, params: list, plan: dict, x, pos, lens=None):
    """x [batch, t, d], pos int32 [batch, t] (the recurrence does not use it), lens
    int32 [batch] or None.  Returns (z, saved, states): the last block's rows, what
    ``backward`` needs, and every block's states after the histories [batch,
    heads, dh, dh] (of the recurrence [batch, d])."""
    if cfg.mixer == "recurrence":
        return _recurrent_forward(cfg, params, x, lens)
    b, t, d = x.shape
    saved, states = [], []
    x = x.reshape(b * t, d)
    pos = pos.reshape(-1)
    for p in params:
        qkv = api.hg_linear_fwd(x, p["W_qkv"], bias=p["b_qkv"])
        q, k, v = _split(cfg, qkv)
        qr, kr = api.hg_qk_norm_rope_fwd(q, k, p["w_q"], p["w_k"], plan["table"], pos)
        q4, k4, v4 = (y.unflatten(0, (b, t)) for y in (qr, kr, v))
        o, s = api.hg_linattn_fwd(q4, k4, v4, plan["log_decay"], scale=plan["scale"], lens=lens, want_state=True)
        o = o.view(b * t, d)
        y = api.hg_linear_fwd(o, p["W_o"], residual=x)
        h = api.hg_glu_fwd(y, p["W_g"])
        z = api.hg_linear_fwd(h, p["W_d"], residual=y)
        saved.append(dict(x=x, qkv=qkv, qr=qr, kr=kr, o=o, y=y, h=h))
        states.append(s)
        x = z
    return x.view(b, t, d), dict(blocks=saved, pos=pos, lens=lens, shape=(b, t)), states


def backward(cfg: EncoderConfig, params: list, plan: dict, saved: dict, dz, grads=None):
    """Returns (dx, grads): dz, dx [batch, t, d]; grads a list of dicts like
    params, added into when given."""
    add = grads is not None
    if not add:
        grads = [{n: torch.empty_like(w) for n, w in p.items()} for p in params]
    if cfg.mixer == "recurrence":
        return _recurrent_backward(cfg, params, saved, dz, grads, add)
    (b, t), pos, lens = saved["shape"], saved["pos"], saved["lens"]
    g = dz.reshape(b * t, cfg.d)
    for p, s, w in zip(reversed(params), reversed(saved["blocks"]), reversed(grads)):
        dh, _, _ = api.hg_linear_bwd(s["h"], p["W_d"], None, g, dW=w["W_d"], accumulate=add)
        dy, _, _ = api.hg_glu_bwd(s["y"], p["W_g"], None, dh, dW=w["W_g"], accumulate=add)
        dy += g
        do, _, _ = api.hg_linear_bwd(s["o"], p["W_o"], None, dy, dW=w["W_o"], accumulate=add)
        q, k, v = _split(cfg, s["qkv"])
        dqkv = torch.empty_like(s["qkv"])
        dq, dk, dv = _split(cfg, dqkv)
        q4, k4, v4, do4, dq4, dk4, dv4 = (y.unflatten(0, (b, t)) for y in
                                          (s["qr"], s["kr"], v, do.view(b * t, cfg.heads, cfg.d_head), dq, dk, dv))
        api.hg_linattn_bwd(q4, k4, v4, plan["log_decay"], do4, scale=plan["scale"], lens=lens, dq=dq4, dk=dk4, dv=dv4)
        api.hg_qk_norm_rope_bwd(q, k, p["w_q"], p["w_k"], plan["table"], pos, dq, dk, dq=dq, dk=dk, dwq=w["w_q"],
                                dwk=w["w_k"], accumulate=add)
        dx, _, _ = api.hg_linear_bwd(s["x"], p["W_qkv"], p["b_qkv"], dqkv, dW=w["W_qkv"], dbias=w["b_qkv"],
                                     accumulate=add)
        g = dx.add_(dy)
    return g.view(b, t, cfg.d), grads


def step(cfg: EncoderConfig, params: list, plan: dict, x, pos, states: list, slots=None):
    """One new token of each row: x [batch, d], pos int32 [batch]; states[i]
    [n, heads, dh, dh] of block i (of the recurrence [n, d]), updated in place
    (slots int32 [batch]: which one each row has).  Returns z [batch, d]."""
    if cfg.mixer == "recurrence":
        return _recurrent_step(cfg, params, x, states, slots)
    for p, s in zip(params, states):
        qkv = api.hg_linear_fwd(x, p["W_qkv"], bias=p["b_qkv"])
        q, k, v = _split(cfg, qkv)
        api.hg_qk_norm_rope_fwd(q, k, p["w_q"], p["w_k"], plan["table"], pos, q_out=q, k_out=k)
        o = api.hg_linattn_step(q, k, v, plan["log_decay"], s, slots=slots, scale=plan["scale"])
        y = api.hg_linear_fwd(o.view(x.shape), p["W_o"], residual=x)
        h = api.hg_glu_fwd(y, p["W_g"])
        x = api.hg_linear_fwd(h, p["W_d"], residual=y, y=y)
    return x


# ---- the example -------------------------------------------------------------

def make_histories(seed: int, batch: int, t: int, d: int, device="cuda"):
    """Synthetic histories: N(0, 1) states of lengths 1 .. t at growing time
    steps; label 1 where the mean of the first column over the last ten steps
    is positive."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(batch, t, d)).astype(np.float32)
    lens = rng.integers(1, t + 1, batch).astype(np.int32)
    pos = np.cumsum(rng.integers(1, 4, (batch, t)), 1).astype(np.int32)
    label = np.array([x[i, max(0, n - 10):n, 0].mean() > 0 for i, n in enumerate(lens)]).astype(np.int8)
    return tuple(torch.from_numpy(v).to(device) for v in (x, pos, lens, label))


def train(cfg: EncoderConfig, steps: int, batch: int = 512, t: int = 96, seed: int = 0, lr: float = 1e-2,
          optimizer: str = "adam"):
    """Returns (losses, params, head, plan).  optimizer: "adam", or "muon" for the
    blocks' matrices along their orthogonalised momentum and Adam for the rest."""
    if optimizer not in ("adam", "muon"):
        raise ValueError(f"no optimizer {optimizer}")
    params, plan = make_params(cfg, seed), make_plan(cfg)
    rng = np.random.default_rng(seed + 1)
    head = {"W1": torch.from_numpy(rng.normal(size=(cfg.d, cfg.d)).astype(np.float32) * cfg.d ** -0.5).cuda(),
            "b1": torch.zeros(cfg.d, device="cuda"),
            "W2": torch.from_numpy(rng.normal(size=(cfg.d, 1)).astype(np.float32) * cfg.d ** -0.5).cuda(),
            "b2": torch.zeros(1, device="cuda")}
    tensors = [p[n] for p in params for n in cfg.params] + list(head.values())
    of_blocks = len(params) * len(cfg.params)
    moments = [(torch.zeros_like(w), torch.zeros_like(w)) for w in tensors]
    rows = torch.arange(batch, device="cuda")
    losses = []
    for i in range(1, steps + 1):
        x, pos, lens, label = make_histories(seed + 10 + i, batch, t, cfg.d)
        z, saved, _ = forward(cfg, params, plan, x, pos, lens)
        last = lens.long() - 1
        loss, dlast, hg = api.hg_mlp_bce_fwd_bwd(z[rows, last], head["W1"], head["b1"], head["W2"], head["b2"], label)
        dz = torch.zeros_like(z)
        dz[rows, last] = dlast
        _, grads = backward(cfg, params, plan, saved, dz)
        flat = [g[n] for g in grads for n in cfg.params] + [hg[n] for n in head]
        for k, (w, g, (m, v)) in enumerate(zip(tensors, flat, moments)):
            if optimizer == "muon" and k < of_blocks and w.dim() == 2:
                # weights are [inputs, outputs]: the published factor, for outputs over inputs
                api.hg_muon_step(w, g, m, lr=lr, scale=max(1.0, w.shape[1] / w.shape[0]) ** 0.5)
            else:
                api.hg_adam_step(w, g, m, v, i, lr=lr)
        losses.append(loss)
    return [float(x) for x in losses], params, head, plan


def main(argv=None):
    ap = argparse.ArgumentParser(description="Trains a sequence encoder, then runs it token by token.")
    ap.add_argument("--mixer", choices=("attention", "recurrence"), default="attention")
    ap.add_argument("--optimizer", choices=("adam", "muon"), default="adam")
    a = ap.parse_args(argv)
    cfg = EncoderConfig(mixer=a.mixer)
    losses, params, _, plan = train(cfg, 200, optimizer=a.optimizer)
    print(f"BCE over 200 steps: {np.mean(losses[:10]):.4f} (first ten) -> {np.mean(losses[-10:]):.4f} (last ten)")
    x, pos, _, _ = make_histories(5, 256, 64, cfg.d)
    whole, _, states = forward(cfg, params, plan, x, pos)
    held = [torch.zeros_like(s) for s in states]
    for i in range(x.shape[1]):
        z = step(cfg, params, plan, x[:, i].contiguous(), pos[:, i].contiguous(), held)
    err = float((z - whole[:, -1]).abs().max() / whole[:, -1].square().mean().sqrt())
    print(f"64 tokens one by one against the whole histories: largest difference {err:.1e} of the rms")


if __name__ == "__main__":
    main()
