"""The operators of a recurrent block of the sequence encoder and of its training,
as timed cases: the gated linear recurrence over whole histories (forward,
backward) and single tokens, the group norm with an activation over rows of
channels (forward, backward), and the optimiser step that orthogonalises the
momentum of a weight matrix.

``listed()`` names fixed cases, ``draw(rng)`` more of the same ranges;
``prepare`` makes the inputs that a program has in hand (all from the seed),
``run`` is one pass: with ``own`` through the public entry points of
``paper_2608_02168_amd.api``, without it in elementary torch operations in 32
bits (64 for the norm of a whole matrix), rounded once at the end.  ``work``
gives the bytes and operations that a pass cannot do without, ``exact`` the
outputs in float64 from the definitions.

The recurrence, for each channel c of a sequence:
    a_t = exp(-rate softplus(decay_c) sigmoid(r_t))
    h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t
The group norm, for each sequence (or each row where t = 1) and group of
adjacent channels, over its tokens and channels:
    y = act(w (x - mean) / sqrt(var + eps) + b)
The step, for each matrix W with gradient G and momentum M:
    M <- mu M + G,  U = G + mu M,  X = U / max(|U|, eps), and `steps` times
    A = X X^T,  X <- p X + (q A + s A A) X   with (p, q, s) = (3.4445, -4.7750, 2.0315)
    W <- (1 - lr wd) W - lr scale X
(X^T X and X (...) where W has more rows than columns).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
RATE, EPS = 8.0, 1e-5
MUON = dict(lr=0.02, mu=0.95, weight_decay=0.01, steps=5, scale=1.0, eps=1e-7)


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # serving: one new token for each of 64 sequences of 80 held ones
        dict(name="recur_token", kind="recur_step", dtype="bf16", batch=64, slots=80, width=1024),
        # one long history of a wide model: few channels, so the work has to be split over its length
        dict(name="recur_long", kind="recur_fwd", dtype="bf16", batch=1, t=65521, width=1024, ragged=False, state=True,
             packed=True),
        # a training batch whose histories differ in length, gates inside one packed projection
        dict(name="recur_train", kind="recur_bwd", dtype="bf16", batch=8, t=2048, width=2048, ragged=True, state=True,
             packed=True),
        # very many short float32 histories at the default width of the layers
        dict(name="recur_histories", kind="recur_bwd", dtype="f32", batch=8192, t=24, width=64, ragged=True, state=False,
             packed=True),
        # serving: rows of 16 tokens, heads of 64 channels
        dict(name="norm_token", kind="norm_fwd", dtype="bf16", batch=16, t=1, width=1024, groups=16, act="silu",
             ragged=False),
        # training: every token's heads by themselves
        dict(name="norm_train", kind="norm_bwd", dtype="bf16", batch=16384, t=1, width=1024, groups=16, act="silu",
             ragged=False),
        # all nodes of a subgraph at once: two sums over 200003 rows for each group
        dict(name="norm_nodes", kind="norm_bwd", dtype="f32", batch=1, t=200003, width=128, groups=8, act="gelu",
             ragged=False),
        # histories normalised over their length, widths and groups that fill no wave
        dict(name="norm_histories", kind="norm_fwd", dtype="f32", batch=512, t=96, width=200, groups=5, act="relu",
             ragged=True),
        # the weights of a layer's relations, all in one call
        dict(name="muon_relations", kind="muon", dtype="f32", count=8, rows=128, cols=128),
        # a projection of a small model, taller than wide, widths that fill no tile
        dict(name="muon_odd", kind="muon", dtype="bf16", count=3, rows=517, cols=200),
        # the gated product's matrix of a float32 model
        dict(name="muon_gated", kind="muon", dtype="f32", count=1, rows=1024, cols=5632),
        # a large matrix, bfloat16 weights and gradients
        dict(name="muon_wide", kind="muon", dtype="bf16", count=1, rows=4096, cols=8192),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 8, one time in four any number."""
    w = _between(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    kind = rng.choice(["recur_fwd", "recur_bwd", "recur_step", "norm_fwd", "norm_bwd", "muon", "muon"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "f32"]))
    if kind == "recur_step":
        width = _width(rng, 8, 4096)
        batch = _between(rng, 1, 2048)
        return dict(c, batch=batch, slots=batch + rng.randrange(0, 1 + batch // 4), width=width)
    if kind.startswith("recur"):
        width = _width(rng, 8, 2560)
        t = _between(rng, 1, 65536)
        batch = _between(rng, 1, max(1, min(8192, (1 << 25) // (t * width))))
        return dict(c, batch=batch, t=t, width=width, ragged=rng.random() < 0.5, state=rng.random() < 0.5,
                    packed=rng.random() < 0.5)
    if kind.startswith("norm"):
        groups = rng.choice([1, 2, 4, 5, 8, 16, 32])
        width = groups * rng.choice([1, 4, 8, 12, 16, 25, 32, 64, 64, 128])
        act = rng.choice(["none", "silu", "gelu"] + ["relu"] * (kind == "norm_fwd"))
        # a row, a history or all rows at a time
        t = rng.choice([1, 1, _between(rng, 2, 4096), _between(rng, 2, 262144)])
        batch = _between(rng, 1, max(1, min(65536, (1 << 25) // (t * width))))
        return dict(c, batch=batch, t=t, width=width, groups=groups, act=act, ragged=t > 1 and rng.random() < 0.5)
    a, b = _width(rng, 16, 4096), _width(rng, 16, 8192)
    if rng.random() < 0.4:
        a, b = b, a
    count = _between(rng, 1, max(1, min(64, (1 << 34) // (min(a, b) * a * b))))
    return dict(c, count=count, rows=a, cols=b)


# ---- inputs -----------------------------------------------------------------

def _type(case):
    return BF16 if case["dtype"] == "bf16" else F32


def _lens(case, g):
    """Lengths from a whole history down to none at all."""
    if not case["ragged"]:
        return None
    lens = torch.randint(0, case["t"] + 1, (case["batch"],), generator=g, device=DEV, dtype=torch.int32)
    lens[0] = case["t"]
    return lens


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = _type(case)

    def normal(*shape, scale=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device=DEV, dtype=F32) * scale).to(dtype or t)

    kind, s = case["kind"], {}
    if kind.startswith("recur"):
        b, w = case["batch"], case["width"]
        # factors at r = 0 from 0.9 to 0.999, spread over the channels: softplus(decay) = -log(a) / (rate / 2)
        a = torch.rand(w, generator=g, device=DEV, dtype=F64) * 0.099 + 0.9
        s["decay"] = torch.log(torch.expm1(-2 * torch.log(a) / RATE)).to(F32)
        if kind == "recur_step":
            x = normal(b, 3 * w)
            s["x"], s["r"], s["i"] = x[:, :w], x[:, w:2 * w], x[:, 2 * w:]
            s["states"] = normal(case["slots"], w, dtype=F32)
            s["slots"] = torch.randperm(case["slots"], generator=g, device=DEV)[:b].to(torch.int32)
            return s
        n = case["t"]
        if case["packed"]:
            x = normal(b, n, 3 * w)
            s["x"], s["r"], s["i"] = x[..., :w], x[..., w:2 * w], x[..., 2 * w:]
        else:
            s["x"], s["r"], s["i"] = (normal(b, n, w) for _ in range(3))
        s["lens"] = _lens(case, g)
        s["state"] = normal(b, w, dtype=F32) if case["state"] else None
        if kind == "recur_bwd":
            s["h"] = _recur(s, case)[0].to(t)
            s["dh"] = normal(b, n, w)
            s["dstate"] = normal(b, w, dtype=F32) if case["state"] else None
        return s
    if kind.startswith("norm"):
        b, n, w, q = case["batch"], case["t"], case["width"], case["groups"]
        s["x"] = (torch.randn(b, n, w, generator=g, device=DEV, dtype=F32) * (0.5 + torch.rand(w, generator=g, device=DEV))
                  + torch.randn(w, generator=g, device=DEV)).to(t)
        s["w"], s["b"] = 1.0 + normal(w, scale=0.1, dtype=F32), normal(w, scale=0.3, dtype=F32)
        s["lens"] = _lens(case, g)
        if kind == "norm_bwd":
            mean, rstd, _ = _moments(s, case)
            s["stats"] = torch.stack([mean.view(b, q), rstd.view(b, q)], -1).contiguous()
            s["dy"] = normal(b, n, w)
        return s
    k, m, n = case["count"], case["rows"], case["cols"]
    r = max(1, min(m, n) // 8)

    def gradient(size):
        # some strong directions over weaker noise in all of them
        u, v = normal(k, m, r, dtype=F32), normal(k, r, n, dtype=F32)
        u = u * torch.linspace(1.0, 0.1, r, device=DEV)
        return size * (u.matmul(v) * r ** -0.5 + normal(k, m, n, scale=0.1, dtype=F32))

    s["param"] = normal(k, m, n, scale=min(m, n) ** -0.5)
    s["grad"] = gradient(1e-3).to(t)
    s["momentum"] = gradient(5e-3)
    return s


def prepare(case, seed):
    return dict(_inputs(case, seed), case=case)


# ---- one pass -----------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2608_02168_amd import api
    c = s["case"]
    kind = c["kind"]
    if kind == "recur_step":
        h = api.hg_recur_step(s["x"], s["r"], s["i"], s["decay"], s["states"], slots=s["slots"], rate=RATE)
        return h, s["states"]
    if kind == "recur_fwd":
        return api.hg_recur_fwd(s["x"], s["r"], s["i"], s["decay"], rate=RATE, lens=s["lens"], state=s["state"],
                                want_state=True)
    if kind == "recur_bwd":
        return api.hg_recur_bwd(s["x"], s["r"], s["i"], s["decay"], s["h"], s["dh"], rate=RATE, lens=s["lens"],
                                state=s["state"], dstate_out=s["dstate"])
    if kind == "norm_fwd":
        return api.hg_group_norm_fwd(s["x"], c["groups"], s["w"], s["b"], act=ACTS[c["act"]], eps=EPS, lens=s["lens"],
                                     want_stats=True)
    if kind == "norm_bwd":
        return api.hg_group_norm_bwd(s["x"], c["groups"], s["w"], s["b"], s["stats"], s["dy"], act=ACTS[c["act"]],
                                     lens=s["lens"])
    api.hg_muon_step(s["param"], s["grad"], s["momentum"], nesterov=True, **MUON)
    return s["param"], s["momentum"]


# ---- the plain form -----------------------------------------------------------

def _live(s, c):
    """[b, t, 1]: the tokens inside their sequence."""
    t = torch.arange(c["t"], device=DEV)
    lens = s["lens"].long() if s["lens"] is not None else torch.full((c["batch"],), c["t"], device=DEV)
    return (t < lens[:, None])[..., None]


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _gates(s):
    """log of the factor a, its complement sqrt(1 - a^2), sigmoid(r), sigmoid(i), x: float32."""
    sr = torch.sigmoid(s["r"].float())
    log_a = -RATE * _softplus(s["decay"]) * sr
    return log_a, torch.sqrt(-torch.expm1(2 * log_a)), sr, torch.sigmoid(s["i"].float()), s["x"].float()


def _scan(a, b, back=False):
    """h_t = a_t h_{t-1} + b_t along dim 1 from h = 0 (back: from the end), by doubling: after
    a round, a and b stand for twice as many steps."""
    d = 1
    while d < a.shape[1]:
        near, far = (slice(None, -d), slice(d, None)) if back else (slice(d, None), slice(None, -d))
        a, b, a_old, b_old = a.clone(), b.clone(), a, b
        b[:, near] = a_old[:, near] * b_old[:, far] + b_old[:, near]
        a[:, near] = a_old[:, near] * a_old[:, far]
        d *= 2
    return b


def _recur(s, c):
    """h and the state after the last token, float32."""
    live = _live(s, c)
    log_a, q, _, si, x = _gates(s)
    a, u = torch.where(live, torch.exp(log_a), 1.0), torch.where(live, q * si * x, 0.0)
    if s["state"] is not None:
        u[:, 0] += a[:, 0] * s["state"]
    h = _scan(a, u)
    return h * live, h[:, -1]


def _plain_recur_bwd(s):
    c, t = s["case"], s["x"].dtype
    live = _live(s, c)
    log_a, q, sr, si, x = _gates(s)
    a = torch.exp(log_a)
    g = s["dh"].float() * live
    after = torch.where(live, a, 1.0)  # factor that takes the gradient over a token
    end = s["dstate"] if s["dstate"] is not None else torch.zeros(c["batch"], c["width"], device=DEV)
    # past the end of a sequence the gradient of the last state is carried to it
    g[:, -1] += end
    g = _scan(torch.cat([after[:, 1:], torch.ones_like(after[:, :1])], 1), g, back=True)
    dstate = after[:, 0] * g[:, 0] if s["state"] is not None else None
    first = s["state"] if s["state"] is not None else torch.zeros_like(end)
    before = torch.cat([first[:, None], s["h"][:, :-1].float()], 1)
    dlog = a * g * before - g * si * x * a * a / q
    dx, di = g * q * si, g * q * x * si * (1 - si)
    dr = dlog * log_a * (1 - sr)
    dsoft = torch.where(live, dlog * sr, 0.0).sum((0, 1))
    ddecay = -RATE * torch.sigmoid(s["decay"]) * dsoft
    return [torch.where(live, v, 0.0).to(t) for v in (dx, dr, di)] + [ddecay, dstate]


def _plain_recur_step(s):
    at = s["slots"].long()
    log_a, q, _, si, x = _gates(s)
    h = torch.exp(log_a) * s["states"][at] + q * si * x
    s["states"][at] = h
    return h.to(s["x"].dtype), s["states"]


def _moments(s, c):
    """mean and 1 / sqrt(var + eps) of each group [b, 1, groups, 1], and x by groups, float32."""
    b, n, w, q = c["batch"], c["t"], c["width"], c["groups"]
    x = s["x"].float().view(b, n, q, w // q)
    if s["lens"] is None:
        mean = x.mean((1, 3), keepdim=True)
        return mean, torch.rsqrt((x - mean).square().mean((1, 3), keepdim=True) + EPS), x
    live = _live(s, c)[..., None]
    some = (s["lens"] > 0).view(b, 1, 1, 1)
    count = (s["lens"].float() * (w // q)).clamp(min=1).view(b, 1, 1, 1)
    mean = torch.where(live, x, 0.0).sum((1, 3), keepdim=True) / count
    var = torch.where(live, x - mean, 0.0).square().sum((1, 3), keepdim=True) / count
    return mean, torch.where(some, torch.rsqrt(var + EPS), 0.0), x


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _act_grad(z, act):
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _plain_norm_fwd(s):
    c = s["case"]
    mean, rstd, x = _moments(s, c)
    z = ((x - mean) * rstd).flatten(2) * s["w"] + s["b"]
    y = _act(z, c["act"])
    if s["lens"] is not None:
        y = torch.where(_live(s, c), y, 0.0)
    return y.to(s["x"].dtype), torch.stack([mean.view(c["batch"], -1), rstd.view(c["batch"], -1)], -1)


def _plain_norm_bwd(s):
    c = s["case"]
    b, n, w, q = c["batch"], c["t"], c["width"], c["groups"]
    mean, rstd = (s["stats"][..., k].view(b, 1, q, 1) for k in (0, 1))
    xh = (s["x"].float().view(b, n, q, -1) - mean) * rstd
    z = xh.flatten(2) * s["w"] + s["b"]
    dz = s["dy"].float() * _act_grad(z, c["act"])
    count = torch.full((b, 1, 1, 1), float(n), device=DEV)
    if s["lens"] is not None:
        live = _live(s, c)
        dz, xh = torch.where(live, dz, 0.0), torch.where(live[..., None], xh, 0.0)
        count = s["lens"].float().clamp(min=1).view(b, 1, 1, 1)
    count = count * (w // q)
    dw, db = (dz * xh.flatten(2)).sum((0, 1)), dz.sum((0, 1))
    e = (dz * s["w"]).view(b, n, q, -1)
    dx = rstd * (e - e.sum((1, 3), keepdim=True) / count - xh * ((e * xh).sum((1, 3), keepdim=True) / count))
    dx = dx.flatten(2)
    if s["lens"] is not None:
        dx = torch.where(live, dx, 0.0)
    return dx.to(s["x"].dtype), dw, db


def _plain_muon(s):
    c, o = s["case"], MUON
    W, G, M = s["param"], s["grad"].float(), s["momentum"]
    M.mul_(o["mu"]).add_(G)
    X = G + o["mu"] * M
    size = X.double().square().sum((1, 2), keepdim=True).sqrt().clamp(min=o["eps"])
    X = X / size.float()
    tall = c["rows"] > c["cols"]
    if tall:
        X = X.transpose(1, 2).contiguous()
    for _ in range(o["steps"]):
        A = torch.stack([x @ x.t() for x in X])
        B = -4.7750 * A + 2.0315 * torch.stack([x @ x for x in A])
        X = 3.4445 * X + torch.stack([x @ y for x, y in zip(B, X)])
    if tall:
        X = X.transpose(1, 2)
    W.copy_((1 - o["lr"] * o["weight_decay"]) * W.float() - o["lr"] * o["scale"] * X)
    return W, M


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "recur_fwd":
        h, state = _recur(s, c)
        return h.to(s["x"].dtype), state
    return {"recur_bwd": _plain_recur_bwd, "recur_step": _plain_recur_step, "norm_fwd": _plain_norm_fwd,
            "norm_bwd": _plain_norm_bwd, "muon": _plain_muon}[kind](s)


# ---- what a pass cannot do without ---------------------------------------------

def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "recur_step":
        n = case["batch"] * case["width"]
        return {"bytes": n * (4 * e + 8) + 4 * case["width"], "flops": 20 * n}
    if kind.startswith("recur"):
        n, w = case["batch"] * case["t"] * case["width"], case["batch"] * case["width"]
        if kind == "recur_fwd":
            return {"bytes": 4 * e * n + 4 * w * (2 if case["state"] else 1), "flops": 20 * n}
        return {"bytes": 8 * e * n + 4 * w * (3 if case["state"] else 0), "flops": 45 * n}
    if kind.startswith("norm"):
        n, stats = case["batch"] * case["t"] * case["width"], 8 * case["batch"] * case["groups"]
        moves = 2 if kind == "norm_fwd" else 3
        return {"bytes": moves * e * n + stats + 8 * case["width"] * (moves - 1), "flops": 12 * (moves - 1) * n}
    k, m, n = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # the two symmetric products by halves
    return {"bytes": k * m * n * (3 * e + 8), "flops": k * MUON["steps"] * (3 * m * m * n + m ** 3)}


# ---- the definitions in float64 -------------------------------------------------

def _exact_recur(case, s):
    """Token by token, on [t, b, w]; past its end a sequence keeps its state."""
    b, n, w = case["batch"], case["t"], case["width"]
    x, r, i = (s[k].double().transpose(0, 1) for k in ("x", "r", "i"))
    lens = s["lens"] if s["lens"] is not None else torch.full((b,), n, device=DEV, dtype=torch.int32)
    live = (torch.arange(n, device=DEV)[:, None] < lens)[..., None].double()
    rho = RATE * torch.logaddexp(s["decay"].double(), torch.zeros(1, dtype=F64, device=DEV))
    S, I = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-i))
    a = torch.exp(-rho * S)
    q = torch.sqrt(-torch.expm1(-2 * rho * S))
    keep = a * live + (1 - live)
    first = s["state"].double() if s["state"] is not None else torch.zeros(b, w, dtype=F64, device=DEV)
    if case["kind"] == "recur_fwd":
        u = q * I * x * live
        h, out = first, torch.empty_like(u)
        for t in range(n):
            torch.addcmul(u[t], keep[t], h, out=out[t])
            h = out[t]
        return (out * live).transpose(0, 1), h.clone()
    dh = s["dh"].double().transpose(0, 1) * live
    R = s["dstate"].double() if s["dstate"] is not None else torch.zeros_like(first)
    g = torch.empty_like(dh)
    R = R.clone()
    for t in reversed(range(n)):
        torch.add(dh[t], R, out=g[t])
        torch.mul(keep[t], g[t], out=R)
    g = g * live
    before = torch.cat([first[None], s["h"].double().transpose(0, 1)[:-1]])
    # with l = log a: dh/dl = a h_before + I x dq/dl and dq/dl = -a^2 / q, dl/dS = -rho, dl/drho = -S
    dl = g * (a * before - I * x * (a * a / q))
    grads = [g * q * I, -rho * dl * S * (1 - S), g * q * x * I * (1 - I)]
    ddecay = -RATE * (dl * S).sum(0).sum(0) / (1 + torch.exp(-s["decay"].double()))
    return [v.transpose(0, 1) for v in grads] + [ddecay, R if s["state"] is not None else None]


def _exact_recur_step(case, s):
    x, r, i = (s[k].double() for k in ("x", "r", "i"))
    rho = RATE * torch.logaddexp(s["decay"].double(), torch.zeros(1, dtype=F64, device=DEV))
    l = -rho / (1 + torch.exp(-r))
    states, at = s["states"].double(), s["slots"].long()
    states[at] = l.exp() * states[at] + (-torch.expm1(2 * l)).sqrt() * x / (1 + torch.exp(-i))
    return states[at], states


def _exact_norm(case, s):
    """The backward by automatic differentiation in float64."""
    b, n, w, q = case["batch"], case["t"], case["width"], case["groups"]
    back = case["kind"] == "norm_bwd"
    x, wt, bias = (s[k].double().clone().requires_grad_(back) for k in ("x", "w", "b"))
    m = torch.ones(b, n, 1, 1, dtype=F64, device=DEV)
    if s["lens"] is not None:
        m = (torch.arange(n, device=DEV) < s["lens"][:, None]).double()[:, :, None, None]
    count = (m.sum(1, keepdim=True) * (w // q)).clamp(min=1)
    v = x.view(b, n, q, w // q) * m
    mean = v.sum(1, keepdim=True).sum(3, keepdim=True) / count
    dev = (v - mean) * m
    var = (dev * dev).sum(1, keepdim=True).sum(3, keepdim=True) / count
    rstd = 1 / (var + EPS).sqrt()
    z = (dev * rstd).view(b, n, w) * wt + bias
    f = {"none": lambda y: y, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
    y = f[case["act"]](z) * m[..., 0]
    if not back:
        some = (m.sum(1, keepdim=True) > 0).double()
        return y, torch.stack([mean.view(b, q), (rstd * some).view(b, q)], -1)
    return torch.autograd.grad(y, (x, wt, bias), s["dy"].double())


def _exact_muon(case, s):
    o = MUON
    out, moms = [], []
    for W, G, M in zip(s["param"].double(), s["grad"].double(), s["momentum"].double()):
        M = o["mu"] * M + G
        X = G + o["mu"] * M
        X = X / max(float(torch.linalg.norm(X)), o["eps"])
        # as odd polynomials of X, the smaller Gram matrix inside
        tall = case["rows"] > case["cols"]
        for _ in range(o["steps"]):
            A = X.T @ X if tall else X @ X.T
            P = 2.0315 * (A @ A) - 4.7750 * A
            P.diagonal().add_(3.4445)
            X = X @ P if tall else P @ X
        out.append(W - o["lr"] * (o["weight_decay"] * W + o["scale"] * X))
        moms.append(M)
    return torch.stack(out), torch.stack(moms)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "recur_step":
        return _exact_recur_step(case, s)
    if kind.startswith("recur"):
        return _exact_recur(case, s)
    return (_exact_norm if kind.startswith("norm") else _exact_muon)(case, s)
