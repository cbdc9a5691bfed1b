"""The operators of a sequence encoder over node histories, as timed cases: the
norm and position rotation of queries and keys, linear attention with a decay
for each head (whole histories and single tokens), the matrix product with
bias, activation and residual, and the gated feed-forward product, forward and
backward.

``listed()`` names fixed cases, ``draw(rng)`` more of the same ranges;
``prepare`` makes the inputs that a program has in hand (all from the seed),
``run`` is one pass: with ``own`` through the public entry points of
``paper_2608_02168_amd.api``, without it in elementary torch operations in 32
bits, rounded once at the end.  ``work`` gives the bytes and operations that a
pass cannot do without, ``exact`` the outputs in float64 from the definitions.

Matrices are in the row-vector convention y = x W.  Heads h of the queries
share key and value head h // (heads / kv_heads).  Log-decays are natural
logarithms, one per query head.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
CHUNK = 64
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # serving: one new token for each of 16 sequences, queries and keys inside a packed projection
        dict(name="qk_tokens", kind="qk_fwd", dtype="bf16", n=16, heads=16, kv_heads=4, d=128, rot=128, inter=False,
             n_pos=8192),
        # prompts of a large batch: 32 query heads on 8 key heads
        dict(name="qk_prompt", kind="qk_fwd", dtype="bf16", n=32768, heads=32, kv_heads=8, d=128, rot=128, inter=False,
             n_pos=8192),
        # training in float32, rotation of adjacent pairs over half of each head, an odd number of tokens
        dict(name="qk_train", kind="qk_bwd", dtype="f32", n=20011, heads=12, kv_heads=12, d=64, rot=32, inter=True,
             n_pos=4096),
        # one long history: few heads, so the work has to be split over its length
        dict(name="attn_long", kind="attn_fwd", dtype="bf16", batch=1, t=16381, heads=16, kv_heads=16, d=128,
             ragged=False, state=True),
        # many short histories at the default width and heads of the attention layers, lengths that differ
        dict(name="attn_histories", kind="attn_fwd", dtype="f32", batch=8192, t=24, heads=4, kv_heads=4, d=16,
             ragged=True, state=False),
        # a training batch, two query heads on each key head
        dict(name="attn_train", kind="attn_bwd", dtype="bf16", batch=8, t=2048, heads=16, kv_heads=8, d=64,
             ragged=True, state=True),
        # serving: one token for 200 of 256 held states
        dict(name="attn_token", kind="attn_step", dtype="bf16", batch=200, slots=256, heads=16, kv_heads=4, d=128),
        # serving one sequence: a projection of a single row with its bias and residual
        dict(name="linear_token", kind="linear_fwd", dtype="bf16", n=1, d_in=4096, d_out=4096, act="none", bias=True,
             res=True),
        # the node update of the layers, sigma(x W + b) + x, in training: very many rows of the layers' width
        dict(name="linear_nodes", kind="linear_bwd", dtype="f32", n=200003, d_in=128, d_out=128, act="silu", bias=True,
             res=False),
        # a small float32 model, widths that fill no tile, some thousand rows
        dict(name="glu_odd", kind="glu_fwd", dtype="f32", n=1777, d=200, f=517, act="gelu", bias=True),
        # a prompt of one sequence
        dict(name="glu_prompt", kind="glu_fwd", dtype="bf16", n=2000, d=1024, f=2816, act="silu", bias=False),
        # training of a wide model
        dict(name="glu_train", kind="glu_bwd", dtype="bf16", n=8192, d=2048, f=8192, act="silu", bias=False),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 8, one time in four any number."""
    w = _between(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    kind = rng.choice(["qk_fwd", "qk_bwd", "attn_fwd", "attn_bwd", "attn_step", "linear_fwd", "linear_bwd", "glu_fwd",
                       "glu_bwd"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind.startswith("qk"):
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4])
        d = rng.choice([16, 32, 64, 80, 96, 128, 256])
        rot = rng.choice([d, d, d // 2 // 2 * 2])
        n = _between(rng, 1, min(40000, (1 << 27) // ((heads + kv) * d)))
        return dict(c, n=n, heads=heads, kv_heads=kv, d=d, rot=rot, inter=rng.random() < 0.5, n_pos=4096)
    if kind in ("attn_fwd", "attn_bwd"):
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        d = rng.choice([16, 32, 64, 64, 80, 128, 128])
        t = _between(rng, 1, 8192)
        # tokens times heads, and for the states of short histories sequences times heads
        batch = _between(rng, 1, max(1, min(4096, (1 << 18) // (heads * t), (1 << 28) // (heads * d * d))))
        return dict(c, batch=batch, t=t, heads=heads, kv_heads=kv, d=d, ragged=rng.random() < 0.5,
                    state=rng.random() < 0.5)
    if kind == "attn_step":
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        d = rng.choice([16, 32, 64, 80, 128])
        batch = _between(rng, 1, max(1, min(4096, (1 << 26) // (heads * d * d))))
        return dict(c, batch=batch, slots=batch + rng.randrange(0, 1 + batch // 4), heads=heads, kv_heads=kv, d=d)
    # no ReLU in a backward case: its slope jumps where 32 and 64 bits may fall on either side of zero
    act = rng.choice(["silu", "gelu"] + ["relu"] * kind.endswith("fwd"))
    if kind.startswith("linear"):
        d_in, d_out = _width(rng, 16, 2560), _width(rng, 16, 2560)
        n = _between(rng, 1, max(1, min(65536, (1 << 34) // (d_in * d_out))))
        return dict(c, n=n, d_in=d_in, d_out=d_out, act=rng.choice(["none", act]), bias=rng.random() < 0.5,
                    res=kind == "linear_fwd" and rng.random() < 0.5)
    d, f = _width(rng, 16, 2048), _width(rng, 16, 2816)
    n = _between(rng, 1, max(1, min(32768, (1 << 34) // (d * f))))
    return dict(c, n=n, d=d, f=f, act=act, bias=rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------

def _type(case):
    return BF16 if case["dtype"] == "bf16" else F32


def _log_decay(heads):
    """1 - 2^-(3 .. 9): from heads that forget within tens of tokens to heads
    that hold hundreds."""
    x = torch.linspace(3.0, 9.0, heads, dtype=F64) if heads > 1 else torch.tensor([5.0], dtype=F64)
    return torch.log1p(-(2.0 ** -x)).to(F32).to(DEV)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = _type(case)

    def normal(*shape, scale=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device=DEV, dtype=F32) * scale).to(dtype or t)

    kind, s = case["kind"], {}
    if kind.startswith("qk"):
        n, hq, hk, d, rot = case["n"], case["heads"], case["kv_heads"], case["d"], case["rot"]
        packed = normal(n, hq + 2 * hk, d, scale=1.5)  # a projection's output: queries, keys, values
        s["q"], s["k"] = packed[:, :hq], packed[:, hq:hq + hk]
        s["wq"], s["wk"] = (1.0 + normal(d, scale=0.1, dtype=F32) for _ in range(2))
        s["pos"] = torch.randint(0, case["n_pos"], (n,), generator=g, device=DEV, dtype=torch.int32)
        freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device=DEV) / rot)
        angle = torch.arange(case["n_pos"], dtype=F64, device=DEV)[:, None] * freq
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).to(F32)
        if kind == "qk_bwd":
            s["dq_out"], s["dk_out"] = normal(n, hq, d), normal(n, hk, d)
        return s
    if kind.startswith("attn"):
        b, hq, hk, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
        s["log_decay"], s["scale"] = _log_decay(hq), d ** -0.5
        if kind == "attn_step":
            packed = normal(b, hq + 2 * hk, d)
            s["q"], s["k"], s["v"] = packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:]
            s["state"] = normal(case["slots"], hq, d, d, scale=3.0, dtype=F32)
            s["slots"] = torch.randperm(case["slots"], generator=g, device=DEV)[:b].to(torch.int32)
            return s
        n = case["t"]
        s["q"] = normal(b, n, hq, d)
        packed = normal(b, n, 2 * hk, d)
        s["k"], s["v"] = packed[:, :, :hk], packed[:, :, hk:]
        # lengths from a whole history down to none at all
        s["lens"] = None
        if case["ragged"]:
            s["lens"] = torch.randint(0, n + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
            s["lens"][0] = n
        s["state"] = normal(b, hq, d, d, scale=3.0, dtype=F32) if case["state"] else None
        if kind == "attn_bwd":
            s["do"] = normal(b, n, hq, d)
            s["dstate"] = normal(b, hq, d, d, dtype=F32) if case["state"] else None
        return s
    if kind.startswith("linear"):
        n, a, b = case["n"], case["d_in"], case["d_out"]
    else:
        n, a, b = case["n"], case["d"], 2 * case["f"]
    s["x"], s["w"] = normal(n, a), normal(a, b, scale=a ** -0.5)
    s["bias"] = normal(b, scale=0.5, dtype=F32) if case["bias"] else None
    if kind == "linear_fwd" and case["res"]:
        s["res"] = normal(n, b)
    if kind == "linear_bwd":
        s["dy"] = normal(n, b)
    if kind == "glu_bwd":
        s["dh"] = normal(n, b // 2)
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
    if kind == "qk_fwd":
        return api.hg_qk_norm_rope_fwd(s["q"], s["k"], s["wq"], s["wk"], s["table"], s["pos"], interleaved=c["inter"])
    if kind == "qk_bwd":
        return api.hg_qk_norm_rope_bwd(s["q"], s["k"], s["wq"], s["wk"], s["table"], s["pos"], s["dq_out"],
                                       s["dk_out"], interleaved=c["inter"])
    if kind == "attn_fwd":
        return api.hg_linattn_fwd(s["q"], s["k"], s["v"], s["log_decay"], scale=s["scale"], lens=s["lens"],
                                  state=s["state"], want_state=True)
    if kind == "attn_bwd":
        return api.hg_linattn_bwd(s["q"], s["k"], s["v"], s["log_decay"], s["do"], scale=s["scale"], lens=s["lens"],
                                  state=s["state"], dstate_out=s["dstate"])
    if kind == "attn_step":
        o = api.hg_linattn_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"],
                                scale=s["scale"])
        return o, s["state"]
    act = ACTS[c["act"]]
    if kind == "linear_fwd":
        return api.hg_linear_fwd(s["x"], s["w"], bias=s["bias"], residual=s.get("res"), act=act)
    if kind == "linear_bwd":
        return api.hg_linear_bwd(s["x"], s["w"], s["bias"], s["dy"], act=act)
    if kind == "glu_fwd":
        return api.hg_glu_fwd(s["x"], s["w"], bias=s["bias"], act=act)
    return api.hg_glu_bwd(s["x"], s["w"], s["bias"], s["dh"], act=act)


# ---- the plain form -----------------------------------------------------------

def _turn(x, cos, sin, inter):
    """Rotation of the first 2 * cos.shape[-1] columns by the given angles."""
    m = cos.shape[-1]
    r, rest = x[..., :2 * m], x[..., 2 * m:]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :m], r[..., m:])
    u, v = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([u, v], -1).flatten(-2) if inter else torch.cat([u, v], -1)
    return torch.cat([r, rest], -1)


def _angles(s):
    m = s["table"].shape[1] // 2
    t = s["table"][s["pos"].long()][:, None]
    return t[..., :m], t[..., m:]


def _plain_qk(s, x, w):
    cos, sin = _angles(s)
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
    return _turn(y, cos, sin, s["case"]["inter"])


def _plain_qk_bwd(s, x, w, dy):
    cos, sin = _angles(s)
    x, dy = x.float(), _turn(dy.float(), cos, -sin, s["case"]["inter"])
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    xh = x * r
    dw = (dy * xh).sum((0, 1))
    dh = dy * w
    return r * (dh - xh * (dh * xh).mean(-1, keepdim=True)), dw


def _chunks(x, c):
    """[b, t, h, d] -> [b, h, n, c, d], the last chunk filled with zeros."""
    b, t, h, d = x.shape
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -t % c))
    return x.view(b, -1, c, h, d).permute(0, 3, 1, 2, 4)


def _whole(x, t):
    """The inverse of _chunks."""
    return x.permute(0, 2, 3, 1, 4).flatten(1, 2)[:, :t]


def _decays(g, steps):
    """exp(g steps) for each head where steps >= 0, and 0 elsewhere: [h, *steps.shape]."""
    g = g.view(-1, *[1] * steps.dim())
    return torch.where(steps >= 0, torch.exp(g * steps.clamp(min=0)), torch.zeros((), device=DEV))


def _plain_scan(q, k, v, g, back):
    """sum over s <= t (back: s >= t) of exp(g |t - s|) (q_t . k_s) v_s, in
    chunks: inside a chunk by the products of its tokens, across chunks by
    the chunks' sums of k^T v."""
    t = q.shape[1]
    c = min(CHUNK, t)
    q, k, v = _chunks(q, c), _chunks(k, c), _chunks(v, c)
    i = torch.arange(c, device=DEV)
    n = torch.arange(q.shape[2], device=DEV)
    sign = -1 if back else 1
    inside = _decays(g, sign * (i[:, None] - i[None, :]))[:, None]
    o = ((q @ k.transpose(-1, -2)) * inside) @ v
    far = _decays(g, i if back else c - 1 - i)[:, None, :, None]   # to the chunk's edge
    near = _decays(g, c - i if back else i + 1)[:, None, :, None]  # from the edge before
    sums = (k * far).transpose(-1, -2) @ v
    across = _decays(g, c * (sign * (n[:, None] - n[None, :]) - 1))
    before = (across @ sums.flatten(-2)).view_as(sums)
    return _whole(o + (q * near) @ before, t)


def _plain_attn_parts(s):
    """Float32 copies, keys and values once per query head, zero past each length; the lengths."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    q, k, v = s["q"].float() * s["scale"], s["k"].float(), s["v"].float()
    k, v = (x.repeat_interleave(group, 2) for x in (k, v))
    t = torch.arange(c["t"], device=DEV)
    lens = s["lens"].long() if s["lens"] is not None else torch.full((c["batch"],), c["t"], device=DEV)
    live = (t < lens[:, None])[:, :, None, None]
    left = lens[:, None] - 1 - t                                        # tokens after t, [b, t]
    left = _decays(s["log_decay"], left).permute(1, 2, 0)[..., None]    # [b, t, h, 1], 0 past the end
    done = _decays(s["log_decay"], t + 1).t()[None, :, :, None]
    whole = _decays(s["log_decay"], lens).t()[:, :, None, None]
    return q * live, k * live, v * live, live, left, done, whole


def _by_head(x):
    return x.transpose(1, 2)


def _plain_attn_fwd(s):
    q, k, v, live, left, done, whole = _plain_attn_parts(s)
    o = _plain_scan(q, k, v, s["log_decay"], False)
    end = _by_head(k * left).transpose(-1, -2) @ _by_head(v)
    if s["state"] is not None:
        o = o + _by_head(_by_head(q * done) @ s["state"])
        end = end + whole * s["state"]
    return (o * live).to(s["q"].dtype), end


def _plain_attn_bwd(s):
    c = s["case"]
    q, k, v, live, left, done, whole = _plain_attn_parts(s)
    do = s["do"].float() * live
    g = s["log_decay"]
    dq = _plain_scan(do, v, k, g, False)
    dk = _plain_scan(v, do, q, g, True)
    dv = _plain_scan(k, q, do, g, True)
    dstate = None
    if s["state"] is not None:
        dq = dq + _by_head(_by_head(do * done) @ s["state"].transpose(-1, -2))
        dk = dk + _by_head(_by_head(v * left) @ s["dstate"].transpose(-1, -2))
        dv = dv + _by_head(_by_head(k * left) @ s["dstate"])
        dstate = _by_head(q * done).transpose(-1, -2) @ _by_head(do) + whole * s["dstate"]
    dq = dq * s["scale"]
    dk, dv = (x.view(c["batch"], c["t"], c["kv_heads"], -1, c["d"]).sum(3) for x in (dk, dv))
    return [None if x is None else (x * live).to(s["q"].dtype) for x in (dq, dk, dv)] + [dstate]


def _plain_attn_step(s):
    group = s["case"]["heads"] // s["case"]["kv_heads"]
    q, k, v = s["q"].float() * s["scale"], s["k"].float(), s["v"].float()
    k, v = (x.repeat_interleave(group, 1) for x in (k, v))
    at = s["slots"].long()
    new = s["state"][at] * torch.exp(s["log_decay"])[:, None, None] + k[..., None] * v[..., None, :]
    s["state"][at] = new
    return (q[..., None, :] @ new)[..., 0, :].to(s["q"].dtype), s["state"]


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _plain_products(s):
    """The linear map and the gated product, forward or backward."""
    c, t = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w
    if s["bias"] is not None:
        z = z + s["bias"]
    if c["kind"] == "linear_fwd":
        y = _act(z, c["act"])
        return (y + s["res"].float() if "res" in s else y).to(t)
    if c["kind"] == "glu_fwd":
        a, b = z.chunk(2, -1)
        return (_act(a, c["act"]) * b).to(t)
    if c["kind"] == "linear_bwd":
        dz = s["dy"].float() * _act_grad(z, c["act"])
    else:
        a, b = z.chunk(2, -1)
        dh = s["dh"].float()
        dz = torch.cat([dh * b * _act_grad(a, c["act"]), dh * _act(a, c["act"])], -1)
    dbias = dz.sum(0) if s["bias"] is not None else None
    return (dz @ w.t()).to(t), (x.t() @ dz).to(t), dbias


def _run_plain(s):
    kind, t = s["case"]["kind"], s["case"]["dtype"]
    if kind == "qk_fwd":
        return tuple(_plain_qk(s, s[x], s["w" + x]).to(s["q"].dtype) for x in "qk")
    if kind == "qk_bwd":
        (dq, dwq), (dk, dwk) = (_plain_qk_bwd(s, s[x], s["w" + x], s["d" + x + "_out"]) for x in "qk")
        return dq.to(s["q"].dtype), dk.to(s["q"].dtype), dwq, dwk
    if kind == "attn_fwd":
        return _plain_attn_fwd(s)
    if kind == "attn_bwd":
        return _plain_attn_bwd(s)
    if kind == "attn_step":
        return _plain_attn_step(s)
    return _plain_products(s)


# ---- what a pass cannot do without ---------------------------------------------

def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind.startswith("qk"):
        rows = case["n"] * (case["heads"] + case["kv_heads"])
        moves = 2 if kind == "qk_fwd" else 3
        return {"bytes": moves * rows * case["d"] * e + case["n"] * (4 + 4 * case["rot"]),
                "flops": rows * case["d"] * (8 if kind == "qk_fwd" else 16)}
    if kind.startswith("attn"):
        hq, hk, d = case["heads"], case["kv_heads"], case["d"]
        state = 4 * hq * d * d
        if kind == "attn_step":
            return {"bytes": case["batch"] * (2 * state + 2 * (hq + hk) * d * e), "flops": case["batch"] * hq * 5 * d * d}
        tokens, t = case["batch"] * case["t"], case["t"]
        # token by token through the state, or pair by pair: the cheaper
        per = min(4 * d * d, 2 * (t + 1) * d)
        held = case["batch"] * state
        if kind == "attn_fwd":
            return {"bytes": tokens * 2 * (hq + hk) * d * e + held * (2 if case["state"] else 1),
                    "flops": tokens * hq * per}
        return {"bytes": tokens * (3 * hq + 4 * hk) * d * e + held * (3 if case["state"] else 0),
                "flops": tokens * hq * 5 * per // 2}
    if kind.startswith("linear"):
        n, a, b = case["n"], case["d_in"], case["d_out"]
        if kind == "linear_fwd":
            return {"bytes": (n * a + a * b + n * b * (2 if case["res"] else 1)) * e + 4 * b * case["bias"],
                    "flops": 2 * n * a * b}
        products = 2 if case["act"] == "none" else 3
        return {"bytes": (2 * n * a + 2 * a * b + n * b) * e + 8 * b * case["bias"], "flops": products * 2 * n * a * b}
    n, a, b = case["n"], case["d"], 2 * case["f"]
    if kind == "glu_fwd":
        return {"bytes": (n * a + a * b + n * b // 2) * e + 4 * b * case["bias"], "flops": 2 * n * a * b}
    return {"bytes": (2 * n * a + 2 * a * b + n * b // 2) * e + 8 * b * case["bias"], "flops": 6 * n * a * b}


# ---- the definitions in float64 -------------------------------------------------

def _exact_qk(case, s):
    m = case["rot"] // 2
    cols = [(2 * i, 2 * i + 1) if case["inter"] else (i, m + i) for i in range(m)]
    lo, hi = (torch.tensor([c[j] for c in cols], dtype=torch.long, device=DEV) for j in (0, 1))
    t = s["table"].double()[s["pos"].long()]
    z = torch.complex(t[:, :m], t[:, m:])[:, None]  # the rotation as a product of complex numbers
    out, dw = [], []
    for x, w, dy in ((s["q"], s["wq"], s.get("dq_out")), (s["k"], s["wk"], s.get("dk_out"))):
        x, w = x.double(), w.double()
        rms = ((x * x).sum(-1, keepdim=True) / case["d"] + 1e-6).sqrt()
        y = x / rms * w if dy is None else dy.double().clone()
        p = torch.complex(y[..., lo], y[..., hi]) * (z if dy is None else z.conj())
        y[..., lo], y[..., hi] = p.real, p.imag
        if dy is None:
            out.append(y)
            continue
        dw.append((y * x / rms).sum(0).sum(0))
        h = y * w
        out.append(h / rms - x * (h * x).sum(-1, keepdim=True) / (case["d"] * rms ** 3))
    return tuple(out + dw)


def _exact_attn(case, s):
    """Token by token: S = exp(g) S + k^T v, o = q S; backward through the same steps."""
    b, hq, d, group = case["batch"], case["heads"], case["d"], case["heads"] // case["kv_heads"]
    # [t, b, h, ...]: a step reads one slice
    q, k, v = (s[x].double().transpose(0, 1) for x in ("q", "k", "v"))
    k, v = (x[:, :, torch.arange(hq, device=DEV) // group] for x in (k, v))
    q = q * s["scale"]
    lam = s["log_decay"].double().exp()[None, :, None, None]
    n = case["t"]
    lens = s["lens"] if s["lens"] is not None else torch.full((b,), n, device=DEV, dtype=torch.int32)
    live = (torch.arange(n, device=DEV)[:, None] < lens).view(n, b, 1, 1)
    first = s["state"].double() if s["state"] is not None else torch.zeros(b, hq, d, d, dtype=F64, device=DEV)
    back = case["kind"] == "attn_bwd"
    do = s["do"].double().transpose(0, 1) * live if back else None
    S, out = first, []
    for t in range(n):
        S = torch.where(live[t][..., None], lam * S + k[t][..., None] * v[t][..., None, :], S)
        out.append((S @ do[t][..., None])[..., 0] if back else (q[t][..., None, :] @ S)[..., 0, :])
    out = torch.stack(out) * live
    if not back:
        return out.transpose(0, 1), S
    dq = out * s["scale"]
    R = s["dstate"].double() if s["dstate"] is not None else torch.zeros_like(first)
    dk, dv = [], []
    for t in reversed(range(n)):
        # R: the gradient of the state after token t
        R = torch.where(live[t][..., None], R + q[t][..., None] * do[t][..., None, :], R)
        dk.append((R @ v[t][..., None])[..., 0])
        dv.append((k[t][..., None, :] @ R)[..., 0, :])
        R = torch.where(live[t][..., None], lam * R, R)
    dk, dv = (torch.stack(x[::-1]) * live for x in (dk, dv))
    dk, dv = (x.unflatten(2, (-1, group)).sum(3) for x in (dk, dv))
    grads = [x.transpose(0, 1) for x in (dq, dk, dv)]
    return grads + [R if s["state"] is not None else None]


def _exact_step(case, s):
    group = case["heads"] // case["kv_heads"]
    at = s["slots"].long()
    of = torch.arange(case["heads"], device=DEV) // group
    q, k, v = s["q"].double(), s["k"].double()[:, of], s["v"].double()[:, of]
    S = s["state"].double()
    S[at] = S[at] * s["log_decay"].double().exp().view(1, -1, 1, 1) + k.unsqueeze(3) * v.unsqueeze(2)
    return s["scale"] * (q.unsqueeze(2) @ S[at]).squeeze(2), S


def _exact_products(case, s):
    """The activations' slopes by autograd on float64."""
    x, w = s["x"].double(), s["w"].double()
    z = x @ w
    if s["bias"] is not None:
        z += s["bias"].double()
    kind = case["kind"]
    back = kind.endswith("bwd")
    z.requires_grad_(back)
    f = {"none": lambda y: y, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
    if kind.startswith("linear"):
        y = f[case["act"]](z)
    else:
        m = z.shape[1] // 2
        y = f[case["act"]](z[:, :m]) * z[:, m:]
    if not back:
        return y + s["res"].double() if "res" in s else y
    up = s["dy"] if kind == "linear_bwd" else s["dh"]
    (dz,) = torch.autograd.grad(y, z, up.double())
    return dz @ w.T, x.T @ dz, dz.sum(0) if s["bias"] is not None else None


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("qk"):
        return _exact_qk(case, s)
    if kind == "attn_step":
        return _exact_step(case, s)
    if kind.startswith("attn"):
        return _exact_attn(case, s)
    return _exact_products(case, s)
