"""The operators of the sequence encoder over node histories, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Linear map and gated product (row-vector convention, z = x W + b):

    linear   y = act(z) + r
    gated    [a u] = z,  h = act(a) * u

Norm and rotation of queries and keys, per head of width d:

    y = x / sqrt(mean(x^2) + eps) * w, then the plane (i, j) of rotation pair p
    turned by the angle of position pos: (y_i cos - y_j sin, y_j cos + y_i sin),
    pairs (2 p, 2 p + 1) when interleaved, else (p, p + rot / 2)

Linear attention with the decay l = exp(log_decay) of a head, token by token:

    S_t = l S_{t-1} + k_t^T v_t,   o_t = scale q_t S_t

Written from these definitions; backward by the chain rule through the same
steps.
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64


def _erf(x):
    return np.vectorize(math.erf, otypes=[F64])(x) if x.size else x


def act(name, z):
    if name == "relu":
        return np.maximum(z, 0)
    if name == "silu":
        return z / (1 + np.exp(-z))
    if name == "gelu":
        return z * 0.5 * (1 + _erf(z / math.sqrt(2)))
    return z


def act_slope(name, z):
    if name == "relu":
        return (z > 0).astype(F64)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def _z(x, W, b):
    z = np.asarray(x, F64) @ np.asarray(W, F64)
    return z if b is None else z + np.asarray(b, F64)


def linear(x, W, b=None, r=None, f="none"):
    y = act(f, _z(x, W, b))
    return y if r is None else y + np.asarray(r, F64)


def linear_bwd(x, W, b, dy, f="none"):
    """(dx, dW, db)"""
    dz = np.asarray(dy, F64) * act_slope(f, _z(x, W, b))
    return dz @ np.asarray(W, F64).T, np.asarray(x, F64).T @ dz, dz.sum(0)


def glu(x, W, b=None, f="silu"):
    z = _z(x, W, b)
    m = z.shape[1] // 2
    return act(f, z[:, :m]) * z[:, m:]


def glu_bwd(x, W, b, dh, f="silu"):
    """(dx, dW, db)"""
    z = _z(x, W, b)
    m = z.shape[1] // 2
    a, u, dh = z[:, :m], z[:, m:], np.asarray(dh, F64)
    dz = np.concatenate([dh * u * act_slope(f, a), dh * act(f, a)], 1)
    return dz @ np.asarray(W, F64).T, np.asarray(x, F64).T @ dz, dz.sum(0)


# ---- norm and rotation --------------------------------------------------------

def rope_table(n_pos, rot, base=10000.0, step=1.0):
    """[n_pos, rot]: cosines, then sines, of position * step * base^(-2 p / rot)."""
    angle = np.arange(n_pos, dtype=F64)[:, None] * (step * base ** (-np.arange(0, rot, 2, dtype=F64) / rot))
    return np.concatenate([np.cos(angle), np.sin(angle)], 1)


def _pairs(rot, interleaved):
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)


def _turn(y, table, pos, interleaved, back=False):
    """Rows of positions outside the table become NaN."""
    rot = table.shape[1]
    ok = (pos >= 0) & (pos < table.shape[0])
    t = np.asarray(table, F64)[np.where(ok, pos, 0)] if table.shape[0] else np.zeros((len(pos), rot))
    c, s = t[:, None, :rot // 2], t[:, None, rot // 2:] * (-1 if back else 1)
    i, j = _pairs(rot, interleaved)
    out = y.copy()
    out[..., i] = y[..., i] * c - y[..., j] * s
    out[..., j] = y[..., j] * c + y[..., i] * s
    out[~ok] = np.nan
    return out


def norm_rope(x, w, table, pos, eps=1e-6, interleaved=False):
    """x [n, h, d]; w [d] or None."""
    x = np.asarray(x, F64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if w is not None:
        y = y * np.asarray(w, F64)
    return _turn(y, table, pos, interleaved)


def norm_rope_bwd(x, w, table, pos, dy, eps=1e-6, interleaved=False):
    """(dx, dw)"""
    x = np.asarray(x, F64)
    g = _turn(np.asarray(dy, F64), table, pos, interleaved, back=True)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dw = (g * x * r).sum((0, 1))
    if w is not None:
        g = g * np.asarray(w, F64)
    return r * g - x * r ** 3 * (g * x).mean(-1, keepdims=True), dw


# ---- linear attention -----------------------------------------------------------

def _heads(x, heads):
    """[..., kv_heads, d] -> [..., heads, d]"""
    return np.repeat(np.asarray(x, F64), heads // x.shape[-2], axis=-2)


def linattn(q, k, v, log_decay, scale=1.0, lens=None, state=None):
    """q [b, t, h, d], k, v [b, t, hk, d] -> (o, state after the last token).
    Rows past a sequence's length are zero and change nothing."""
    b, n, h, d = q.shape
    q, k, v = np.asarray(q, F64) * scale, _heads(k, h), _heads(v, h)
    lam = np.exp(np.asarray(log_decay, F64))[:, None, None]
    S = np.zeros((b, h, d, d)) if state is None else np.asarray(state, F64).copy()
    o = np.zeros_like(q)
    for i in range(b):
        for t in range(n if lens is None else min(max(int(lens[i]), 0), n)):
            S[i] = lam * S[i] + k[i, t][:, :, None] * v[i, t][:, None, :]
            o[i, t] = np.einsum("hd,hde->he", q[i, t], S[i])
    return o, S


def linattn_bwd(q, k, v, log_decay, do, scale=1.0, lens=None, state=None, dstate=None):
    """(dq, dk, dv, gradient of the initial state)"""
    b, n, h, d = q.shape
    hk = k.shape[2]
    q, k, v, do = np.asarray(q, F64) * scale, _heads(k, h), _heads(v, h), np.asarray(do, F64)
    lam = np.exp(np.asarray(log_decay, F64))[:, None, None]
    S0 = np.zeros((b, h, d, d)) if state is None else np.asarray(state, F64)
    R = np.zeros((b, h, d, d)) if dstate is None else np.asarray(dstate, F64).copy()
    dq, dk, dv = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        S = S0[i]
        for t in range(m):
            S = lam * S + k[i, t][:, :, None] * v[i, t][:, None, :]
            dq[i, t] = scale * np.einsum("hde,he->hd", S, do[i, t])
        for t in reversed(range(m)):
            R[i] += q[i, t][:, :, None] * do[i, t][:, None, :]
            dk[i, t] = np.einsum("hde,he->hd", R[i], v[i, t])
            dv[i, t] = np.einsum("hd,hde->he", k[i, t], R[i])
            R[i] = lam * R[i]
    group = h // hk
    dk, dv = (x.reshape(b, n, hk, group, d).sum(3) for x in (dk, dv))
    return dq, dk, dv, R


def linattn_step(q, k, v, log_decay, state, slots=None, scale=1.0):
    """q [b, h, d], state [slots, h, d, d] -> (o, new states).  A row whose slot
    is outside the states gives zeros and changes nothing."""
    b, h, d = q.shape
    q, k, v = np.asarray(q, F64) * scale, _heads(k, h), _heads(v, h)
    S = np.asarray(state, F64).copy()
    lam = np.exp(np.asarray(log_decay, F64))[:, None, None]
    o = np.zeros_like(q)
    for i in range(b):
        at = i if slots is None else int(slots[i])
        if 0 <= at < S.shape[0]:
            S[at] = lam * S[at] + k[i][:, :, None] * v[i][:, None, :]
            o[i] = np.einsum("hd,hde->he", q[i], S[at])
    return o, S
