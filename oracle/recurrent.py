"""The operators of a recurrent block and of its training, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Gated linear recurrence, per channel, token by token:

    a_t = exp(-rate softplus(decay) sigmoid(r_t))
    h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t

Group norm over the tokens and the adjacent channels of a group:

    y = act(w (x - mean) / sqrt(var + eps) + b)

Update of a matrix along its orthogonalised momentum:

    M = mu M + G,  U = G + mu M (nesterov) or M,  X = U / max(|U|, eps)
    X = p X + (q A + s A A) X with A = X X^T, `steps` times
    W = (1 - lr weight_decay) W - lr scale X

Written from these definitions; backward by the chain rule through the same
steps.
"""
from __future__ import annotations

import numpy as np

from .encoder import act as _act, act_slope as _act_slope

F64 = np.float64
COEF = (3.4445, -4.7750, 2.0315)


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def softplus(z):
    return np.logaddexp(z, 0.0)


def _lens(lens, b, t):
    return np.full(b, t) if lens is None else np.clip(np.asarray(lens, np.int64), 0, t)


def _gates(r, i, decay, rate):
    l = -rate * softplus(decay) * sigmoid(r)
    return l, np.exp(l), np.sqrt(-np.expm1(2 * l)), sigmoid(i)


def recur_fwd(x, r, i, decay, rate, lens=None, state=None):
    """h [b, t, w] (zero past a length) and the states after the last tokens [b, w]."""
    x, r, i, decay = (np.asarray(v, F64) for v in (x, r, i, decay))
    b, t, w = x.shape
    n = _lens(lens, b, t)
    out, last = np.zeros((b, t, w)), np.zeros((b, w)) if state is None else np.array(state, F64)
    for s in range(b):
        h = last[s]
        for k in range(n[s]):
            _, a, q, si = _gates(r[s, k], i[s, k], decay, rate)
            h = a * h + q * si * x[s, k]
            out[s, k] = h
        last[s] = h
    return out, last


def recur_bwd(x, r, i, decay, rate, h, dh, lens=None, state=None, dstate_out=None):
    """dx, dr, di, ddecay, dstate, with h as given (the forward's, however rounded)."""
    x, r, i, decay, h, dh = (np.asarray(v, F64) for v in (x, r, i, decay, h, dh))
    b, t, w = x.shape
    n = _lens(lens, b, t)
    dx, dr, di = (np.zeros((b, t, w)) for _ in range(3))
    ddecay = np.zeros(w)
    dstate = np.zeros((b, w)) if dstate_out is None else np.array(dstate_out, F64)
    for s in range(b):
        c = dstate[s]
        for k in range(n[s] - 1, -1, -1):
            l, a, q, si = _gates(r[s, k], i[s, k], decay, rate)
            sr = sigmoid(r[s, k])
            before = h[s, k - 1] if k else (np.zeros(w) if state is None else np.asarray(state, F64)[s])
            g = dh[s, k] + c
            dx[s, k] = g * q * si
            di[s, k] = g * q * x[s, k] * si * sigmoid(-i[s, k])
            # dq/dl = -a^2 / q; times l or sr it goes to 0 where l does
            with np.errstate(divide="ignore", invalid="ignore"):
                slope = np.where(q > 0, a * a / q, 0.0)
            dlog = g * (a * before - si * x[s, k] * slope)
            dr[s, k] = dlog * l * sigmoid(-r[s, k])
            ddecay += -rate * sigmoid(decay) * dlog * sr
            c = a * g
        dstate[s] = c
    return dx, dr, di, ddecay, dstate


def recur_step(x, r, i, decay, rate, states, slots=None):
    """h [b, w] and the states after one token each; a slot outside is idle."""
    x, r, i, decay = (np.asarray(v, F64) for v in (x, r, i, decay))
    states = np.array(states, F64)
    h = np.zeros(x.shape)
    for k in range(x.shape[0]):
        at = k if slots is None else int(slots[k])
        if 0 <= at < len(states):
            _, a, q, si = _gates(r[k], i[k], decay, rate)
            states[at] = h[k] = a * states[at] + q * si * x[k]
    return h, states


def _groups(x, groups):
    b, t, w = x.shape
    return x.reshape(b, t, groups, w // groups)


def group_norm_fwd(x, groups, w=None, b=None, act="none", eps=1e-5, lens=None):
    """y [b, t, width] (zero past a length) and stats [b, groups, 2]."""
    x = np.asarray(x, F64)
    n = _lens(lens, x.shape[0], x.shape[1])
    y, stats = np.zeros(x.shape), np.zeros((x.shape[0], groups, 2))
    w = np.ones(x.shape[2]) if w is None else np.asarray(w, F64)
    b = np.zeros(x.shape[2]) if b is None else np.asarray(b, F64)
    for s in range(x.shape[0]):
        v = _groups(x[s:s + 1, :n[s]], groups)
        if not n[s]:
            continue
        mean = v.mean((0, 1, 3))
        rstd = 1 / np.sqrt(((v - mean[:, None]) ** 2).mean((0, 1, 3)) + eps)
        u = ((v - mean[:, None]) * rstd[:, None]).reshape(n[s], -1)
        y[s, :n[s]] = _act(act, u * w + b)
        stats[s] = np.stack([mean, rstd], -1)
    return y, stats


def group_norm_bwd(x, groups, w, b, stats, dy, act="none", lens=None):
    """dx, dw, db with the statistics as given."""
    x, dy, stats = (np.asarray(v, F64) for v in (x, dy, stats))
    width = x.shape[2]
    n = _lens(lens, x.shape[0], x.shape[1])
    w = np.ones(width) if w is None else np.asarray(w, F64)
    b = np.zeros(width) if b is None else np.asarray(b, F64)
    dx, dw, db = np.zeros(x.shape), np.zeros(width), np.zeros(width)
    for s in range(x.shape[0]):
        if not n[s]:
            continue
        mean, rstd = stats[s, :, 0], stats[s, :, 1]
        u = ((_groups(x[s:s + 1, :n[s]], groups) - mean[:, None]) * rstd[:, None])[0]
        flat = u.reshape(n[s], width)
        dz = dy[s, :n[s]] * _act_slope(act, flat * w + b)
        dw += (dz * flat).sum(0)
        db += dz.sum(0)
        e = (dz * w).reshape(u.shape)
        m0, m1 = e.mean((0, 2)), (e * u).mean((0, 2))
        dx[s, :n[s]] = (rstd[:, None] * (e - m0[:, None] - u * m1[:, None])).reshape(n[s], width)
    return dx, dw, db


def orthogonal(U, steps=5, eps=1e-7):
    """X after `steps` of the iteration from U / max(|U|, eps)."""
    p, q, s = COEF
    X = np.asarray(U, F64)
    X = X / max(np.sqrt((X * X).sum()), eps)
    for _ in range(steps):
        if X.shape[0] <= X.shape[1]:
            A = X @ X.T
            X = p * X + (q * A + s * A @ A) @ X
        else:
            A = X.T @ X
            X = p * X + X @ (q * A + s * A @ A)
    return X


def muon_step(W, G, M, lr, mu=0.95, weight_decay=0.0, nesterov=True, steps=5, scale=1.0, eps=1e-7):
    """The updated matrix and momentum."""
    W, G, M = (np.asarray(v, F64) for v in (W, G, M))
    M = mu * M + G
    X = orthogonal(G + mu * M if nesterov else M, steps, eps)
    return (1 - lr * weight_decay) * W - lr * scale * X, M
