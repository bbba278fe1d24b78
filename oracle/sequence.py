"""Float64 definitions of the sequence operators and of their gradients: cross attention over
segments, the causal convolution and the selective scan over packed ragged sequences.

Plain loops over segments, heads and steps; gradients by the chain rule, written out.  Inputs are
NumPy arrays of the values that the library is given (bfloat16 tensors as the numbers they hold).
"""
from __future__ import annotations

import numpy as np


# ---- cross attention ---------------------------------------------------------------
def _segments(q, k, q_off, k_off, mask):
    group = q.shape[1] // k.shape[1]
    for s in range(len(q_off) - 1):
        keys = np.arange(k_off[s], k_off[s + 1])
        if mask is not None:
            keys = keys[np.asarray(mask)[keys] != 0]
        for h in range(q.shape[1]):
            yield slice(q_off[s], q_off[s + 1]), keys, h, h // group


def attention(q, k, v, q_off, k_off, scale, mask=None):
    """o [rows][heads][d] and lse [rows][heads]."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    o = np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    for rows, keys, h, hk in _segments(q, k, q_off, k_off, mask):
        if len(keys) == 0 or rows.stop == rows.start:
            continue
        s = scale * (q[rows, h] @ k[keys, hk].T)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        o[rows, h] = (p / total) @ v[keys, hk]
        lse[rows, h] = (top + np.log(total))[:, 0]
    return o, lse


def attention_grad(do, q, k, v, q_off, k_off, scale, mask=None):
    """dq, dk, dv."""
    do, q, k, v = (np.asarray(t, np.float64) for t in (do, q, k, v))
    o, lse = attention(q, k, v, q_off, k_off, scale, mask)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for rows, keys, h, hk in _segments(q, k, q_off, k_off, mask):
        if len(keys) == 0 or rows.stop == rows.start:
            continue
        p = np.exp(scale * (q[rows, h] @ k[keys, hk].T) - lse[rows, h, None])
        dp = do[rows, h] @ v[keys, hk].T
        ds = p * (dp - (do[rows, h] * o[rows, h]).sum(1, keepdims=True)) * scale
        dq[rows, h] = ds @ k[keys, hk]
        dk[keys, hk] += ds.T @ q[rows, h]
        dv[keys, hk] += p.T @ do[rows, h]
    return dq, dk, dv


# ---- convolution -------------------------------------------------------------------
def sigmoid(x):
    return 0.5 * (1.0 + np.tanh(0.5 * x))


def _window(x, off, s, W, state):
    """The inputs of sequence s with the W - 1 before them."""
    before = np.zeros((W - 1, x.shape[1])) if state is None else np.asarray(state[s], np.float64)
    return np.concatenate([before, x[off[s]:off[s + 1]]])


def conv(x, off, w, b=None, silu=True, state=None):
    """y and the carried-out state."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    W = w.shape[1]
    y = np.zeros(x.shape)
    out = np.zeros((len(off) - 1, W - 1, x.shape[1]))
    for s in range(len(off) - 1):
        xs = _window(x, off, s, W, state)
        for t in range(off[s + 1] - off[s]):
            a = (w.T * xs[t:t + W]).sum(0) + (0.0 if b is None else b)
            y[off[s] + t] = a * sigmoid(a) if silu else a
        out[s] = xs[len(xs) - (W - 1):]
    return y, out


def conv_grad(dy, x, off, w, b=None, silu=True, state=None, d_state_out=None):
    """dx, dw, db, dstate."""
    x, w, dy = (np.asarray(t, np.float64) for t in (x, w, dy))
    W = w.shape[1]
    dx, dw, db = np.zeros(x.shape), np.zeros(w.shape), np.zeros(w.shape[0])
    dstate = np.zeros((len(off) - 1, W - 1, x.shape[1]))
    for s in range(len(off) - 1):
        xs = _window(x, off, s, W, state)
        dxs = np.zeros(xs.shape)
        if d_state_out is not None:
            dxs[len(xs) - (W - 1):] += d_state_out[s]
        for t in range(off[s + 1] - off[s]):
            a = (w.T * xs[t:t + W]).sum(0) + (0.0 if b is None else b)
            g = sigmoid(a)
            da = dy[off[s] + t] * (g * (1.0 + a * (1.0 - g)) if silu else 1.0)
            dxs[t:t + W] += w.T * da
            dw += (xs[t:t + W] * da).T
            db += da
        dstate[s] = dxs[:W - 1]
        dx[off[s]:off[s + 1]] = dxs[W - 1:]
    return dx, dw, db, dstate


# ---- scan --------------------------------------------------------------------------
def softplus(x):
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def _states(u, dt, A, Bm, off, s, h0):
    h = np.zeros(A.shape) if h0 is None else np.asarray(h0[s], np.float64)
    hs = [h]
    for t in range(off[s], off[s + 1]):
        h = np.exp(dt[t][:, None] * A) * h + (dt[t] * u[t])[:, None] * Bm[t][None, :]
        hs.append(h)
    return hs


def scan(u, delta, A, Bm, Cm, off, D=None, z=None, delta_bias=None, h0=None):
    """y and the last states."""
    u, delta, A, Bm, Cm = (np.asarray(t, np.float64) for t in (u, delta, A, Bm, Cm))
    dt = softplus(delta + (0.0 if delta_bias is None else delta_bias))
    y = np.zeros(u.shape)
    hT = np.zeros((len(off) - 1,) + A.shape)
    for s in range(len(off) - 1):
        hs = _states(u, dt, A, Bm, off, s, h0)
        hT[s] = hs[-1]
        for i, t in enumerate(range(off[s], off[s + 1])):
            y[t] = hs[i + 1] @ Cm[t] + (0.0 if D is None else D * u[t])
            if z is not None:
                y[t] *= z[t] * sigmoid(z[t])
    return y, hT


def scan_grad(dy, u, delta, A, Bm, Cm, off, D=None, z=None, delta_bias=None, h0=None, dhT=None):
    """Dict of du, ddelta, dA, dB, dC, dD, ddelta_bias, dz, dh0."""
    dy, u, delta, A, Bm, Cm = (np.asarray(t, np.float64) for t in (dy, u, delta, A, Bm, Cm))
    raw = delta + (0.0 if delta_bias is None else delta_bias)
    dt = softplus(raw)
    r = {"du": np.zeros(u.shape), "ddelta": np.zeros(u.shape), "dA": np.zeros(A.shape), "dB": np.zeros(Bm.shape),
         "dC": np.zeros(Cm.shape), "dD": np.zeros(u.shape[1]), "dz": np.zeros(u.shape),
         "dh0": np.zeros((len(off) - 1,) + A.shape)}
    for s in range(len(off) - 1):
        hs = _states(u, dt, A, Bm, off, s, h0)
        g = np.zeros(A.shape) if dhT is None else np.asarray(dhT[s], np.float64).copy()
        for i in range(off[s + 1] - off[s] - 1, -1, -1):
            t = off[s] + i
            d_out = dy[t]
            if z is not None:
                sg = sigmoid(z[t])
                y = hs[i + 1] @ Cm[t] + (0.0 if D is None else D * u[t])
                r["dz"][t] = d_out * y * sg * (1.0 + z[t] * (1.0 - sg))
                d_out = d_out * z[t] * sg
            g = g + d_out[:, None] * Cm[t][None, :]
            r["dC"][t] = d_out @ hs[i + 1]
            a = np.exp(dt[t][:, None] * A)
            r["dB"][t] = (dt[t] * u[t]) @ g
            s1 = g @ Bm[t]
            w = g * a * hs[i]
            r["du"][t] = dt[t] * s1 + (0.0 if D is None else D * d_out)
            r["dD"] += d_out * u[t]
            r["ddelta"][t] = (u[t] * s1 + (w * A).sum(1)) * sigmoid(raw[t])
            r["dA"] += w * dt[t][:, None]
            g = g * a
        r["dh0"][s] = g
    r["ddelta_bias"] = r["ddelta"].sum(0)
    return r
