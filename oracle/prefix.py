"""Float64 definitions of the operators over a shared prefix: rotation by position, appending to a paged
cache, attention of new rows to cached keys, and attention of packed sequences to their program's keys
and their own, with its gradient.

Plain loops over sequences and heads; gradients by the chain rule, written out.  Inputs are NumPy arrays of the
values that the library is given (bfloat16 tensors as the numbers they hold).
"""
from __future__ import annotations

import numpy as np


# ---- rotation ------------------------------------------------------------------------
def positions(off, first=None):
    """Position of every packed row."""
    out = np.zeros(off[-1], np.int64)
    for s in range(len(off) - 1):
        out[off[s]:off[s + 1]] = np.arange(off[s + 1] - off[s]) + (0 if first is None else int(first[s]))
    return out


def rotate(x, position, freq, interleaved=False, inverse=False):
    """x [rows][heads][dim], its first 2 len(freq) features turned by position x freq."""
    x = np.asarray(x, np.float64)
    h = len(freq)
    angle = position[:, None].astype(np.float64) * np.asarray(freq, np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    if inverse:
        s = -s
    i = np.arange(h)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


# ---- paged cache ---------------------------------------------------------------------
def append(k, v, k_cache, v_cache, pages, lens, off, first=None, freq=None, interleaved=False, q=None):
    """(q rotated, k_cache, v_cache) after the call."""
    k_cache, v_cache = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    page = k_cache.shape[2]
    at = np.zeros(off[-1], np.int64)
    for s in range(len(off) - 1):
        n = off[s + 1] - off[s]
        at[off[s]:off[s + 1]] = lens[s] - n + np.arange(n)
    seq = np.repeat(np.arange(len(off) - 1), np.diff(off))
    position = at + (0 if first is None else np.asarray(first)[seq])
    turn = (lambda x: np.asarray(x, np.float64)) if freq is None else (lambda x: rotate(x, position, freq, interleaved))
    k, q = turn(k), None if q is None else turn(q)
    for r in range(off[-1]):
        p = pages[seq[r], at[r] // page]
        k_cache[p, :, at[r] % page] = k[r]
        v_cache[p, :, at[r] % page] = np.asarray(v[r], np.float64)
    return q, k_cache, v_cache


def keys_of(cache, table, n):
    """The first n keys [n][kv_heads][dim] of a page table."""
    page = cache.shape[2]
    j = np.arange(n)
    return np.asarray(cache, np.float64)[np.asarray(table)[j // page], :, j % page]


# ---- attention -----------------------------------------------------------------------
def _softmax(q, k, scale, seen):
    """Weights and log-sums of rows over the keys they see (none: weights 0, -inf)."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.where(np.isfinite(top), top, 0.0) + np.log(total)
    return p / np.where(total == 0.0, 1.0, total), lse[:, 0]


def cached(q, k_cache, v_cache, pages, lens, off, scale, seg_off=None, prefix_pages=None, prefix_lens=None):
    """o and lse."""
    q = np.asarray(q, np.float64)
    o, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    G = q.shape[1] // k_cache.shape[1]
    for s in range(len(off) - 1):
        n, L = off[s + 1] - off[s], int(lens[s])
        if n == 0:
            continue
        k, v = keys_of(k_cache, pages[s], L), keys_of(v_cache, pages[s], L)
        seen = np.arange(L)[None] <= (L - n + np.arange(n))[:, None]
        if seg_off is not None:
            p = int(np.searchsorted(seg_off, s, side="right")) - 1
            P = int(prefix_lens[p])
            k = np.concatenate([keys_of(k_cache, prefix_pages[p], P), k])
            v = np.concatenate([keys_of(v_cache, prefix_pages[p], P), v])
            seen = np.concatenate([np.ones((n, P), bool), seen], 1)
        rows = slice(off[s], off[s + 1])
        for h in range(q.shape[1]):
            # what a row does not see is not used, whatever it holds
            for i in range(n):
                at = np.nonzero(seen[i])[0]
                w, z = _softmax(q[rows, h][i:i + 1], k[at, h // G], scale, np.ones((1, len(at)), bool))
                o[off[s] + i, h] = (w @ v[at, h // G])[0]
                lse[off[s] + i, h] = z[0]
    return o, lse


def _parts(q, k, v, pk, pv, off, q_off, p_off, mask):
    """Per (sequence, head): its rows, its program's shown keys, the head, its key head, which of [shown, own] a row sees."""
    G = q.shape[1] // k.shape[1]
    for p in range(len(q_off) - 1):
        shown = np.arange(p_off[p], p_off[p + 1])
        if mask is not None:
            shown = shown[np.asarray(mask)[shown] != 0]
        for s in range(len(off) - 1):
            a, b = max(off[s], q_off[p]), min(off[s + 1], q_off[p + 1])
            if a >= b:
                continue
            seen = np.concatenate([np.ones((b - a, len(shown)), bool), np.tril(np.ones((b - a, b - a), bool))], 1)
            for h in range(q.shape[1]):
                yield slice(a, b), shown, h, h // G, seen


def prefix(q, k, v, pk, pv, off, q_off, p_off, scale, mask=None):
    """o and lse."""
    q, k, v, pk, pv = (np.asarray(t, np.float64) for t in (q, k, v, pk, pv))
    o, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    for rows, shown, h, g, seen in _parts(q, k, v, pk, pv, off, q_off, p_off, mask):
        w, z = _softmax(q[rows, h], np.concatenate([pk[shown, g], k[rows, g]]), scale, seen)
        o[rows, h] = w @ np.concatenate([pv[shown, g], v[rows, g]])
        lse[rows, h] = z
    return o, lse


def prefix_grad(do, q, k, v, pk, pv, off, q_off, p_off, scale, mask=None, o=None):
    """dq, dk, dv, dpk, dpv.  o: the forward's result as the gradient is given it (rounded to the tensors' type)."""
    do, q, k, v, pk, pv = (np.asarray(t, np.float64) for t in (do, q, k, v, pk, pv))
    o = prefix(q, k, v, pk, pv, off, q_off, p_off, scale, mask)[0] if o is None else np.asarray(o, np.float64)
    dq, dk, dv, dpk, dpv = (np.zeros(t.shape) for t in (q, k, v, pk, pv))
    for rows, shown, h, g, seen in _parts(q, k, v, pk, pv, off, q_off, p_off, mask):
        keys, values = np.concatenate([pk[shown, g], k[rows, g]]), np.concatenate([pv[shown, g], v[rows, g]])
        w, _ = _softmax(q[rows, h], keys, scale, seen)
        ds = w * (do[rows, h] @ values.T - (do[rows, h] * o[rows, h]).sum(1, keepdims=True)) * scale
        dq[rows, h] = ds @ keys
        gk, gv, n = ds.T @ q[rows, h], w.T @ do[rows, h], len(shown)
        dpk[shown, g] += gk[:n]
        dpv[shown, g] += gv[:n]
        dk[rows, g] += gk[n:]
        dv[rows, g] += gv[n:]
    return dq, dk, dv, dpk, dpv


def grad_spread(do, q, k, v, pk, pv, off, q_off, p_off, scale, mask, o):
    """How far dq, dk, dv, dpk, dpv can be from prefix_grad's when any of the rows take the mean of their score gradients, do . o, from
    the exact o instead of this one: bounds element by element."""
    do, q, k, v, pk, pv, o = (np.asarray(t, np.float64) for t in (do, q, k, v, pk, pv, o))
    exact = prefix(q, k, v, pk, pv, off, q_off, p_off, scale, mask)[0]
    dq, dk, dv, dpk, dpv = (np.zeros(t.shape) for t in (q, k, v, pk, pv))
    for rows, shown, h, g, seen in _parts(q, k, v, pk, pv, off, q_off, p_off, mask):
        keys = np.concatenate([pk[shown, g], k[rows, g]])
        w, _ = _softmax(q[rows, h], keys, scale, seen)
        change = np.abs((do[rows, h] * (o - exact)[rows, h]).sum(1, keepdims=True)) * scale
        dq[rows, h] = np.abs(w @ keys) * change
        gk, n = (w * change).T @ np.abs(q[rows, h]), len(shown)
        dpk[shown, g] += gk[:n]
        dk[rows, g] += gk[n:]
    return dq, dk, dv, dpk, dpv
