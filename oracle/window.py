"""Windowed jagged HSTU attention and its one-token form, in float64 (numpy),
written from the definition: test infrastructure, shares no code with the HIP
path.

A query i sees key j <= i of its sequence if i - j < window or j < sinks;
everything else is the attention of oracle.py.
"""
from __future__ import annotations

import numpy as np

LN_EPS = 1e-6


def bucket(x, nb):
    """|x| < 4 -> |x|; else four buckets an octave by the two bits under the
    leading one; clamped to nb - 1."""
    x = np.atleast_1d(np.abs(np.asarray(x, dtype=np.int64)))
    out = np.minimum(x, 3).astype(np.int64)
    big = x >= 4
    y = x[big]
    e = np.zeros_like(y)
    rest = y.copy()
    while np.any(rest > 1):
        e += rest > 1
        rest >>= 1
    out[big] = 4 * (e - 1) + ((y >> (e - 2)) & 3)
    return np.minimum(out, nb - 1)


def seen(L, window, sinks):
    """[L][L] truth values: query (row) sees key (column)."""
    i = np.arange(L)[:, None]
    j = np.arange(L)[None, :]
    return (j <= i) & ((i - j < window) | (j < sinks))


def _bias(h, i, j, ts, N, pos_w, time_w):
    b = np.zeros(np.broadcast(i, j).shape)
    if pos_w is not None:
        b = b + pos_w[h][j - i + N - 1]
    if time_w is not None:
        b = b + time_w[h][bucket(ts[i] - ts[j], time_w.shape[1])]
    return b


def _layer_norm(o):
    mean = o.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((o - mean) ** 2).mean(1, keepdims=True) + LN_EPS)
    return (o - mean) * rstd, rstd


def attention(q, k, v, u, off, N, window, sinks, pos_w=None, time_w=None, ts=None, dy=None,
              alpha=1.0):
    """q, k, v, u, dy [T][H][d] (u, dy also [T][H*d]; any float type), off [B+1]; the outputs
    of the forward, and with dy of the backward, by name."""
    f = lambda x: None if x is None else np.asarray(x, dtype=np.float64)
    q, k, v, u, dy, pos_w, time_w = map(f, (q, k, v, u, dy, pos_w, time_w))
    T, H, d = q.shape
    u = u.reshape(T, H * d)
    dy = None if dy is None else dy.reshape(T, H * d)
    o = np.zeros((T, H, d))
    for b in range(len(off) - 1):
        r = slice(int(off[b]), int(off[b + 1]))
        L = r.stop - r.start
        if L == 0:
            continue
        i, j = np.arange(L)[:, None], np.arange(L)[None, :]
        m = seen(L, window, sinks)
        for h in range(H):
            s = alpha * (q[r, h] @ k[r, h].T) + _bias(h, i, j, None if ts is None else ts[r], N,
                                                      pos_w, time_w)
            a = np.where(m, s / (1.0 + np.exp(-s)) / N, 0.0)
            o[r, h] = a @ v[r, h]
    n, rstd = _layer_norm(o.reshape(T, H * d))
    out = dict(o=o, y=n * u)
    if dy is None:
        return out
    g = dy * u
    dO = rstd * (g - g.mean(1, keepdims=True) - n * (g * n).mean(1, keepdims=True))
    dO = dO.reshape(T, H, d)
    out.update(du=n * dy, dq=np.zeros((T, H, d)), dk=np.zeros((T, H, d)),
               dv=np.zeros((T, H, d)),
               d_pos=None if pos_w is None else np.zeros_like(pos_w),
               d_time=None if time_w is None else np.zeros_like(time_w))
    for b in range(len(off) - 1):
        r = slice(int(off[b]), int(off[b + 1]))
        L = r.stop - r.start
        if L == 0:
            continue
        i, j = np.arange(L)[:, None], np.arange(L)[None, :]
        m = seen(L, window, sinks)
        t = None if ts is None else ts[r]
        for h in range(H):
            s = alpha * (q[r, h] @ k[r, h].T) + _bias(h, i, j, t, N, pos_w, time_w)
            sg = 1.0 / (1.0 + np.exp(-s))
            a = np.where(m, s * sg / N, 0.0)
            ds = np.where(m, (dO[r, h] @ v[r, h].T) * sg * (1.0 + s * (1.0 - sg)) / N, 0.0)
            out["dq"][r, h] = alpha * ds @ k[r, h]
            out["dk"][r, h] = alpha * ds.T @ q[r, h]
            out["dv"][r, h] = a.T @ dO[r, h]
            if pos_w is not None:
                np.add.at(out["d_pos"][h], np.broadcast_to(j - i + N - 1, (L, L)), ds)
            if time_w is not None:
                np.add.at(out["d_time"][h], bucket(t[i] - t[j], time_w.shape[1]), ds)
    return out


def one_token(q, u, k, v, N, window, sinks, pos_w=None, time_w=None, ts=None, alpha=1.0):
    """The last token of one sequence: q [H][d], u [H*d], its whole history k, v
    [L][H][d] (ts [L]), the token itself last; (o [H][d], y [H*d])."""
    f = lambda x: None if x is None else np.asarray(x, dtype=np.float64)
    q, u, k, v, pos_w, time_w = map(f, (q, u, k, v, pos_w, time_w))
    L, H = k.shape[0], q.shape[0]
    o = np.zeros(q.shape)
    if L > 0:
        j = np.nonzero(seen(L, window, sinks)[L - 1])[0]
        for h in range(H):
            s = alpha * (k[j, h] @ q[h]) + _bias(h, np.full(j.shape, L - 1), j, ts, N, pos_w,
                                                 time_w)
            o[h] = (s / (1.0 + np.exp(-s)) / N) @ v[j, h]
    n, _ = _layer_norm(o.reshape(1, -1))
    return o, n[0] * u
