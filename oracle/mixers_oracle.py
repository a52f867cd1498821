"""Plain numpy fp64 implementations of the mixers beside the layer, written from their definitions: linear attention with
a decay for each KV head (token by token) and sliding-window attention with sinks (pair by pair), with their
gradients.  q [B, T, Hq, d]; k, v [B, T, Hkv, d]; lens [B] or None.  Test infrastructure only."""
import math

import numpy as np


def _lens(lens, B, T):
    return [T] * B if lens is None else [int(min(max(n, 0), T)) for n in lens]


def linear(q, k, v, log_decay, state=None, lens=None, scale=None):
    """(out, state behind the last token)."""
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out = np.zeros_like(q)
    S = np.zeros((B, Hkv, d, d)) if state is None else state.copy()
    lam = np.exp(np.asarray(log_decay, np.float64))
    for b, n in enumerate(_lens(lens, B, T)):
        for h in range(Hkv):
            for t in range(n):
                S[b, h] = lam[h] * S[b, h] + np.outer(k[b, t, h], v[b, t, h])
                out[b, t, h * G:(h + 1) * G] = scale * q[b, t, h * G:(h + 1) * G] @ S[b, h]
    return out, S


def linear_backward(q, k, v, log_decay, dout, state=None, dstate=None, lens=None, scale=None):
    """(dq, dk, dv, gradient of the state at the start)."""
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    lam = np.exp(np.asarray(log_decay, np.float64))
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    R = np.zeros((B, Hkv, d, d)) if dstate is None else dstate.copy()
    for b, n in enumerate(_lens(lens, B, T)):
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            S = np.zeros((d, d)) if state is None else state[b, h].copy()
            for t in range(n):
                S = lam[h] * S + np.outer(k[b, t, h], v[b, t, h])
                dq[b, t, heads] = scale * dout[b, t, heads] @ S.T
            for t in range(n - 1, -1, -1):
                R[b, h] += scale * q[b, t, heads].T @ dout[b, t, heads]
                dk[b, t, h] = R[b, h] @ v[b, t, h]
                dv[b, t, h] = k[b, t, h] @ R[b, h]
                R[b, h] *= lam[h]
    return dq, dk, dv, R


def window_sees(t, n_keys, window, n_sink):
    """Positions that a query at position t sees."""
    return [j for j in range(min(t + 1, n_keys)) if t - j < window or j < n_sink]


def window(q, k, v, window, n_sink=0, lens=None, scale=None):
    """(out, lse) of q [B, Tq, Hq, d] over k, v [B, Tk, Hkv, d]: query i stands at position i + Tk - Tq."""
    B, Tq, Hq, d = q.shape
    Tk, Hkv = k.shape[1:3]
    G = Hq // Hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, lse = np.zeros_like(q), np.full((B, Tq, Hq), -np.inf)
    for b, n in enumerate(_lens(lens, B, Tk)):
        for i in range(Tq):
            t = i + Tk - Tq
            if t >= n:
                continue
            seen = window_sees(t, n, window, n_sink)
            for h in range(Hq):
                s = scale * k[b, seen, h // G] @ q[b, i, h]
                m = s.max()
                p = np.exp(s - m)
                lse[b, i, h] = m + math.log(p.sum())
                out[b, i, h] = (p / p.sum()) @ v[b, seen, h // G]
    return out, lse


def window_backward(q, k, v, dout, window, n_sink=0, lens=None, scale=None, absolute=False):
    """(dq, dk, dv); absolute: the same sums over the absolute values of their terms (for bounds), with |dP| + |D| for dP - D."""
    B, Tq, Hq, d = q.shape
    Tk, Hkv = k.shape[1:3]
    G = Hq // Hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    mag = np.abs if absolute else (lambda x: x)
    for b, n in enumerate(_lens(lens, B, Tk)):
        for i in range(Tq):
            t = i + Tk - Tq
            if t >= n:
                continue
            seen = window_sees(t, n, window, n_sink)
            for h in range(Hq):
                kk, vv = k[b, seen, h // G], v[b, seen, h // G]
                s = scale * kk @ q[b, i, h]
                p = np.exp(s - s.max())
                p /= p.sum()
                dp, do = mag(vv) @ mag(dout[b, i, h]), mag(dout[b, i, h])
                D = mag(p @ vv) @ do if absolute else p @ dp
                ds = scale * p * (dp + D if absolute else dp - D)
                dq[b, i, h] = ds @ mag(kk)
                np.add.at(dk[b, :, h // G], seen, np.outer(ds, mag(q[b, i, h])))
                np.add.at(dv[b, :, h // G], seen, np.outer(p, do))
    return dq, dk, dv
