"""fp64 oracle of the head norm with rotary positions and of attention, from their definitions; loops over sequences and heads, numpy only."""
import numpy as np


# ---- norm and rotary position ---------------------------------------------------------------------------------------

def _pairs(dim, pairs, halves):
    """(first channel, second channel) of every pair."""
    P = sum(pairs)
    return (np.arange(P), np.arange(P) + P) if halves else (2 * np.arange(P), 2 * np.arange(P) + 1)


def _angles(pos, freq, pairs):
    axis = np.repeat(np.arange(len(pairs)), pairs)
    return np.asarray(pos, dtype=np.float64)[:, axis] * np.asarray(freq, dtype=np.float64)


def rotate(x, pos, freq, pairs, halves, back=False):
    """x [rows, heads, dim]."""
    a, b = _pairs(x.shape[2], pairs, halves)
    t = _angles(pos, freq, pairs)[:, None, :] * (-1 if back else 1)
    y = x.copy()
    y[:, :, a] = x[:, :, a] * np.cos(t) - x[:, :, b] * np.sin(t)
    y[:, :, b] = x[:, :, a] * np.sin(t) + x[:, :, b] * np.cos(t)
    return y


def qk_rotary(x, gamma, pos, freq, pairs, halves, norm, eps):
    """y of one side, x [rows, heads, dim]."""
    x = np.asarray(x, dtype=np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * (1.0 if gamma is None else np.asarray(gamma, dtype=np.float64))
    return rotate(x, pos, freq, pairs, halves)


def qk_rotary_bwd(x, gamma, pos, freq, pairs, halves, norm, eps, dy):
    """(dx, dgamma)."""
    g = rotate(np.asarray(dy, dtype=np.float64), pos, freq, pairs, halves, back=True)
    if not norm:
        return g, None
    x = np.asarray(x, dtype=np.float64)
    r = 1 / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    t = g * (1.0 if gamma is None else np.asarray(gamma, dtype=np.float64))
    return r * (t - x * r * r * (t * x).mean(axis=2, keepdims=True)), (g * x * r).sum(axis=(0, 1))


# ---- attention ------------------------------------------------------------------------------------------------------

def sees(lq, lk, left, right):
    """[lq, lk]: the last query stands at the last key."""
    place = np.arange(lq)[:, None] + lk - lq
    j = np.arange(lk)[None, :]
    return ((left < 0) | (j >= place - left)) & ((right < 0) | (j <= place + right))


def _softmax(q, k, scale, mask):
    s = np.where(mask, scale * (q @ k.T), -np.inf)
    m = s.max(axis=1, initial=-np.inf)
    e = np.where(mask, np.exp(s - np.where(np.isfinite(m), m, 0.0)[:, None]), 0.0)
    total = e.sum(axis=1)
    some = total > 0
    p = e / np.where(some, total, 1.0)[:, None]
    return p, np.where(some, m + np.log(np.where(some, total, 1.0)), -np.inf)


def attention(q, k, v, seqs, scale, left, right):
    """q [rows, heads, dim], k, v [rows, kv_heads, dim]; seqs: (first query, queries, first key, keys) of each sequence.
    Returns o, lse [heads, rows], and size [rows, heads, dim] = sum p |v|, which roundings of p are relative to."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    h, share = q.shape[1], q.shape[1] // k.shape[1]
    o, lse, size = np.zeros(q.shape), np.full((h, q.shape[0]), -np.inf), np.zeros(q.shape)
    for q0, lq, k0, lk in seqs:
        mask = sees(lq, lk, left, right)
        for i in range(h):
            kk, vv = k[k0:k0 + lk, i // share], v[k0:k0 + lk, i // share]
            p, l = _softmax(q[q0:q0 + lq, i], kk, scale, mask)
            o[q0:q0 + lq, i], lse[i, q0:q0 + lq], size[q0:q0 + lq, i] = p @ vv, l, p @ np.abs(vv)
    return o, lse, size


def attention_bwd(q, k, v, o, dout, seqs, scale, left, right):
    """(dq, dk, dv) with delta = dout . o of the o given; and for each the two sizes that errors are relative to: of the rounded factor
    (ds or p) times the other one, and of everything that was added up to it."""
    q, k, v, o, dout = (np.asarray(t, dtype=np.float64) for t in (q, k, v, o, dout))
    h, share = q.shape[1], q.shape[1] // k.shape[1]
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    rounded, added = [np.zeros(t.shape) for t in out], [np.zeros(t.shape) for t in out]
    for q0, lq, k0, lk in seqs:
        mask = sees(lq, lk, left, right)
        for i in range(h):
            g = i // share
            qi, oi, di, kk, vv = q[q0:q0 + lq, i], o[q0:q0 + lq, i], dout[q0:q0 + lq, i], k[k0:k0 + lk, g], v[k0:k0 + lk, g]
            p, _ = _softmax(qi, kk, scale, mask)
            ds = p * (di @ vv.T - (di * oi).sum(axis=1)[:, None])
            all_ds = p * (np.abs(di) @ np.abs(vv).T + np.abs(di * oi).sum(axis=1)[:, None])
            rows, keys = (slice(q0, q0 + lq), i), (slice(k0, k0 + lk), g)
            for n, at, left_factor, size, right_factor in ((0, rows, ds, all_ds, kk), (1, keys, ds.T, all_ds.T, qi), (2, keys, p.T, p.T, di)):
                f = 1.0 if n == 2 else scale
                out[n][at] += f * (left_factor @ right_factor)
                rounded[n][at] += f * (np.abs(left_factor) @ np.abs(right_factor))
                added[n][at] += f * (np.abs(size) @ np.abs(right_factor))
    return out, rounded, added
