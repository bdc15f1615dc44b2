"""Oracle of group normalisation, the gradient norm, AdamW and log-probabilities.

TEST INFRASTRUCTURE ONLY (see the package docstring).  numpy, fp64, each function the plain definition; the 8-bit states'
random bits and rounding are whole-number definitions and are written out as such.

Pins (tests/test_train_ops_pins.py): finite differences of every gradient, loop-written brute force, invariances of the norm,
closed forms of AdamW's first step and of constant gradients, SplitMix64's published values, unbiased rounding, the entropy of uniform rows.
Layouts: x [N,H,W,C]; z [rows,classes].
"""
import numpy as np


# ---- group norm ---------------------------------------------------------------------------------------------------

def _groups(a, groups):
    n, h, w, c = a.shape
    return a.reshape(n, h * w, groups, c // groups)


def group_norm_stats(x, groups, eps):
    """(mean, rstd), each [N, groups]."""
    g = _groups(np.asarray(x, dtype=np.float64), groups)
    mean = g.mean(axis=(1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def _xhat(x, mean, rstd, groups):
    g = _groups(np.asarray(x, dtype=np.float64), groups)
    return ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(np.shape(x))


def _sigmoid(u):
    return 0.5 * (1.0 + np.tanh(0.5 * u))


def group_norm_fwd(x, gamma, beta, groups, eps, act="none"):
    """(y, mean, rstd); act: "none", "relu" or "silu"."""
    mean, rstd = group_norm_stats(x, groups, eps)
    u = _xhat(x, mean, rstd, groups) * gamma + beta
    y = np.maximum(u, 0.0) if act == "relu" else u * _sigmoid(u) if act == "silu" else u
    return y, mean, rstd


def group_norm_bwd(x, dy, gamma, beta, mean, rstd, groups, act="none", y_saved=None):
    """(dx, dgamma, dbeta); act "relu" masks by y_saved, or takes dy as masked already where y_saved is None."""
    g = np.asarray(dy, dtype=np.float64)
    mean, rstd = np.asarray(mean, dtype=np.float64), np.asarray(rstd, dtype=np.float64)
    xhat = _xhat(x, mean, rstd, groups)
    if act == "relu" and y_saved is not None:
        g = g * (np.asarray(y_saved) > 0)
    if act == "silu":
        u = xhat * gamma + beta
        s = _sigmoid(u)
        g = g * (s + u * s * (1.0 - s))
    t, xg = _groups(g * gamma, groups), _groups(xhat, groups)
    dx = (t - t.mean(axis=(1, 3), keepdims=True) - xg * (t * xg).mean(axis=(1, 3), keepdims=True)) * rstd[:, None, :, None]
    return dx.reshape(np.shape(x)), (g * xhat).sum(axis=(0, 1, 2)), g.sum(axis=(0, 1, 2))


# ---- optimizer ----------------------------------------------------------------------------------------------------

def grad_norm(grads, max_norm):
    """(norm, scale)."""
    with np.errstate(over="ignore", invalid="ignore"):
        norm = float(np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads)))
    if not np.isfinite(norm):
        return norm, 0.0
    return norm, min(1.0, max_norm / norm) if norm > 0 else 1.0


def adamw(w, m, v, g, lr, beta1, beta2, eps, step, weight_decay=0.0, scale=1.0):
    """(w', m', v')."""
    w, m, v, g = (np.asarray(a, dtype=np.float64) for a in (w, m, v, g))
    if not abs(scale) > 0:
        return w, m, v
    g = g * scale
    m2 = beta1 * m + (1 - beta1) * g
    v2 = beta2 * v + (1 - beta2) * g * g
    mhat, vhat = m2 / (1 - beta1 ** step), v2 / (1 - beta2 ** step)
    return w - lr * weight_decay * w - lr * mhat / (np.sqrt(vhat) + eps), m2, v2


BLOCK, CHUNK = 256, 4096


def splitmix64(seed, counter):
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + (np.asarray(counter, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def random16(seed, first, count):
    """(for m, for v): 16 random bits for each of the elements number first ... first + count - 1 of a parameter list."""
    e = np.arange(first, first + count, dtype=np.uint64)
    z = splitmix64(seed, e >> np.uint64(1)) >> ((e & np.uint64(1)) * np.uint64(32))
    return (z & np.uint64(0xffff)).astype(np.int64), ((z >> np.uint64(16)) & np.uint64(0xffff)).astype(np.int64)


def e4m3_values():
    """The 127 finite values of codes 0 ... 126 (sign bit clear)."""
    c = np.arange(127)
    e, f = c >> 3, c & 7
    return np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))


def decode8(codes):
    codes = np.asarray(codes, dtype=np.uint8)
    v = np.append(e4m3_values(), np.nan)[codes & 127]
    return np.where(codes & 128, -v, v)


def round8(a, rnd16):
    """Codes of a >= 0 (at most 448): the upper neighbour where (distance from the lower, in their gap) + rnd16 / 2^16 >= 1."""
    vals = e4m3_values()
    lo = np.clip(np.searchsorted(vals, a, side="right") - 1, 0, 126)
    gap = np.where(lo < 126, np.append(np.diff(vals), 1.0)[lo], 1.0)
    frac = (a - vals[lo]) / gap
    return np.minimum(lo + ((frac + rnd16 / 65536.0) >= 1.0), 126).astype(np.uint8)


def block_top(x):
    """Largest magnitude of each 256 elements."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    return np.array([x[i:i + BLOCK].max() for i in range(0, len(x), BLOCK)])


def store8(x, rnd16, positive=False):
    """(codes, scales): x by blocks of 256, the largest magnitude at 448.  positive: a value above 0 keeps code 1 at least."""
    x = np.asarray(x, dtype=np.float64)
    top = block_top(x)
    each = np.repeat(top, BLOCK)[:len(x)]
    a = np.where(each > 0, np.abs(x) * 448.0 / np.where(each > 0, each, 1.0), 0.0)
    codes = round8(a, rnd16)
    if positive:
        codes = np.where(a > 0, np.maximum(codes, 1), codes).astype(np.uint8)
    return np.where(x < 0, codes | 128, codes).astype(np.uint8), top / 448.0


def load8(codes, scales):
    return decode8(codes) * np.repeat(np.asarray(scales, dtype=np.float64), BLOCK)[:len(codes)]


def adamw8(w, m8, ms, v8, vs, g, seed, first, **hyper):
    """(w', m codes, m scales, v codes, v scales); `first`: number of the tensor's first element in its list."""
    m, root = load8(m8, ms), load8(v8, vs)
    w2, m2, v2 = adamw(w, m, root * root, g, **hyper)
    if not abs(hyper.get("scale", 1.0)) > 0:
        return w2, m8, ms, v8, vs
    rm, rv = random16(seed, first, len(np.asarray(g)))
    return (w2, *store8(m2, rm), *store8(np.sqrt(v2), rv, positive=True))


# The moments and their 8-bit storage with every operation rounded to fp32 in the order of the definition: what an
# implementation of that definition returns bit for bit.

def moments_f32(m, v, g, beta1, beta2, scale=1.0):
    f = np.float32
    g = np.asarray(g, dtype=f) * f(scale)
    m2 = f(beta1) * np.asarray(m, dtype=f) + f(1 - beta1) * g
    return m2, f(beta2) * np.asarray(v, dtype=f) + f(1 - beta2) * (g * g)


def load8_f32(codes, scales):
    return decode8(codes).astype(np.float32) * np.repeat(np.asarray(scales, dtype=np.float32), BLOCK)[:len(codes)]


def store8_f32(x, rnd16, positive=False):
    f = np.float32
    x = np.asarray(x, dtype=f)
    top = block_top(x).astype(f)
    inv = np.where(top > 0, f(448) * (f(1) / np.where(top > 0, top, f(1))), f(0)).astype(f)
    a = np.abs(x) * np.repeat(inv, BLOCK)[:len(x)]
    codes = round8(np.minimum(a, f(448)).astype(np.float64), rnd16)
    small = (a * f(512) + rnd16.astype(f) * f(1 / 65536)).astype(f).astype(np.int32)   # multiples of 2^-9: the sum is rounded too
    codes = np.where(a < 2.0 ** -6, small, codes)
    if positive:
        codes = np.where(a > 0, np.maximum(codes, 1), codes)
    return np.where(x < 0, codes | 128, codes).astype(np.uint8), top * f(1 / 448)


def adamw8_states_f32(m8, ms, v8, vs, g, seed, first, beta1, beta2, scale=1.0):
    """(m codes, m scales, v codes, v scales)."""
    root = load8_f32(v8, vs)
    m, v = moments_f32(load8_f32(m8, ms), root * root, g, beta1, beta2, scale)
    rm, rv = random16(seed, first, len(m))
    return (*store8_f32(m, rm), *store8_f32(np.sqrt(v), rv, positive=True))


# ---- log-probabilities --------------------------------------------------------------------------------------------

def logprobs(z, ids, top_k):
    """(logp, entropy, lse, top_logp, top_ids) of rows of scores; an id outside the classes gives 0."""
    z = np.asarray(z, dtype=np.float64)
    rows, classes = z.shape
    logp, ent, lse = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    top, at = np.zeros((rows, top_k)), np.zeros((rows, top_k), dtype=np.int32)
    for r in range(rows):
        rank = np.where(np.isnan(z[r]), np.inf, z[r])
        order = np.lexsort((np.arange(classes), -rank, ~np.isnan(z[r])))[:top_k]   # NaN first, then by value, then by index
        at[r] = order
        m = z[r].max()
        if m == -np.inf:
            lse[r], top[r] = -np.inf, -np.inf
            logp[r] = -np.inf
        else:
            with np.errstate(invalid="ignore"):
                lse[r] = m + np.log(np.exp(z[r] - m).sum())
                p = np.exp(z[r] - lse[r])
                ent[r] = -sum_p_log_p(p)
                top[r] = z[r][order] - lse[r]
                if 0 <= ids[r] < classes:
                    logp[r] = z[r][ids[r]] - lse[r]
        if not 0 <= ids[r] < classes:
            logp[r] = 0.0
    return logp, ent, lse, top, at


def sum_p_log_p(p):
    return (p * np.log(np.where(p > 0, p, 1.0))).sum()


def logprobs_bwd(z, ids, dlogp, dentropy):
    """d(sum dlogp logp + dentropy entropy) / dz."""
    z = np.asarray(z, dtype=np.float64)
    dz = np.zeros_like(z)
    for r in range(len(z)):
        m = z[r].max()
        if m == -np.inf:
            continue
        p = np.exp(z[r] - m) / np.exp(z[r] - m).sum()
        h = -sum_p_log_p(p)
        dz[r] = -dentropy[r] * p * (np.log(np.where(p > 0, p, 1.0)) + h)
        if 0 <= ids[r] < z.shape[1]:
            dz[r] -= dlogp[r] * p
            dz[r][ids[r]] += dlogp[r]
    return dz
