"""Pins of oracle/train_ops.py (CPU): the definitions against finite differences, brute force, invariances and closed forms."""
import numpy as np
import pytest

from oracle import train_ops as O


def rng(seed):
    return np.random.RandomState(seed)


@pytest.mark.parametrize("shape,groups", [((2, 3, 4, 6), 3), ((1, 1, 1, 8), 2), ((3, 2, 2, 5), 1), ((2, 3, 3, 4), 4)])
def test_group_norm_by_loops(shape, groups):
    r = rng(1)
    x, gamma, beta = r.randn(*shape), r.randn(shape[3]), r.randn(shape[3])
    y, mean, rstd = O.group_norm_fwd(x, gamma, beta, groups, 1e-5)
    cg = shape[3] // groups
    for n in range(shape[0]):
        for g in range(groups):
            vals = [x[n, h, w, c] for h in range(shape[1]) for w in range(shape[2]) for c in range(g * cg, (g + 1) * cg)]
            m = sum(vals) / len(vals)
            var = sum((v - m) ** 2 for v in vals) / len(vals)
            assert abs(mean[n, g] - m) < 1e-12 and abs(rstd[n, g] - (var + 1e-5) ** -0.5) < 1e-9
            for c in range(g * cg, (g + 1) * cg):
                want = (x[n, :, :, c] - m) * (var + 1e-5) ** -0.5 * gamma[c] + beta[c]
                assert np.allclose(y[n, :, :, c], want, atol=1e-10)


def test_group_norm_does_not_see_offset_or_scale():
    r = rng(2)
    x = r.randn(2, 5, 5, 8)
    one, zero = np.ones(8), np.zeros(8)
    y = O.group_norm_fwd(x, one, zero, 4, 1e-12)[0]
    assert np.allclose(O.group_norm_fwd(3.0 * x + 7.0, one, zero, 4, 1e-12)[0], y, atol=1e-9)
    g = y.reshape(2, 25, 4, 2)
    assert np.allclose(g.mean(axis=(1, 3)), 0, atol=1e-12) and np.allclose(g.var(axis=(1, 3)), 1, atol=1e-9)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_group_norm_gradients_by_differences(act):
    r = rng(3)
    shape, groups = (2, 3, 3, 6), 3
    x, gamma, beta, dy = r.randn(*shape), 1 + 0.3 * r.randn(6), 0.3 * r.randn(6), r.randn(*shape)
    y, mean, rstd = O.group_norm_fwd(x, gamma, beta, groups, 1e-3, act)
    dx, dgamma, dbeta = O.group_norm_bwd(x, dy, gamma, beta, mean, rstd, groups, act, y if act == "relu" else None)
    loss = lambda x_, g_, b_: float((O.group_norm_fwd(x_, g_, b_, groups, 1e-3, act)[0] * dy).sum())   # noqa: E731
    h = 1e-6
    for which, arr, grad in ((0, x, dx), (1, gamma, dgamma), (2, beta, dbeta)):
        for i in r.choice(arr.size, min(arr.size, 24), replace=False):
            lo, hi = arr.copy(), arr.copy()
            lo.flat[i] -= h
            hi.flat[i] += h
            args = [x, gamma, beta]
            up, down = list(args), list(args)
            up[which], down[which] = hi, lo
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad.flat[i]) < 1e-6
    if act == "relu":   # a gradient that has been masked before gives the same
        again = O.group_norm_bwd(x, dy * (y > 0), gamma, beta, mean, rstd, groups, act, None)
        assert all(np.array_equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))


def test_grad_norm():
    assert O.grad_norm([[3.0], [0.0, 4.0]], 1.0) == (5.0, 0.2)
    assert O.grad_norm([[3.0], [0.0, 4.0]], 10.0) == (5.0, 1.0)
    assert O.grad_norm([], 1.0) == (0.0, 1.0)
    assert O.grad_norm([[1.0, np.inf]], 1.0)[1] == 0.0 and O.grad_norm([[np.nan]], 1.0)[1] == 0.0


def test_adamw_closed_forms():
    h = dict(lr=0.01, beta1=0.9, beta2=0.999, eps=1e-8)
    w, z = np.array([1.0, -2.0, 3.0]), np.zeros(3)
    g = np.array([0.5, -1e-3, 0.0])
    # the first step moves every weight by lr against the sign of its gradient
    w1, m, v = O.adamw(w, z, z, g, step=1, **h)
    assert np.allclose(w1, w - 0.01 * np.sign(g), atol=1e-6)
    # so does every step under a constant gradient
    for step in range(2, 50):
        w1, m, v = O.adamw(w1, m, v, g, step=step, **h)
    assert np.allclose(w1, w - 0.49 * np.sign(g), atol=1e-4)
    # decay alone, and a scale that is the gradient's
    assert np.allclose(O.adamw(w, z, z, z, step=1, weight_decay=0.1, **h)[0], w * (1 - 0.001))
    a, b = O.adamw(w, z, z, g, step=1, scale=0.25, **h), O.adamw(w, z, z, 0.25 * g, step=1, **h)
    assert all(np.array_equal(p, q) for p, q in zip(a, b))
    for skipped in (0.0, np.nan):
        assert all(np.array_equal(p, q) for p, q in zip(O.adamw(w, g, g, g, step=3, scale=skipped, **h), (w, g, g)))


def test_splitmix64_known_values():
    # first outputs for seed 1234567, as published with the generator
    got = [int(v) for v in O.splitmix64(1234567, np.arange(3))]
    assert got == [6457827717110365317, 3203168211198807973, 9817491932198370423]


def test_e4m3_table():
    v = O.e4m3_values()
    assert len(v) == 127 and v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[126] == 448.0
    assert np.all(np.diff(v) > 0)
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(t, O.decode8(np.arange(256)).astype(np.float32), equal_nan=True)


def test_round8_is_unbiased_and_keeps_representable_values():
    every = np.arange(65536)
    for a in (448.0, 447.0, 1.0, 1.03, 0.9999, 2.0 ** -6, 0.0151, 2.0 ** -9, 0.7 * 2.0 ** -9, 1e-5, 0.0):
        got = O.e4m3_values()[O.round8(np.full(65536, a), every)]
        gap = max(2.0 ** -9, 2.0 ** (np.floor(np.log2(a)) - 3)) if a > 0 else 1.0
        assert abs(got.mean() - a) <= gap * 2.0 ** -15   # 16 random bits
        assert len(np.unique(got)) <= 2
        if a in O.e4m3_values():
            assert np.all(got == a)


def test_store8():
    r = rng(4)
    x = r.randn(700) * np.exp(r.randn(700))
    x[256:512] = 0.0
    codes, scales = O.store8(x, r.randint(0, 65536, 700))
    back = O.load8(codes, scales)
    assert scales.shape == (3,) and scales[1] == 0 and np.all(back[256:512] == 0)
    top = np.abs(x[:256]).max()
    assert np.abs(back[:256]).max() == pytest.approx(top) and np.abs(back[:256] - x[:256]).max() <= top * 32 / 448
    codes, _ = O.store8(np.array([1.0, 1e-9, 0.0]), np.zeros(3, dtype=np.int64), positive=True)
    assert list(codes) == [126, 1, 0]


def test_logprobs_plain_cases():
    logp, ent, lse, top, at = O.logprobs(np.zeros((1, 8)), [3], 3)
    assert np.allclose(logp, -np.log(8)) and np.allclose(ent, np.log(8)) and np.allclose(lse, np.log(8))
    assert list(at[0]) == [0, 1, 2] and np.allclose(top, -np.log(8))
    z = np.array([[1.0, 3.0, -np.inf, 3.0, 2.0], [-np.inf] * 5, [0.0, 1.0, 2.0, 3.0, 4.0]])
    logp, ent, lse, top, at = O.logprobs(z, [2, 0, 7], 5)
    assert logp[0] == -np.inf and logp[1] == -np.inf and logp[2] == 0.0
    assert list(at[0]) == [1, 3, 4, 0, 2] and list(at[1]) == [0, 1, 2, 3, 4] and ent[1] == 0 and lse[1] == -np.inf
    p = np.exp(z[0] - lse[0])
    assert abs(p.sum() - 1) < 1e-12 and abs(ent[0] + sum(q * np.log(q) for q in p if q > 0)) < 1e-12
    assert np.isnan(O.logprobs(np.array([[1.0, np.nan, 5.0]]), [0], 2)[0][0]) and list(O.logprobs(np.array([[1.0, np.nan, 5.0]]), [0], 2)[4][0]) == [1, 2]


def test_logprobs_gradient_by_differences():
    r = rng(5)
    z = 2 * r.randn(3, 7)
    z[1, 2] = -np.inf
    ids, dlogp, dent = [4, 0, -1], r.randn(3), r.randn(3)
    dz = O.logprobs_bwd(z, ids, dlogp, dent)
    loss = lambda zz: float((O.logprobs(zz, ids, 0)[0] * dlogp).sum() + (O.logprobs(zz, ids, 0)[1] * dent).sum())   # noqa: E731
    for i in range(z.size):
        if not np.isfinite(z.flat[i]):
            assert dz.flat[i] == 0
            continue
        lo, hi = z.copy(), z.copy()
        lo.flat[i] -= 1e-6
        hi.flat[i] += 1e-6
        assert abs((loss(hi) - loss(lo)) / 2e-6 - dz.flat[i]) < 1e-7
    assert np.all(O.logprobs_bwd(np.full((1, 4), -np.inf), [1], [1.0], [1.0]) == 0)


def test_states_in_fp32_follow_the_definition_in_64_bits():
    r = rng(6)
    n = 3000
    m8, ms = O.store8(r.randn(n) * 1e-3, r.randint(0, 65536, n))
    v8, vs = O.store8(np.abs(r.randn(n)) * 1e-2 + 1e-4, r.randint(0, 65536, n), True)
    g = (r.randn(n) * 1e-2).astype(np.float32)
    ms, vs = ms.astype(np.float32), vs.astype(np.float32)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=3)
    _, cm, sm, cv, sv = O.adamw8(np.zeros(n), m8, ms, v8, vs, g, 11, 4096, **hyper)
    got = O.adamw8_states_f32(m8, ms, v8, vs, g, 11, 4096, 0.9, 0.999)
    assert np.allclose(got[1], sm, rtol=1e-5) and np.allclose(got[3], sv, rtol=1e-6)
    for a, b in ((got[0], cm), (got[2], cv)):
        assert (a != b).sum() <= 2 and np.abs((a & 127).astype(int) - (b & 127)).max() <= 1
