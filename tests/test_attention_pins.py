"""Pins of oracle/attention_ops.py: closed forms, finite differences, and independence of parts that must not matter."""
import numpy as np
import pytest

from oracle import attention_ops as O

R = np.random.default_rng(5)


def difference(f, x, d, h=1e-6):
    """Derivative of the scalar f at x in direction d."""
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("pairs", [[3], [1, 2], [2, 1, 1]])
def test_rotation_is_one(pairs, halves):
    x, pos = R.normal(size=(5, 2, 8)), R.uniform(0, 50, size=(5, len(pairs)))
    freq = R.uniform(0.01, 1, size=sum(pairs))
    y = O.rotate(x, pos, freq, pairs, halves)
    assert np.allclose((x ** 2).sum(axis=2), (y ** 2).sum(axis=2), rtol=1e-12)
    assert np.allclose(O.rotate(y, pos, freq, pairs, halves, back=True), x, atol=1e-12)
    assert np.array_equal(y[:, :, 2 * sum(pairs):], x[:, :, 2 * sum(pairs):])
    # products of a query and a key depend on how far apart they are, not on where they stand
    a = O.rotate(x, pos, freq, pairs, halves)[0, 0] @ O.rotate(x, pos + 3, freq, pairs, halves)[0, 1]
    b = O.rotate(x, pos + 7, freq, pairs, halves)[0, 0] @ O.rotate(x, pos + 10, freq, pairs, halves)[0, 1]
    assert abs(a - b) < 1e-12


def test_quarter_turns():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    freq = np.array([np.pi / 2, np.pi])
    assert np.allclose(O.rotate(x, np.ones((1, 1)), freq, [2], False), [[[-2, 1, -3, -4]]])
    assert np.allclose(O.rotate(x, np.ones((1, 1)), freq, [2], True), [[[-3, -2, 1, -4]]])


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_gradient(halves, norm):
    x, gamma, pos, freq = R.normal(size=(4, 3, 8)), R.normal(size=8), R.uniform(0, 9, size=(4, 2)), R.uniform(0, 1, size=3)
    dy = R.normal(size=x.shape)
    args = (pos, freq, [2, 1], halves, norm, 1e-3)
    dx, dgamma = O.qk_rotary_bwd(x, gamma, *args, dy)
    d = R.normal(size=x.shape)
    assert abs(difference(lambda t: (O.qk_rotary(t, gamma, *args) * dy).sum(), x, d) - (dx * d).sum()) < 1e-7
    if norm:
        d = R.normal(size=8)
        assert abs(difference(lambda t: (O.qk_rotary(x, t, *args) * dy).sum(), gamma, d) - (dgamma * d).sum()) < 1e-7


SEQS = [(0, 3, 0, 5), (3, 4, 5, 2), (7, 2, 7, 0), (9, 1, 7, 4)]


@pytest.mark.parametrize("left,right", [(-1, -1), (-1, 0), (1, 0), (2, 1)])
def test_attention_gradient(left, right):
    q, k, v, dout = (R.normal(size=s) for s in ((10, 4, 6), (11, 2, 6), (11, 2, 6), (10, 4, 6)))
    f = lambda *t: (O.attention(*t, SEQS, 0.4, left, right)[0] * dout).sum()   # noqa: E731
    o, lse, _ = O.attention(q, k, v, SEQS, 0.4, left, right)
    (dq, dk, dv), _, _ = O.attention_bwd(q, k, v, o, dout, SEQS, 0.4, left, right)
    for n, (x, g) in enumerate(((q, dq), (k, dk), (v, dv))):
        d = R.normal(size=x.shape)
        args = [q, k, v]
        assert abs(difference(lambda t: f(*args[:n], t, *args[n + 1:]), x, d) - (g * d).sum()) < 1e-7
    assert np.all(o[7:9] == 0) and np.all(lse[:, 7:9] == -np.inf)


def test_attention_of_equal_keys_is_a_mean():
    q, k, v = R.normal(size=(3, 1, 4)), np.ones((5, 1, 4)), R.normal(size=(5, 1, 4))
    o, lse, _ = O.attention(q, k, v, [(0, 3, 0, 5)], 0.5, -1, 0)
    for i in range(3):
        assert np.allclose(o[i, 0], v[:3 + i, 0].mean(axis=0)) and np.isclose(lse[0, i], np.log(3 + i) + 0.5 * q[i, 0].sum())


def test_window_positions():
    assert O.sees(2, 4, 1, 0).tolist() == [[False, True, True, False], [False, False, True, True]]
    assert O.sees(3, 1, -1, 0).tolist() == [[False], [False], [True]]
    assert O.sees(2, 2, 0, 1).tolist() == [[True, True], [False, True]]
