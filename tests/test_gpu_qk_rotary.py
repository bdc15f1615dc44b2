"""GPU parity of the head norm with rotary positions, forward and backward, against oracle/attention_ops.py, through the C ABI.

Tolerances, from the arithmetic: a result is the sum of two products, each with rstd (a sum of `dim` squares, all positive, and a root: dim / 8 + 8 roundings of
2^-24 with the sums of eight and over lanes), a cosine or sine that is 1e-7 off, and four more roundings; then half a step of the type.  dgamma adds up rows x heads
such terms in fp32, no chain longer than 200 of them, in 64 bits behind that."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def env():
    from paper_2112_10065_amd import binding as dp
    from oracle import attention_ops
    assert torch.cuda.is_available()
    return dp, attention_ops


class Case:
    """Queries and keys inside wider rows (`gap` elements around them), results too."""

    def __init__(self, env, rows, heads, kv_heads, dim, pairs, halves, norm, bf16, gap=8, gamma=True, far=1000, device="cuda"):
        self.dp, self.O = env
        r = np.random.default_rng([rows, heads, dim, halves])
        self.rows, self.heads, self.dim, self.pairs, self.halves, self.norm, self.bf16, self.gap, self.device = rows, (heads, kv_heads), dim, pairs, halves, norm, bf16, gap, device
        self.tdt = torch.bfloat16 if bf16 else torch.float32
        self.widths = [h * dim for h in self.heads]
        self.x, self.dy = ([self.up(r.normal(size=(rows, h, dim)) * r.uniform(0.3, 3, size=dim)) for h in self.heads] for _ in range(2))
        self.gamma = [r.uniform(0.5, 1.5, size=dim).astype(np.float32) if gamma and norm else None for _ in range(2)]
        self.pos = np.floor(r.uniform(0, far, size=(rows, len(pairs)))).astype(np.float32)
        self.freq = 10000.0 ** -r.uniform(0, 1, size=sum(pairs))
        dev = lambda a: None if a is None else torch.from_numpy(a).to(device)   # noqa: E731
        self.gd, self.pd, self.fd = [dev(g) for g in self.gamma], dev(self.pos), dev(self.freq)
        flags = (dp_flag(self.dp, "DP_QK_NORM") if norm else 0) | (dp_flag(self.dp, "DP_ROTARY_HALVES") if halves else 0)
        s = [w + 2 * gap for w in self.widths]
        self.desc = self.dp.qk_rotary_desc(rows, heads, kv_heads, dim, pairs, self.dp.DP_BF16 if bf16 else self.dp.DP_F32, flags, EPS, *s, *s, *s)

    def up(self, a):
        return torch.from_numpy(a.astype(np.float32)).to(self.device).to(self.tdt)

    def wide(self, parts):
        """[rows, gap + heads + gap] with 55 in the gaps, and the addresses of the heads."""
        rooms = [torch.full((self.rows, w + 2 * self.gap), 55.0, dtype=self.tdt, device=self.device) for w in self.widths]
        if parts is not None:
            for room, p, w in zip(rooms, parts, self.widths):
                room[:, self.gap:self.gap + w] = p.reshape(self.rows, w)
        return rooms

    def inner(self, room, side):
        return room[:, self.gap:self.gap + self.widths[side]]

    def at(self, rooms):
        return [self.inner(r, i) for i, r in enumerate(rooms)]

    def check_gaps(self, rooms):
        for i, r in enumerate(rooms):
            assert torch.all(r[:, :self.gap] == 55) and torch.all(r[:, self.gap + self.widths[i]:] == 55)

    def forward(self, in_place=False, stream=None):
        x = self.wide(self.x)
        y = x if in_place else self.wide(None)
        self.dp.dp_qk_rotary_fwd(self.desc, *self.at(x), *self.gd, self.pd, self.fd, *self.at(y), stream)
        return y

    def rel(self):
        return (self.dim / 8 + 16) * 2.0 ** -24 + 2e-7

    def half_step(self):
        return 2.0 ** -8 if self.bf16 else 2.0 ** -24

    def turned_size(self, u):
        """Of each channel, the sum of the magnitudes of its pair."""
        a, b = self.O._pairs(self.dim, self.pairs, self.halves)
        s = np.abs(u)
        out = s.copy()
        out[:, :, a] = out[:, :, b] = s[:, :, a] + s[:, :, b]
        return out

    def args(self, side):
        return self.gamma[side], self.pos, self.freq, self.pairs, self.halves, self.norm, EPS

    def check_forward(self, y):
        self.check_gaps(y)
        for side in range(2):
            x = self.x[side].double().cpu().numpy()
            want = self.O.qk_rotary(x, *self.args(side))
            u = self.O.rotate(want, self.pos, self.freq, self.pairs, self.halves, back=True)
            got = self.inner(y[side], side).double().cpu().numpy().reshape(want.shape)
            tol = self.rel() * self.turned_size(u) + self.half_step() * np.abs(want) + 1e-37
            assert np.all(np.abs(got - want) <= tol), (side, np.abs(got - want).max())

    def backward(self, in_place=False, stream=None, want_gamma=True):
        x, dy = self.wide(self.x), self.wide(self.dy)
        dx = dy if in_place else self.wide(None)
        dgamma = [torch.full((self.dim,), 7.0, device=self.device) if self.norm and want_gamma else None for _ in range(2)]
        nbytes = self.dp.dp_qk_rotary_workspace_bytes(self.desc, self.dp.DP_PASS_DGRAD)
        ws = torch.full((nbytes + 16,), 0xff, dtype=torch.uint8, device=self.device)
        self.dp.dp_qk_rotary_bwd(self.desc, *self.at(x), *self.gd, self.pd, self.fd, *self.at(dy), *self.at(dx), *dgamma, ws, stream)
        return dx, dgamma

    def check_backward(self, dx, dgamma):
        self.check_gaps(dx)
        for side in range(2):
            x, dy = (t[side].double().cpu().numpy() for t in (self.x, self.dy))
            want, want_g = self.O.qk_rotary_bwd(x, *self.args(side), dy)
            got = self.inner(dx[side], side).double().cpu().numpy().reshape(want.shape)
            g = self.turned_size(dy)
            size = g
            if self.norm and x.size:
                r = 1 / np.sqrt((x * x).mean(axis=2, keepdims=True) + EPS)
                t = g * np.abs(1.0 if self.gamma[side] is None else self.gamma[side].astype(np.float64))
                size = r * (t + np.abs(x) * r * r * (t * np.abs(x)).mean(axis=2, keepdims=True))
                if dgamma[side] is not None:
                    terms = (g * np.abs(x) * r).sum(axis=(0, 1))
                    err = np.abs(dgamma[side].double().cpu().numpy() - want_g)
                    assert np.all(err <= terms * (self.rel() + 200 * 2.0 ** -24)), (side, err.max())
            tol = 2 * self.rel() * size + self.half_step() * np.abs(want) + 1e-37
            assert np.all(np.abs(got - want) <= tol), (side, np.abs(got - want).max())


def dp_flag(dp, name):
    return getattr(dp, name)


SHAPES = [(1, 1, 1, 8, [4]), (3, 4, 2, 16, [8]), (5, 5, 1, 40, [4, 8, 8]), (17, 12, 12, 64, [16, 16]), (33, 10, 2, 72, [19]), (9, 3, 1, 72, [36]), (130, 16, 4, 128, [16, 24, 24]),
          (2, 28, 28, 80, [3, 5]), (7, 2, 2, 96, [12, 12, 16]), (4, 1, 3, 112, [1]), (6, 3, 2, 136, [60]), (3, 2, 1, 256, [128]), (2050, 2, 1, 32, [16]), (1, 40, 8, 24, [0, 12]), (11, 6, 0, 64, [32])]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
@pytest.mark.parametrize("halves", [True, False], ids=["halves", "pairs"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_parity(env, shape, halves, norm, bf16):
    c = Case(env, *shape, halves, norm, bf16)
    if shape[2] == 0:   # queries alone
        c.wide = lambda parts, w=c.wide: w(parts)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("halves", [True, False])
def test_in_place(env, halves):
    c = Case(env, 37, 6, 2, 64, [20, 8], halves, True, True)
    c.check_forward(c.forward(in_place=True))
    c.check_backward(*c.backward(in_place=True))
    c.check_backward(*c.backward(in_place=True, want_gamma=False))


def test_without_gamma(env):
    c = Case(env, 20, 4, 4, 48, [24], True, True, False, gamma=False)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


def test_far_and_fractional_places(env):
    c = Case(env, 64, 2, 1, 64, [32], False, False, False, far=200000)
    c.check_forward(c.forward())
    c.pos[:] = c.pos * 0.37 - 1000
    c.pd.copy_(torch.from_numpy(c.pos))
    c.check_forward(c.forward())
    c.pos[:] = c.pos * 1e7
    c.pd.copy_(torch.from_numpy(c.pos))
    y = c.forward()   # angles of 1e11: 64 bits leave 2e-5 of a turn
    want = c.O.qk_rotary(c.x[0].double().cpu().numpy(), *c.args(0))
    got = c.inner(y[0], 0).double().cpu().numpy().reshape(want.shape)
    assert np.abs(got - want).max() <= 2e12 * 2.0 ** -52 * np.abs(want).max() * 4 + 1e-5


def test_no_rows(env):
    dp, _ = env
    d = dp.qk_rotary_desc(0, 2, 1, 32, [16], flags=dp.DP_QK_NORM)
    dgamma = [torch.full((32,), 7.0, device="cuda") for _ in range(2)]
    dp.dp_qk_rotary_bwd(d, None, None, None, None, None, None, None, None, None, None, *dgamma)
    assert all(torch.all(g == 0) for g in dgamma)


def test_a_row_that_is_not_finite_stays_one(env):
    c = Case(env, 12, 4, 2, 64, [32], True, True, True)
    c.x[0][5, 1, 3] = float("nan")
    c.x[1][7, 0, 0] = float("inf")
    y = c.forward()
    for side, row, head in ((0, 5, 1), (1, 7, 0)):
        t = c.inner(y[side], side).reshape(12, -1, 64).isfinite()
        assert not t[row, head].all()
        t[row, head] = True
        assert t.all()


def test_same_bits_on_another_stream_and_in_a_graph(env):
    c = Case(env, 700, 9, 3, 72, [10, 26], True, True, True)
    y, (dx, dg) = c.forward(), c.backward()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, (dx2, dg2) = c.forward(), c.backward()
    torch.cuda.synchronize()
    x, dy, out, dx3 = c.wide(c.x), c.wide(c.dy), c.wide(None), c.wide(None)
    dg3 = [torch.zeros(72, device="cuda") for _ in range(2)]
    ws = torch.full((c.dp.dp_qk_rotary_workspace_bytes(c.desc, c.dp.DP_PASS_DGRAD),), 0xff, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.dp.dp_qk_rotary_fwd(c.desc, *c.at(x), *c.gd, c.pd, c.fd, *c.at(out))
        c.dp.dp_qk_rotary_bwd(c.desc, *c.at(x), *c.gd, c.pd, c.fd, *c.at(dy), *c.at(dx3), *dg3, ws)
    for _ in range(3):
        for t in out + dx3:
            t.fill_(55.0)
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        for a, b, e in zip(y + dx + dg, y2 + dx2 + dg2, out + dx3 + dg3):
            assert torch.equal(a, b) and torch.equal(a, e)


@pytest.mark.parametrize("halves", [True, False])
def test_nothing_to_turn(env, halves):
    """The norm alone: freq has no elements, and no places need be given."""
    for pairs in ([0], [0, 0]):
        c = Case(env, 23, 5, 2, 72, pairs, halves, True, False)
        c.check_forward(c.forward())
        c.check_backward(*c.backward())
        c.pd = c.fd = None
        c.check_forward(c.forward())
