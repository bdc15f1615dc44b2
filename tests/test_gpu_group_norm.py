"""GPU parity of group normalisation with an activation against oracle/train_ops.py, through the C ABI.

Tolerances, from the arithmetic: statistics and the normalisation are fp32, sums are trees or chains of partial means, so an output's
error is a few 2^-24 of the largest value that enters it: x's offset over its spread (mean), or 1.  2e-6 of that, plus half a unit of
bf16 (2^-9, doubled for the neighbour that fp32 may tip it into) where the output is bf16.  Sums over samples and pixels (dgamma,
dbeta) are measured against the sum of magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def env():
    from paper_2112_10065_amd import binding as dp, synth
    from oracle import train_ops
    import gpu_util as U
    assert torch.cuda.is_available()
    return dp, U, train_ops, synth


# n, h, w, c, groups: whole vectors and not, groups inside, across and wider than a vector, one element per group, slabs
# of channels, one pixel, pixels that no block divides, long images, many samples
SHAPES = [(1, 1, 1, 8, 1), (1, 1, 1, 32, 32), (2, 1, 3, 16, 4), (1, 14, 14, 512, 32), (2, 7, 9, 64, 32), (3, 5, 4, 80, 8), (2, 6, 6, 12, 3),
          (2, 33, 31, 24, 24), (1, 9, 9, 7, 7), (2, 5, 5, 15, 5), (1, 3, 3, 2048, 32), (2, 2, 2, 4096, 1), (1, 4, 4, 5000, 8), (1, 2, 2, 601, 1),
          (5, 17, 13, 48, 2), (2, 112, 111, 64, 32), (1, 300, 1, 16, 2), (40, 2, 3, 32, 8), (1, 57, 56, 256, 32), (3, 28, 28, 512, 32), (1, 61, 3, 264, 33)]


def values(synth, tag, shape, bf16, scale=1.0, offset=0.0):
    x = (synth.normal(tag, shape) * scale + offset).astype(np.float32)
    return synth.round_bf16(x) if bf16 else x


def upload(U, a, bf16):
    from paper_2112_10065_amd import synth
    return U.bf16_dev(synth.f32_to_bf16_bits(a)) if bf16 else torch.from_numpy(np.ascontiguousarray(a)).to(U.DEV)


class Case:
    def __init__(self, env, shape, act, bf16, scale=1.0, offset=0.0, affine=True):
        dp, U, O, synth = env
        self.dp, self.U, self.O = dp, U, O
        self.n, self.h, self.w, self.c, self.groups = shape
        self.act, self.bf16, self.tdt = act, bf16, torch.bfloat16 if bf16 else torch.float32
        full = shape[:4]
        tag = f"gn/{shape}/{act}/{scale}/{offset}"
        self.x = values(synth, tag, full, bf16, scale, offset)
        self.dy = values(synth, tag + "/dy", full, bf16)
        self.gamma = (1 + 0.3 * synth.normal(tag + "/g", (self.c,))).astype(np.float32) if affine else None
        self.beta = (0.3 * synth.normal(tag + "/b", (self.c,))).astype(np.float32) if affine else None
        flags = {"none": 0, "relu": dp.DP_RELU, "silu": dp.DP_SILU}[act]
        self.desc = dp.group_norm_desc(self.n, self.h, self.w, self.c, self.groups, dp.DP_BF16 if bf16 else dp.DP_F32, flags, EPS)
        self.dev = {k: upload(U, v, b) if v is not None else None for k, v, b in
                    (("x", self.x, bf16), ("dy", self.dy, bf16), ("gamma", self.gamma, False), ("beta", self.beta, False))}
        self.one = lambda v: np.ones(self.c) if v is None else v.astype(np.float64)    # noqa: E731
        self.zero = lambda v: np.zeros(self.c) if v is None else v.astype(np.float64)  # noqa: E731

    def ws(self, pass_):
        return torch.full((self.dp.dp_group_norm_workspace_bytes(self.desc, pass_),), 0xff, dtype=torch.uint8, device=self.U.DEV)

    def forward(self, stats=True, stream=None):
        d, U = self.dev, self.U
        y = torch.full((self.n, self.h, self.w, self.c), 7.0, dtype=self.tdt, device=U.DEV)
        mean, rstd = (torch.full((self.n, self.groups), 7.0, device=U.DEV) for _ in range(2))
        self.dp.dp_group_norm_fwd(self.desc, d["x"], d["gamma"], d["beta"], y, mean if stats else None, rstd if stats else None, self.ws(0), stream)
        return y, mean, rstd

    def backward(self, y, mean, rstd, want=(True, True, True), dx=None, stream=None):
        d, U = self.dev, self.U
        dx = dx if dx is not None else torch.full((self.n, self.h, self.w, self.c), 7.0, dtype=self.tdt, device=U.DEV)
        dgamma, dbeta = (torch.full((self.c,), 7.0, device=U.DEV) for _ in range(2))
        got = [t if w else None for t, w in zip((dx, dgamma, dbeta), want)]
        self.dp.dp_group_norm_bwd(self.desc, d["x"], d["dy"], y, d["gamma"], d["beta"], mean, rstd, *got, self.ws(1), stream)
        return got

    def check_forward(self, y, mean, rstd):
        U, O = self.U, self.O
        want_y, want_mean, want_rstd = O.group_norm_fwd(self.x, self.one(self.gamma), self.zero(self.beta), self.groups, EPS, self.act)
        big = np.abs(self.x).max() + 1e-30
        assert np.abs(U.to_np(mean) - want_mean).max() <= 2e-6 * big
        # a relative error of the variance, with what the mean's error adds
        assert np.abs(U.to_np(rstd) / want_rstd - 1).max() <= 2e-6 * max(1.0, (big * want_rstd.max()))
        lim = 2e-6 * np.repeat(want_rstd, self.c // self.groups, axis=1)[:, None, None, :] * big * np.abs(self.one(self.gamma)) * 4 + 2e-6
        lim = lim + (2.0 ** -8 * np.abs(want_y) if self.bf16 else 0.0)
        assert np.all(np.abs(U.to_np(y) - want_y) <= lim)

    def check_backward(self, got, y, mean, rstd):
        U, O = self.U, self.O
        y_saved = U.to_np(y) if y is not None else None
        m, r = U.to_np(mean), U.to_np(rstd)
        dx, dgamma, dbeta = O.group_norm_bwd(self.x, self.dy, self.one(self.gamma), self.zero(self.beta), m, r, self.groups, self.act, y_saved)
        xhat = O._xhat(self.x, m.astype(np.float64), r.astype(np.float64), self.groups)
        off = np.abs(m * r).max()          # x's offset in units of its spread: what x - mean loses
        big = max(1.0, np.abs(xhat).max()) ** 2 * np.abs(self.dy).max() * np.abs(self.one(self.gamma)).max() * r.max()
        if got[0] is not None:
            lim = 2e-6 * (1 + off) * 4 * big + (2.0 ** -8 * np.abs(dx) if self.bf16 else 0.0)
            assert np.all(np.abs(U.to_np(got[0]) - dx) <= lim)
        mass = np.abs(self.dy).astype(np.float64)
        for g, want, m_ in ((got[1], dgamma, (mass * (1 + np.abs(xhat))).sum(axis=(0, 1, 2))), (got[2], dbeta, mass.sum(axis=(0, 1, 2)))):
            if g is not None:
                assert np.all(np.abs(U.to_np(g) - want) <= 4e-6 * (1 + off) * m_)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_group_norm(env, shape, act, bf16):
    k = Case(env, shape, act, bf16, scale=1.5, offset=0.5)
    y, mean, rstd = k.forward()
    k.check_forward(y, mean, rstd)
    got = k.backward(y, mean, rstd)
    torch.cuda.synchronize()
    k.check_backward(got, y if act == "relu" else None, mean, rstd)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("scale,offset", [(1.0, 1000.0), (1e-3, 1.0), (1e4, 0.0), (1e-6, 0.0), (0.0, 3.0)])
def test_offsets_and_scales(env, scale, offset, bf16):
    """A large offset costs x - mean its last bits and the variance nothing more; a constant image has variance 0."""
    k = Case(env, (2, 40, 37, 32, 8), "silu", bf16, scale, offset)
    y, mean, rstd = k.forward()
    k.check_forward(y, mean, rstd)
    k.check_backward(k.backward(y, mean, rstd), None, mean, rstd)


def test_relu_gradient_that_is_masked_already(env):
    k = Case(env, (2, 9, 9, 32, 4), "relu", True)
    y, mean, rstd = k.forward()
    k.check_backward(k.backward(None, mean, rstd), None, mean, rstd)


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True)])
def test_outputs_are_optional(env, want):
    k = Case(env, (2, 9, 11, 48, 3), "silu", True)
    y, mean, rstd = k.forward()
    assert torch.equal(k.forward(stats=False)[0], y)
    whole, some = k.backward(y, mean, rstd), k.backward(y, mean, rstd, want)
    for a, b, w in zip(whole, some, want):
        assert (b is None) == (not w) and (not w or torch.equal(a, b))


def test_without_gamma_and_beta(env):
    k = Case(env, (2, 9, 11, 48, 3), "relu", True, affine=False)
    y, mean, rstd = k.forward()
    k.check_forward(y, mean, rstd)
    k.check_backward(k.backward(y, mean, rstd), y, mean, rstd)


def test_gradient_in_place_of_dy(env):
    for shape in ((1, 14, 14, 512, 32), (2, 50, 50, 64, 32)):
        k = Case(env, shape, "silu", True)
        y, mean, rstd = k.forward()
        want = k.backward(y, mean, rstd)
        got = k.backward(y, mean, rstd, dx=k.dev["dy"])
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_values_that_are_not_finite_stay_in_their_group(env, bf16):
    dp, U, O, synth = env
    for shape in ((2, 9, 9, 32, 4), (1, 30, 30, 24, 3)):
        k = Case(env, shape, "relu", bf16)
        clean = [t.clone() for t in k.forward()]
        for bad in (float("nan"), float("inf")):
            k.dev["x"] = upload(U, k.x, bf16)
            k.dev["x"][0, 3, 2, 9] = bad
            y, mean, rstd = k.forward()
            cg = shape[3] // shape[4]
            g = 9 // cg
            hit = torch.zeros_like(y, dtype=torch.bool)
            hit[0, :, :, g * cg:(g + 1) * cg] = True
            assert torch.equal(y[~hit], clean[0][~hit]) and bool(torch.isnan(y[0, 3, 2, 9]))
            assert bool(torch.isnan(rstd[0, g])) and not bool(torch.isfinite(mean[0, g]))


def test_results_repeat_and_streams(env):
    """Bitwise the same every time, on another stream, and while other work runs."""
    k = Case(env, (4, 56, 56, 64, 32), "silu", True)
    first = [t.clone() for t in k.forward()]
    back = [t.clone() for t in k.backward(*first)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            got = k.forward(stream=side)
            grad = k.backward(*got, stream=side)
        busy = torch.randn(2048, 2048, device="cuda") @ torch.randn(2048, 2048, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first + back, list(got) + list(grad)))
        del busy


def test_in_a_graph(env):
    """Captured once, replayed on new inputs between eager work: the eager results every time."""
    dp, U, O, synth = env
    k = Case(env, (2, 28, 28, 128, 32), "silu", True)
    d, shape = k.dev, (2, 28, 28, 128)
    y, dx = (torch.empty(shape, dtype=k.tdt, device=U.DEV) for _ in range(2))
    mean, rstd = (torch.empty((2, 32), device=U.DEV) for _ in range(2))
    dgamma, dbeta = (torch.empty(128, device=U.DEV) for _ in range(2))
    ws = [k.ws(0), k.ws(1)]

    def both():
        dp.dp_group_norm_fwd(k.desc, d["x"], d["gamma"], d["beta"], y, mean, rstd, ws[0])
        dp.dp_group_norm_bwd(k.desc, d["x"], d["dy"], None, d["gamma"], d["beta"], mean, rstd, dx, dgamma, dbeta, ws[1])

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    outs = (y, mean, rstd, dx, dgamma, dbeta)
    for i in range(4):
        d["x"].copy_(torch.randn(shape, device=U.DEV, generator=torch.Generator(U.DEV).manual_seed(i)))
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_full_size(env):
    """The first layers' activation at per-GPU batch 32: two samples against the oracle, all of them by what the norm makes of them."""
    dp, U, O, synth = env
    n, h, w, c, groups = 32, 224, 224, 64, 32
    gen = torch.Generator(U.DEV).manual_seed(3)
    x = (torch.randn((n, h, w, c), device=U.DEV, generator=gen) * 1.5 + 0.5).to(torch.bfloat16)
    dy = torch.randn((n, h, w, c), device=U.DEV, generator=gen).to(torch.bfloat16)
    gamma, beta = (1 + 0.3 * torch.randn(c, device=U.DEV, generator=gen)), 0.3 * torch.randn(c, device=U.DEV, generator=gen)
    desc = dp.group_norm_desc(n, h, w, c, groups, dp.DP_BF16, dp.DP_SILU, EPS)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty((n, groups), device=U.DEV) for _ in range(2))
    dgamma, dbeta = (torch.empty(c, device=U.DEV) for _ in range(2))
    ws = U.workspace(max(dp.dp_group_norm_workspace_bytes(desc, p) for p in (0, 1)))
    dp.dp_group_norm_fwd(desc, x, gamma, beta, y, mean, rstd, ws)
    dp.dp_group_norm_bwd(desc, x, dy, None, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    g64, b64 = (t.cpu().numpy().astype(np.float64) for t in (gamma, beta))
    for i in (0, 31):
        xi, dyi = U.to_np(x[i:i + 1]), U.to_np(dy[i:i + 1])
        wy, wm, wr = O.group_norm_fwd(xi, g64, b64, groups, EPS, "silu")
        wdx, _, _ = O.group_norm_bwd(xi, dyi, g64, b64, wm, wr, groups, "silu")
        assert np.abs(U.to_np(mean[i:i + 1]) - wm).max() <= 2e-6 * 10 and np.abs(U.to_np(rstd[i:i + 1]) / wr - 1).max() <= 2e-6 * 10
        assert np.all(np.abs(U.to_np(y[i:i + 1]) - wy) <= 2.0 ** -8 * np.abs(wy) + 1e-4)
        assert np.all(np.abs(U.to_np(dx[i:i + 1]) - wdx) <= 2.0 ** -8 * np.abs(wdx) + 1e-4)
    # sums over 1.6 million pixels, in 64 bits on the device
    xh = (x.double().view(n, h * w, groups, 2) - mean.double()[:, None, :, None]) * rstd.double()[:, None, :, None]
    u = xh.view(n, h, w, c) * gamma.double() + beta.double()
    s = torch.sigmoid(u)
    g = dy.double() * (s + u * s * (1 - s))
    assert bool(((dbeta - g.sum(dim=(0, 1, 2))).abs() <= 4e-6 * g.abs().sum(dim=(0, 1, 2))).all())
    gx = g * xh.view(n, h, w, c)
    assert bool(((dgamma - gx.sum(dim=(0, 1, 2))).abs() <= 4e-6 * (g.abs() + gx.abs()).sum(dim=(0, 1, 2))).all())


def test_very_many_samples(env):
    """4 million samples of one pixel: more groups than a grid has teams, offsets beyond 2^31 bytes; some samples against the oracle."""
    dp, U, O, synth = env
    n, c, groups = 1 << 22, 256, 32
    gen = torch.Generator(U.DEV).manual_seed(4)
    x = torch.randn((n, 1, 1, c), device=U.DEV, generator=gen, dtype=torch.bfloat16)
    y = torch.empty_like(x)
    desc = dp.group_norm_desc(n, 1, 1, c, groups, dp.DP_BF16, 0, EPS)
    ws = U.workspace(dp.dp_group_norm_workspace_bytes(desc, 0))
    mean, rstd = (torch.empty((n, groups), device=U.DEV) for _ in range(2))
    dp.dp_group_norm_fwd(desc, x, None, None, y, mean, rstd, ws)
    pick = torch.tensor([0, 1, 12345, (1 << 21) + 7, n - 2, n - 1], device=U.DEV)
    want, wm, wr = O.group_norm_fwd(U.to_np(x[pick]), np.ones(c), np.zeros(c), groups, EPS)
    assert np.abs(U.to_np(mean[pick]) - wm).max() <= 1e-5 and np.abs(U.to_np(rstd[pick]) / wr - 1).max() <= 1e-5
    assert np.all(np.abs(U.to_np(y[pick]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("shape", [(1, 16, 16, 128, 16), (1, 16, 17, 128, 16), (40, 8, 8, 256, 32), (40, 8, 9, 256, 32), (2, 46, 45, 16, 2), (2, 64, 64, 16, 2),
                                   (2, 64, 65, 16, 2), (1, 3, 5, 1024, 2), (1, 2, 2, 2048, 2), (1, 11, 3, 1024, 4), (33, 45, 46, 256, 32), (2, 7, 7, 32, 8),
                                   (3, 23, 9, 48, 24), (130, 4, 4, 64, 8)], ids=lambda s: "x".join(map(str, s)))
def test_at_the_edges_of_the_forms(env, shape, act, bf16):
    """Images that just fit a wavefront's or a team's registers, and just do not; groups of a fraction of a vector up to 64 vectors."""
    k = Case(env, shape, act, bf16, scale=1.5, offset=0.5)
    y, mean, rstd = k.forward()
    k.check_forward(y, mean, rstd)
    got = k.backward(y, mean, rstd)
    torch.cuda.synchronize()
    k.check_backward(got, y if act == "relu" else None, mean, rstd)


# groups that are no power of two of whole vectors: 24, 40, 504 channels (bf16: whole vectors), 12, 20, 28 (two to a column), 6, 10, 14 (four), 5, 7, 3
# (fp32: four, bf16: eight); images of one pixel, below one row of lanes, at the limits of four, eight and sixteen wavefronts and just past them
COLUMNS = [(1, 1, 1, 48, 4), (1, 1, 1, 72, 12), (3, 2, 2, 80, 8), (2, 20, 34, 96, 8), (2, 20, 35, 96, 8), (1, 34, 40, 48, 8), (1, 37, 37, 48, 8), (2, 44, 46, 72, 3),
           (17, 52, 52, 48, 2), (1, 52, 52, 48, 2), (1, 5, 6, 1008, 2), (1, 16, 16, 1008, 2), (9, 7, 7, 640, 32), (5, 9, 9, 160, 16), (40, 6, 6, 160, 8), (4, 11, 12, 112, 8),
           (2, 13, 9, 56, 2), (3, 13, 11, 40, 8), (2, 13, 11, 56, 8), (2, 13, 11, 24, 8), (70, 3, 5, 320, 32), (1, 31, 33, 320, 32)]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", COLUMNS, ids=["x".join(map(str, s)) for s in COLUMNS])
def test_groups_of_any_width(env, shape, act, bf16):
    k = Case(env, shape, act, bf16, scale=1.5, offset=0.5, affine=shape[1] != 13)
    y, mean, rstd = k.forward()
    k.check_forward(y, mean, rstd)
    got = k.backward(y, mean, rstd)
    torch.cuda.synchronize()
    k.check_backward(got, y if act == "relu" else None, mean, rstd)
    assert torch.equal(k.forward(stats=False)[0], y)
    for want in ((True, False, False), (False, True, False), (False, True, True)):
        some = k.backward(y, mean, rstd, want)
        assert all(not w or torch.equal(a, b) for a, b, w in zip(got, some, want))
    placed = k.backward(y, mean, rstd, dx=k.dev["dy"])
    assert all(torch.equal(a, b) for a, b in zip(got, placed))


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("per", [3, 6, 10, 12, 24])
def test_a_group_keeps_its_infinities(env, per, bf16):
    """Groups that share vectors: a value that is not finite, in x or in dy, changes its own group and no other."""
    dp, U, O, synth = env
    k = Case(env, (2, 9, 9, per * 8, 8), "silu", bf16)
    y, mean, rstd = k.forward()
    dx, dgamma, dbeta = k.backward(y, mean, rstd)
    for g in (0, 1, 2, 7):
        own = slice(g * per, (g + 1) * per)
        hit = torch.zeros_like(y, dtype=torch.bool)
        hit[1, :, :, own] = True
        for bad in (float("nan"), float("-inf")):
            k.dev["x"] = upload(U, k.x, bf16)
            k.dev["x"][1, 4, 5, own.stop - 1] = bad
            got = k.forward()
            assert torch.equal(got[0][~hit], y[~hit]) and bool(torch.isnan(got[2][1, g])) and bool(torch.isnan(got[0][1, 4, 5, own.stop - 1]))
            k.dev["x"] = upload(U, k.x, bf16)
            k.dev["dy"] = upload(U, k.dy, bf16)
            k.dev["dy"][1, 4, 5, own.start] = bad
            got = k.backward(y, mean, rstd)
            assert torch.equal(got[0][~hit], dx[~hit]) and not bool(torch.isfinite(got[0][1, 0, 0, own]).any())
            others = torch.ones(per * 8, dtype=torch.bool)
            others[own.start] = False
            assert torch.equal(got[1][others], dgamma[others]) and torch.equal(got[2][others], dbeta[others])
            k.dev["dy"] = upload(U, k.dy, bf16)


@pytest.mark.parametrize("shape", [(2, 13, 17, 3, 3), (1, 5, 9, 15, 5), (3, 40, 41, 7, 7), (1, 31, 37, 33, 11)])
def test_an_outlier_in_front(env, shape):
    """The first value ten spreads away: the sums of squares are still about a value near the mean, and their difference loses a few roundings only."""
    dp, U, O, synth = env
    k = Case(env, shape, "none", False)
    k.x[:, 0, 0, :] = 10.0
    k.dev["x"] = upload(U, k.x, False)
    y, mean, rstd = k.forward()
    want = O.group_norm_fwd(k.x, k.one(k.gamma), k.zero(k.beta), k.groups, EPS, "none")
    # eight pixels' mean is 1.3 spreads off at most: (1 + 1.3^2) times the rounding of sums of a few hundred terms (1e-6), half of it in the root
    assert np.abs(U.to_np(rstd) / want[2] - 1).max() <= 1.5e-6
    k.check_forward(y, mean, rstd)


def sums_of_one(x, dy, mean, rstd, groups, chunk=4096):
    """dgamma, dbeta and their magnitudes without activation, in 64 bits on the device."""
    n, h, w, c = x.shape
    out = [torch.zeros(c, dtype=torch.float64, device=x.device) for _ in range(4)]
    for i in range(0, n, chunk):
        g = dy[i:i + chunk].double()
        xh = ((x[i:i + chunk].double().view(-1, h * w, groups, c // groups) - mean[i:i + chunk].double()[:, None, :, None]) * rstd[i:i + chunk].double()[:, None, :, None]).view(g.shape)
        for o, v in zip(out, (g * xh, g, g.abs() * (1 + xh.abs()), g.abs())):
            o += v.sum(dim=(0, 1, 2))
    return out


def check_sums(env, n, h, w, c, groups, bf16=False):
    """A gradient of one sign, whose sums' roundings all go one way: 4e-6 of the mass, as elsewhere."""
    dp, U, _, _ = env
    gen = torch.Generator(U.DEV).manual_seed(n + h)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn((n, h, w, c), device=U.DEV, generator=gen).to(dt)
    dy = torch.full((n, h, w, c), 0.1, device=U.DEV).to(dt)
    desc = dp.group_norm_desc(n, h, w, c, groups, dp.DP_BF16 if bf16 else dp.DP_F32, 0, EPS)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty((n, groups), device=U.DEV) for _ in range(2))
    dgamma, dbeta = (torch.full((c,), 7.0, device=U.DEV) for _ in range(2))
    ws = torch.full((max(dp.dp_group_norm_workspace_bytes(desc, p) for p in (0, 1)) + 16,), 0xff, dtype=torch.uint8, device=U.DEV)
    dp.dp_group_norm_fwd(desc, x, None, None, y, mean, rstd, ws)
    ws.fill_(0xff)
    dp.dp_group_norm_bwd(desc, x, dy, None, None, None, mean, rstd, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    wg, wb, mg, mb = sums_of_one(x, dy, mean, rstd, groups, max(1, (1 << 25) // (h * w * c)))
    assert bool(((dgamma - wg).abs() <= 4e-6 * mg).all()) and bool(((dbeta - wb).abs() <= 4e-6 * mb).all())
    again = [torch.full((c,), 7.0, device=U.DEV) for _ in range(2)]
    ws.fill_(0xff)
    dp.dp_group_norm_bwd(desc, x, dy, None, None, None, mean, rstd, None, *again, ws)
    assert torch.equal(again[0], dgamma) and torch.equal(again[1], dbeta)
    return x, dy, y, dx, mean, rstd


@pytest.mark.parametrize("n,h,w,c,groups", [(65536, 1, 1, 32, 4), (1 << 20, 1, 1, 32, 4), (3001, 5, 3, 24, 2), (40000, 2, 1, 5, 5), (2100, 40, 40, 6, 1), (4099, 3, 3, 40, 4)])
def test_parameter_gradients_of_very_many_samples(env, n, h, w, c, groups):
    check_sums(env, n, h, w, c, groups)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape,where", [((1, 8, 8, 768, 1), "channel"), ((2, 8, 8, 2048, 1), "channel"), ((1, 3, 5, 5000, 1), "channel"), ((1, 8, 8, 4096, 2), "slab"),
                                         ((1, 256, 256, 16, 1), "front"), ((2, 300, 200, 8, 1), "front"), ((1, 128, 128, 8, 1), "pixel"), ((3, 130, 127, 3, 1), "pixel")])
def test_outliers_that_lead(env, shape, where, bf16):
    """The first channel of a wide group, the first channels of a group in parts, the first pixels of a long image or its first one lie a
    hundred or more spreads away from the rest: every sum of squares is taken about a mean, so rstd is off by the roundings of sums of a few hundred terms,
    not by these times the number of channels or pixels behind the outlier."""
    dp, U, O, synth = env
    k = Case(env, shape, "none", bf16)
    if where == "channel":
        k.x[..., 0] += 100
    elif where == "slab":
        k.x[..., :64] += 100
    elif where == "front":
        k.x.reshape(shape[0], -1, shape[3])[:, :128] += 100
    else:
        k.x[:, 0, 0] += 2000
    k.x = synth.round_bf16(k.x) if bf16 else k.x
    k.dev["x"] = upload(U, k.x, bf16)
    y, mean, rstd = k.forward()
    want = O.group_norm_fwd(k.x, k.one(k.gamma), k.zero(k.beta), k.groups, EPS, "none")
    assert np.abs(U.to_np(rstd) / want[2] - 1).max() <= 1e-6
    k.check_forward(y, mean, rstd)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,h,w,c,groups", [(1, 128, 128, 512, 512), (1, 112, 112, 256, 256), (2, 131, 127, 300, 300), (1, 224, 224, 1024, 512), (1, 96, 97, 250, 250),
                                            (1, 200, 200, 96, 32), (1, 100, 100, 1536, 256)])
def test_many_narrow_groups(env, n, h, w, c, groups, bf16):
    """Norms of a channel or two, images too large for one kernel: statistics and gradients, sums of a gradient of one sign among them."""
    U = env[1]
    x, dy, y, dx, mean, rstd = check_sums(env, n, h, w, c, groups, bf16)
    xd, cg = x.double().view(n, h * w, groups, c // groups), c // groups
    wm = xd.mean(dim=(1, 3), keepdim=True)
    wr = 1 / torch.sqrt((xd - wm).square().mean(dim=(1, 3), keepdim=True) + EPS)
    assert float((mean - wm.view(n, groups)).abs().max()) <= 2e-6 * float(x.abs().max()) and float((rstd / wr.view(n, groups) - 1).abs().max()) <= 2e-6
    xh, t = (xd - wm) * wr, dy.double().view(xd.shape)
    big = float(x.abs().max())
    assert bool(((y.double() - xh.view(x.shape)).abs() <= 8e-6 * big + (2.0 ** -8 * xh.view(x.shape).abs() if bf16 else 0)).all())
    want = ((t - t.mean(dim=(1, 3), keepdim=True) - xh * (t * xh).mean(dim=(1, 3), keepdim=True)) * wr).view(x.shape)
    lim = 8e-6 * max(1.0, float(xh.abs().max())) ** 2 * 0.1 * float(wr.max())
    assert bool(((dx.double() - want).abs() <= lim + (2.0 ** -8 * want.abs() if bf16 else 0)).all())


@pytest.mark.parametrize("n,h,w,c,groups", [(1030, 512, 512, 4, 1), (600, 300, 300, 8, 2), (1, 2048, 2048, 32, 32)])
def test_parameter_gradients_of_many_large_images(env, n, h, w, c, groups):
    """Thousands of pixels to a thread."""
    check_sums(env, n, h, w, c, groups)


def test_silu_to_the_last_bits(env):
    """u in single channels by beta alone (gamma 0), from -80 to 80: u * sigmoid(u) and its derivative to a few roundings of fp32 (2^-24 each: two of the
    exponential, the sum, two of the reciprocal, three products), relative to the value and to the derivative's two terms."""
    dp, U, _, _ = env
    for shape, groups in (((1, 1, 1, 4096), 8), ((1, 1, 1, 4100), 1), ((1, 1, 1, 4099), 1)):
        c = shape[3]
        beta = np.linspace(-80, 80, c).astype(np.float32)
        desc = dp.group_norm_desc(*shape, groups, dp.DP_F32, dp.DP_SILU, EPS)
        x = torch.randn(shape, device=U.DEV, generator=torch.Generator(U.DEV).manual_seed(1))
        gamma, bd, dy = torch.zeros(c, device=U.DEV), torch.from_numpy(beta).to(U.DEV), torch.ones(shape, device=U.DEV)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = (torch.empty((1, groups), device=U.DEV) for _ in range(2))
        dgamma, dbeta = (torch.empty(c, device=U.DEV) for _ in range(2))
        ws = U.workspace(max(dp.dp_group_norm_workspace_bytes(desc, p) for p in (0, 1)))
        dp.dp_group_norm_fwd(desc, x, gamma, bd, y, mean, rstd, ws)
        dp.dp_group_norm_bwd(desc, x, dy, None, gamma, bd, mean, rstd, dx, dgamma, dbeta, ws)
        u = beta.astype(np.float64)
        q, not_q = 1 / (1 + np.exp(-u)), 1 / (1 + np.exp(u))
        assert np.all(np.abs(U.to_np(y).reshape(-1) - u * q) <= 6e-7 * np.abs(u * q))
        assert np.all(np.abs(U.to_np(dbeta) - q * (1 + u * not_q)) <= 8e-7 * q * (1 + np.abs(u) * (not_q + 1.2e-7 / 8e-7)))
