"""GPU parity of attention, forward and backward, against oracle/attention_ops.py, through the C ABI.

Tolerances, from the arithmetic.  A score is a sum of dim products in fp32: off by (dim + 4) 2^-24 of the sum of their magnitudes, `reach` at the most; p is off by twice as
much (its own and that of the sum), by the rounding of lse and the exponential's: relative, `rel`.  With bf16, p, ds and every result are rounded once more by at most 2^-8
of their value.  Sums of up to `terms` summands add terms 2^-24 of their magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
# A probability under 2^-126 = 1.2e-38, the smallest normal number, may count as 0: up to 1e4 of them times factors of up to 1e3 are missing then.
FLOOR = 1.2e-31


@pytest.fixture(scope="module")
def env():
    from paper_2112_10065_amd import binding as dp
    from oracle import attention_ops
    assert torch.cuda.is_available()
    return dp, attention_ops


class Case:
    """q_side, kv_side: None (whole sequences), lengths (padded), or ("packed", lengths, rows in front, rows behind).  Rows in no use hold NaN."""

    def __init__(self, env, n, q_len, kv_len, heads, kv_heads, dim, left=-1, right=-1, bf16=True, q_side=None, kv_side=None, scale=0.0, spread=1.5, gap=8, seed=0):
        self.dp, self.O = env
        r = np.random.default_rng([n, q_len, kv_len, heads, dim, seed])
        self.n, self.heads, self.kv_heads, self.dim, self.left, self.right, self.bf16 = n, heads, kv_heads, dim, left, right, bf16
        self.tdt = torch.bfloat16 if bf16 else torch.float32
        self.scale = scale or dim ** -0.5
        (self.q_rows, self.q_at, q_args), (self.kv_rows, self.kv_at, kv_args) = self.side(q_side, n, q_len), self.side(kv_side, n, kv_len)
        self.seqs_list = [(q0, lq, k0, lk) for (q0, lq), (k0, lk) in zip(self.q_at, self.kv_at)]
        self.seqs = self.dp.attention_seqs(**{"q_" + k: v for k, v in q_args.items()}, **{"kv_" + k: v for k, v in kv_args.items()}) if q_args or kv_args else None
        self.gap, self.widths = gap, (heads * dim, kv_heads * dim)
        self.q, self.dout = (self.make(r, self.q_rows, heads, spread, self.q_at) for _ in range(2))
        self.k = self.make(r, self.kv_rows, kv_heads, 1.0, self.kv_at)
        self.v = self.make(r, self.kv_rows, kv_heads, 1.0, self.kv_at, 0.3)
        sq, sk = self.widths[0] + gap, self.widths[1] + gap
        self.desc = self.dp.attention_desc(n, q_len, kv_len, heads, kv_heads, dim, self.dp.DP_BF16 if bf16 else self.dp.DP_F32, left, right, scale, self.q_rows, self.kv_rows, sq, sk, sk,
                                           self.widths[0])

    def side(self, spec, n, longest):
        if spec is None:
            return n * longest, [(b * longest, longest) for b in range(n)], {}
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
        if spec[0] != "packed":
            return n * longest, [(b * longest, l) for b, l in enumerate(spec)], {"lens": dev(list(spec))}
        starts = spec[2] + np.concatenate([[0], np.cumsum(spec[1])])
        return int(starts[-1]) + spec[3], [(int(s), l) for s, l in zip(starts, spec[1])], {"starts": dev(starts.tolist())}

    def make(self, r, rows, heads, spread, at, offset=0.0):
        used = np.zeros(rows, dtype=bool)
        for first, l in at:
            used[first:first + l] = True
        a = (r.normal(size=(rows, heads, self.dim)) * spread + offset * r.normal(size=self.dim)).astype(np.float32)
        a[~used] = np.nan
        return torch.from_numpy(a).to("cuda").to(self.tdt)

    def wide(self, t, fill=55.0):
        rows, w = t.shape[0], t.shape[1] * t.shape[2]
        room = torch.full((rows, w + self.gap), fill, dtype=t.dtype, device="cuda")
        room[:, :w] = t.reshape(rows, w)
        return room

    def host(self, t):
        return torch.nan_to_num(t.double(), nan=0.0).cpu().numpy()

    def own(self, at, length, rows, packed):
        """Rows that the call writes."""
        w = np.zeros(rows, dtype=bool)
        for first, l in at:
            w[first:first + (l if packed else length)] = True
        return w

    def forward(self, stream=None, lse=True):
        o = torch.full((self.q_rows, self.widths[0]), 7.0, dtype=self.tdt, device="cuda")
        lse = torch.full((self.heads, self.q_rows), 7.0, device="cuda") if lse else None
        ws = torch.full((self.dp.dp_attention_workspace_bytes(self.desc, self.dp.DP_PASS_FWD) + 16,), 0xff, dtype=torch.uint8, device="cuda")
        self.dp.dp_attention_fwd(self.desc, self.wide(self.q), self.wide(self.k), self.wide(self.v), o, lse, self.seqs, ws, stream)
        return o, lse

    def sizes(self):
        """(rel, terms): how far p may be off, relative, without its rounding; summands of the longest sum."""
        reach = big = 0.0
        q, k = np.abs(self.host(self.q)), np.abs(self.host(self.k))
        share = self.heads // self.kv_heads
        for q0, lq, k0, lk in self.seqs_list:
            if lq and lk:
                for h in range(self.heads):
                    reach = max(reach, self.scale * float((q[q0:q0 + lq, h] @ k[k0:k0 + lk, h // share].T).max()))
        big = reach + 12
        longest = max([max(l[1] * share, l[3]) for l in self.seqs_list] + [1])
        return (2 * (self.dim + 6) * reach + 4 * big + 16) * 2.0 ** -24, min(longest, 256) * 2.0 ** -24

    def half_step(self):
        return 2.0 ** -8 if self.bf16 else 2.0 ** -24

    def check_forward(self, got, q_packed=False):
        o, lse = got
        want, want_lse, size = self.O.attention(self.host(self.q), self.host(self.k), self.host(self.v), self.seqs_list, self.scale, self.left, self.right)
        own = self.own(self.q_at, self.desc.q_len, self.q_rows, q_packed)
        rel, terms = self.sizes()
        o = o.double().cpu().numpy().reshape(want.shape)
        tol = (rel + terms) * size + self.half_step() * (np.abs(want) * 1.01 + (size if self.bf16 else 0)) + FLOOR
        err = np.abs(o - want)[own]
        assert np.all(err <= tol[own]), (err.max(), (err / tol[own]).max())
        assert np.all(o[~own] == 7)
        if lse is not None:
            lse = lse.double().cpu().numpy()
            assert np.all(lse[:, ~own] == 7)
            a, b = lse[:, own], want_lse[:, own]
            fine = np.isfinite(b)
            assert np.array_equal(a[~fine], b[~fine])
            assert np.all(np.abs(a[fine] - b[fine]) <= rel + terms + 2.0 ** -22 * (1 + np.abs(b[fine])))
        return want, want_lse

    def saved(self, want, want_lse):
        return torch.from_numpy(want.reshape(self.q_rows, self.widths[0])).to("cuda").to(self.tdt), torch.from_numpy(want_lse.astype(np.float32)).to("cuda")

    def backward(self, o, lse, stream=None):
        dq, dk, dv = (torch.full((t.shape[0], t.shape[1] * t.shape[2] + self.gap), 55.0, dtype=self.tdt, device="cuda") for t in (self.q, self.k, self.v))
        ws = torch.full((self.dp.dp_attention_workspace_bytes(self.desc, self.dp.DP_PASS_DGRAD) + 16,), 0xff, dtype=torch.uint8, device="cuda")
        self.dp.dp_attention_bwd(self.desc, self.wide(self.q), self.wide(self.k), self.wide(self.v), o, self.dout.reshape(self.q_rows, self.widths[0]), lse, dq, dk, dv, self.seqs, ws, stream)
        return dq, dk, dv

    def check_backward(self, got, o, q_packed=False, kv_packed=False):
        want, rounded, added = self.O.attention_bwd(self.host(self.q), self.host(self.k), self.host(self.v), self.host(o).reshape(self.q.shape), self.host(self.dout), self.seqs_list, self.scale,
                                                    self.left, self.right)
        rel, terms = self.sizes()
        # dp - delta: two sums of dim products
        rel = rel + 2 * (self.dim + 4) * 2.0 ** -24
        for i, name in enumerate(("dq", "dk", "dv")):
            side = (self.q_at, self.desc.q_len, self.q_rows, q_packed) if i == 0 else (self.kv_at, self.desc.kv_len, self.kv_rows, kv_packed)
            own = self.own(*side)
            w = self.widths[min(i, 1)]
            g = got[i].double().cpu().numpy()
            assert np.all(g[:, w:] == 55) and np.all(g[~own] == 55), name
            tol = (rel + terms) * added[i] + self.half_step() * (np.abs(want[i]) * 1.01 + (rounded[i] * (1 + 64 * rel) if self.bf16 else 0)) + FLOOR
            if self.bf16:   # what is rounded to bf16 is off by rel already, relative to what was added up to it
                tol = tol + self.half_step() * rel * added[i]
            err = np.abs(g[:, :w].reshape(want[i].shape) - want[i])[own]
            assert np.all(err <= tol[own]), (name, err.max(), (err / tol[own]).max())

    def check(self, q_packed=False, kv_packed=False):
        want, want_lse = self.check_forward(self.forward(), q_packed)
        o, lse = self.saved(want, want_lse)
        unused = ~self.own(self.q_at, 0, self.q_rows, True)
        o[torch.from_numpy(unused).cuda()] = float("nan")      # the rows of padding are not read
        lse[:, torch.from_numpy(unused).cuda()] = float("nan")
        self.check_backward(self.backward(o, lse), o, q_packed, kv_packed)


SHAPES = [(1, 1, 1, 1, 1, 8), (2, 1, 3, 4, 2, 16), (1, 33, 65, 2, 1, 24), (3, 64, 64, 3, 3, 32), (2, 129, 127, 4, 1, 40), (1, 197, 197, 3, 3, 64), (2, 63, 200, 8, 2, 72), (1, 300, 45, 2, 2, 80),
          (1, 130, 257, 6, 2, 96), (2, 31, 513, 5, 1, 112), (1, 256, 256, 4, 2, 128), (1, 5, 1000, 16, 2, 128), (70, 40, 40, 8, 4, 64), (1, 7, 0, 2, 1, 32), (2, 0, 9, 2, 2, 48)]
MASKS = [(-1, -1), (-1, 0), (0, 0), (17, 5), (100, 0), (-1, 70), (40, -1)]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_parity(env, shape, mask, bf16):
    Case(env, *shape, *mask, bf16).check()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("mask", [(-1, -1), (-1, 0), (20, 3)], ids=str)
@pytest.mark.parametrize("dim", [40, 64, 128])
def test_padded(env, dim, mask, bf16):
    """Lengths of zero, one and all; fewer queries than keys, and more; the rows of padding hold NaN."""
    Case(env, 7, 70, 150, 4, 2, dim, *mask, bf16, q_side=[70, 1, 0, 64, 33, 70, 5], kv_side=[150, 1, 7, 0, 64, 65, 128]).check()
    Case(env, 3, 2, 150, 6, 2, dim, *mask, bf16, kv_side=[0, 150, 3]).check()
    Case(env, 3, 70, 40, 2, 2, dim, *mask, bf16, q_side=[70, 0, 3]).check()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("mask", [(-1, -1), (-1, 0), (31, 31)], ids=str)
@pytest.mark.parametrize("dim", [32, 96])
def test_packed(env, dim, mask, bf16):
    """Rows in front of the first sequence and behind the last are left as they were."""
    lq, lk = [3, 0, 130, 64, 1, 40], [3, 9, 130, 0, 200, 10]
    Case(env, 6, 130, 200, 4, 2, dim, *mask, bf16, q_side=("packed", lq, 2, 3), kv_side=("packed", lk, 1, 70)).check(True, True)
    Case(env, 6, 130, 200, 4, 1, dim, *mask, bf16, q_side=("packed", lq, 0, 0), kv_side=lk).check(True, False)
    Case(env, 6, 130, 200, 2, 2, dim, *mask, bf16, q_side=lq, kv_side=("packed", lk, 0, 5)).check(False, True)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 1, 5000, 8, 1, 128, -1, 0), (5, 1, 2000, 8, 2, 64, -1, 0), (2, 3, 3001, 32, 4, 96, -1, 0), (1, 1, 4097, 1, 1, 40, 700, 0), (1, 40, 2500, 3, 1, 128, -1, -1)], ids=str)
def test_few_queries_over_many_keys(env, case, bf16):
    """The keys are dealt out to several blocks and their results joined."""
    c = Case(env, *case[:6], *case[6:], bf16)
    assert c.dp.dp_attention_workspace_bytes(c.desc, c.dp.DP_PASS_FWD) > 0
    c.check()
    n, kv = case[0], case[2]
    Case(env, *case[:6], *case[6:], bf16, kv_side=[max(0, kv - 617 * b) if b != 1 else 0 for b in range(n)]).check_forward(
        Case(env, *case[:6], *case[6:], bf16, kv_side=[max(0, kv - 617 * b) if b != 1 else 0 for b in range(n)]).forward())


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_few_queries_padded_and_packed_over_many_keys(env, bf16):
    """Splits of the keys with queries that are not in use, or packed; every workspace begins as NaN."""
    Case(env, 4, 3, 2100, 8, 2, 64, -1, 0, bf16, q_side=[3, 0, 1, 2], kv_side=[2100, 1700, 0, 1]).check()
    Case(env, 4, 3, 2100, 8, 2, 72, -1, -1, bf16, q_side=("packed", [3, 0, 1, 2], 1, 2), kv_side=("packed", [2100, 1700, 0, 1], 0, 1)).check(True, True)
    Case(env, 4, 3, 2100, 8, 2, 128, 900, 0, bf16, q_side=("packed", [3, 0, 1, 2], 1, 2)).check(True, False)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("dim", [40, 64, 128])
def test_queries_dealt_out(env, dim, bf16):
    """Few blocks of keys with many queries: dk and dv are sums over several blocks, some of them of nothing."""
    for left, right in ((-1, -1), (-1, 0), (300, 40)):
        c = Case(env, 1, 900, 70, 6, 1, dim, left, right, bf16)
        assert c.dp.dp_attention_workspace_bytes(c.desc, c.dp.DP_PASS_DGRAD) > 2 * 4 * 6 * 900
        c.check()
    Case(env, 3, 900, 70, 6, 1, dim, -1, 0, bf16, q_side=[900, 0, 130], kv_side=("packed", [70, 5, 33], 1, 2)).check(False, True)


@pytest.mark.parametrize("dim", [48, 64, 96, 112, 128])
def test_queries_dealt_out_to_wide_blocks(env, dim):
    """Long sequences of few heads: dk and dv of 128 keys are sums over several blocks; a short sequence has fewer tiles of queries than there are blocks to share them."""
    for c, packed in ((Case(env, 1, 1500, 1500, 8, 1, dim, -1, 0), False), (Case(env, 2, 1400, 1400, 6, 2, dim, -1, 0, q_side=[1400, 900]), False),
                      (Case(env, 2, 2600, 2600, 4, 1, dim, q_side=("packed", [2600, 20], 1, 2), kv_side=("packed", [2600, 33], 0, 3)), True)):
        assert c.dp.dp_attention_workspace_bytes(c.desc, c.dp.DP_PASS_DGRAD) > 2 * (4 * c.heads * c.q_rows + 16)
        c.check(packed, packed)


@pytest.mark.parametrize("kv_heads", [1, 2, 3, 4, 6, 8])
def test_causal_tiles_dealt_to_dies(env, kv_heads):
    """Whole sequences whose tiles are numbered by how many heads there are, and whose number may be a multiple of eight or not."""
    for length in (1024, 1100):
        Case(env, 1, length, length, 2 * kv_heads, kv_heads, 64, -1, 0).check()
    Case(env, 2, 520, 700, 2 * kv_heads, kv_heads, 128, -1, 0).check()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("mask", [(-1, -1), (-1, 0), (50, 9)], ids=str)
@pytest.mark.parametrize("dim", [24, 40, 64, 72, 96, 104, 128])
def test_many_blocks(env, dim, mask, bf16):
    """Enough of them to fill the card: blocks of 128 columns, forward and backward."""
    Case(env, 33, 70, 150, 16, 8, dim, *mask, bf16).check()
    lq, lk = [(b * 37) % 71 for b in range(33)], [(b * 61) % 151 for b in range(33)]
    Case(env, 33, 70, 150, 8, 8, dim, *mask, bf16, q_side=("packed", lq, 1, 2), kv_side=lk).check(True, False)


@pytest.mark.parametrize("mask", [(-1, -1), (-1, 0), (13, 5)], ids=str)
@pytest.mark.parametrize("dim", [32, 40, 64, 80, 96, 112, 128])
def test_many_blocks_in_full_rounds(env, dim, mask):
    """fp32 takes blocks of 128 columns where they come out even, or where there are many."""
    Case(env, 64, 40, 50, 16, 16, dim, *mask, False).check()
    if dim in (64, 80):
        Case(env, 64, 131, 150, 16, 8, dim, *mask, False, q_side=[131 - b % 7 for b in range(64)], kv_side=[150 - b % 40 for b in range(64)]).check()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_large_scores_and_scale(env, bf16):
    """Scores of hundreds: the running maximum grows again and again, most probabilities vanish."""
    Case(env, 1, 150, 400, 2, 1, 64, bf16=bf16, spread=30.0).check()
    Case(env, 1, 150, 400, 2, 1, 64, -1, 0, bf16=bf16, scale=0.9, spread=0.2).check()


def test_rising_scores(env):
    """Each key beats the ones before it by more than the last bits of a bf16 sum hold."""
    c = Case(env, 1, 64, 512, 1, 1, 32, bf16=False)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    c.k[:, 0, 0] = torch.arange(512, device="cuda") * 3.0
    c.check()
    c.k[:, 0, 0] = torch.arange(512, device="cuda").flip(0) * 3.0 - 2000
    c.check()


def test_not_finite(env):
    """A NaN in a key reaches the queries that see it and no others; an infinite score makes its row NaN."""
    c = Case(env, 2, 100, 100, 2, 2, 64, -1, 0)
    c.k[30, 0, 5] = float("nan")
    o = c.forward()[0].reshape(200, 2, 64)
    assert o[:30].isfinite().all() and o[:, 1].isfinite().all() and o[100:].isfinite().all() and o[30:100, 0].isnan().all()
    c = Case(env, 1, 40, 40, 1, 1, 64)
    c.q[3, 0, 0], c.k[7, 0, 0] = float("inf"), 1.0
    o, lse = c.forward()
    assert o[3].isnan().all() and o[4:].isfinite().all() and o[:3].isfinite().all() and not lse[0, 3].isfinite()


def test_starts_and_lengths_out_of_range(env):
    """Cut to the rows there are: nothing outside is read or written."""
    dp, _ = env
    q, k, v = (torch.randn(40, 2 * 32, device="cuda").bfloat16() for _ in range(3))
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")   # noqa: E731
    d = dp.attention_desc(3, 16, 16, 2, 2, 32, q_rows=40, kv_rows=40)
    room = torch.full((60, 64), 7.0, device="cuda").bfloat16()
    o, lse = room[10:50], torch.full((2, 40), 7.0, device="cuda")
    for seqs in (dp.attention_seqs(q_starts=dev([-5, 10, 1000, 2000]), kv_starts=dev([30, 20, -3, 90])), dp.attention_seqs(q_starts=dev([0, 40, 40, 40]), kv_starts=dev([0, 40, 40, 40]))):
        dp.dp_attention_fwd(d, q, k, v, o, lse, seqs)
        torch.cuda.synchronize()
        assert (room[:10] == 7).all() and (room[50:] == 7).all() and (o[26:] == 7).all()
    assert (o[:16] != 0).any(dim=1).all() and (o[16:26] == 0).all()   # the first call's queries had no keys
    d = dp.attention_desc(2, 16, 16, 2, 2, 32)
    qq = q[:32].contiguous()
    o1, o2 = torch.empty(32, 64, device="cuda").bfloat16(), torch.empty(32, 64, device="cuda").bfloat16()
    dp.dp_attention_fwd(d, qq, k, v, o1, None, dp.attention_seqs(q_lens=dev([99, -4]), kv_lens=dev([1 << 30, 8])))
    dp.dp_attention_fwd(d, qq, k, v, o2, None, dp.attention_seqs(q_lens=dev([16, 0]), kv_lens=dev([16, 8])))
    assert torch.equal(o1, o2)


def test_same_bits_on_another_stream_and_in_a_graph(env):
    for args in ((2, 200, 300, 8, 2, 64, -1, 0), (2, 1, 3000, 8, 2, 128, -1, 0)):
        c = Case(env, *args)
        o, lse = c.forward()
        grads = c.backward(o, lse)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            o2, lse2 = c.forward()
            grads2 = c.backward(o2, lse2)
        torch.cuda.synchronize()
        q, k, v, dout = c.wide(c.q), c.wide(c.k), c.wide(c.v), c.dout.reshape(c.q_rows, -1)
        o3, lse3, grads3 = torch.empty_like(o), torch.empty_like(lse), [torch.full_like(t, 55.0) for t in grads]
        ws = [torch.full((c.dp.dp_attention_workspace_bytes(c.desc, p) + 16,), 0xff, dtype=torch.uint8, device="cuda") for p in (c.dp.DP_PASS_FWD, c.dp.DP_PASS_DGRAD)]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.dp.dp_attention_fwd(c.desc, q, k, v, o3, lse3, c.seqs, ws[0])
            c.dp.dp_attention_bwd(c.desc, q, k, v, o3, dout, lse3, *grads3, c.seqs, ws[1])
        for _ in range(3):
            for t in (o3, lse3):
                t.fill_(3.0)
            for t in grads3:
                t.fill_(55.0)
            for w in ws:
                w.fill_(0xff)
            g.replay()
            torch.cuda.synchronize()
            for a, b, e in zip((o, lse, *grads), (o2, lse2, *grads2), (o3, lse3, *grads3)):
                assert torch.equal(a, b) and torch.equal(a, e)


def test_without_lse(env):
    c = Case(env, 2, 150, 150, 4, 2, 64, -1, 0)
    a, _ = c.forward()
    b, _ = c.forward(lse=False)
    assert torch.equal(a, b)


def test_rows_far_apart(env):
    """Offsets beyond 2^31 elements: the second sequence's cache begins 2.3e9 elements behind the first one's."""
    dp, O = env
    kv_len, hk, dim, lens = 2_250_000, 8, 128, (5, 300)
    k, v = (torch.empty((2 * kv_len, hk * dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    used = torch.cat([torch.arange(lens[0]), kv_len + torch.arange(lens[1])]).cuda()
    for t in (k, v):
        t[used] = torch.randn((len(used), hk * dim), generator=g, device="cuda").bfloat16()
    q = torch.randn((2, 2 * hk * dim), generator=g, device="cuda").bfloat16()
    d = dp.attention_desc(2, 1, kv_len, 2 * hk, hk, dim, right=0)
    o, lse = torch.empty_like(q), torch.empty((2 * hk, 2), device="cuda")
    seqs = dp.attention_seqs(kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    ws = torch.empty(dp.dp_attention_workspace_bytes(d, dp.DP_PASS_FWD) + 16, dtype=torch.uint8, device="cuda")
    dp.dp_attention_fwd(d, q, k, v, o, lse, seqs, ws)
    want, want_lse, size = O.attention(q.double().cpu().numpy().reshape(2, -1, dim), *(t[used].double().cpu().numpy().reshape(-1, hk, dim) for t in (k, v)), [(0, 1, 0, 5), (1, 1, 5, 300)],
                                       dim ** -0.5, -1, 0)
    # bf16: p and o are rounded by at most 2^-8, the rest is far below
    assert np.all(np.abs(o.double().cpu().numpy().reshape(want.shape) - want) <= 2.0 ** -8 * (np.abs(want) + size) * 1.02)
    assert np.allclose(lse.cpu().numpy(), want_lse, rtol=0, atol=1e-4)


@pytest.mark.parametrize("n", [65, 200, 300])
def test_many_short_sequences(env, n):
    """More sequences than a wavefront has lanes, and than blocks count; packed in less memory than n of the longest would need."""
    r = np.random.default_rng(n)
    lq, lk = r.integers(0, 90, n).tolist(), r.integers(0, 140, n).tolist()
    Case(env, n, 90, 140, 2, 1, 64, -1, 0, q_side=("packed", lq, 1, 2), kv_side=("packed", lk, 0, 3)).check(True, True)
    Case(env, n, 1, 3000, 2, 1, 64, -1, 0, kv_side=r.integers(0, 3001, n).tolist()).check()


def test_a_far_longer_longest_sequence(env):
    """What may be the longest is millions of rows, none is: blocks of 32 columns for each of them would be more than a launch has."""
    r = np.random.default_rng(5)
    lq, lk = r.integers(0, 50, 300).tolist(), r.integers(0, 60, 300).tolist()
    Case(env, 300, 3_500_000, 3_500_000, 1, 1, 32, -1, 0, q_side=("packed", lq, 1, 2), kv_side=("packed", lk, 0, 3)).check(True, True)


def test_tokens_one_by_one_give_the_whole(env):
    """A sequence taken token by token over its growing cache: the causal result's rows, whatever lies behind the cache's end."""
    dp, _ = env
    n, total, h, hk, dim = 3, 150, 8, 2, 64
    c = Case(env, n, total, total, h, hk, dim, -1, 0)
    whole, lse = c.forward()
    k, v = (torch.full((n, total, hk * dim), float("nan"), device="cuda").bfloat16() for _ in range(2))
    q, ks, vs = (t.reshape(n, total, -1) for t in (c.q, c.k, c.v))
    d = dp.attention_desc(n, 1, total, h, hk, dim, right=0)
    ws = torch.empty(dp.dp_attention_workspace_bytes(d, dp.DP_PASS_FWD) + 16, dtype=torch.uint8, device="cuda")
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    seqs = dp.attention_seqs(kv_lens=lens)
    for t in range(total):
        k[:, t], v[:, t] = ks[:, t], vs[:, t]
        lens.fill_(t + 1)
        o, l1 = torch.empty((n, h * dim), device="cuda").bfloat16(), torch.empty((h, n), device="cuda")
        dp.dp_attention_fwd(d, q[:, t].contiguous(), k, v, o, l1, seqs, ws)
        want = whole.reshape(n, total, -1)[:, t].float()
        # p and o are each rounded twice on both sides, and p at most 2^-8 of a value whose weighted mean is at most the largest |v| seen
        tol = 2.0 ** -8 * 2 * (want.abs() + vs[:, :t + 1].float().abs().amax(dim=(1, 2))[:, None])
        assert torch.all((o.float() - want).abs() <= tol)
        assert torch.all((l1 - lse.reshape(h, n, total)[:, :, t]).abs() <= 1e-4)


def test_gradient_against_differences(env):
    """(f(x + h d) - f(x - h d)) / 2h of f = sum(o dout) in fp32, summed in 64 bits; how far it may be off: what the results' own tolerance gives, and the step of 2h beside that of h."""
    for left, right in ((-1, -1), (-1, 0), (9, 2)):
        c = Case(env, 2, 37, 50, 4, 2, 40, left, right, bf16=False, gap=8)
        o, lse = c.forward()
        grads = c.backward(o, lse)
        rel, terms = c.sizes()
        base = [c.q.clone(), c.k.clone(), c.v.clone()]
        noise = float(((rel + terms) * c.O.attention(c.host(c.q), c.host(c.k), c.host(c.v), c.seqs_list, c.scale, left, right)[2] * np.abs(c.host(c.dout))).sum())
        for i, g in enumerate(grads):
            gen = torch.Generator(device="cuda").manual_seed(i)
            d = torch.randn(base[i].shape, generator=gen, device="cuda")
            w = c.widths[min(i, 1)]

            def f(step):
                for t, b in zip((c.q, c.k, c.v), base):
                    t.copy_(b)
                (c.q, c.k, c.v)[i].add_(d * step)
                return float((c.forward()[0].double() * c.dout.reshape(c.q_rows, -1).double()).sum())
            slope = {h: (f(h) - f(-h)) / (2 * h) for h in (0.01, 0.02)}
            f(0.0)
            want = float((g[:, :w].double() * d.reshape(-1, w).double()).sum())
            assert abs(want - slope[0.01]) <= 2 * noise / 0.01 + abs(slope[0.02] - slope[0.01]), (i, want, slope, noise)


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_next_tokens_of_very_many_sequences(env, bf16):
    """More tiles of keys, if every sequence were as long as the longest may be, than a gradient's launch has blocks: the forward pass has none for them."""
    r = np.random.default_rng(6)
    c = Case(env, 1024, 1, 131072, 8, 8, 32, -1, 0, bf16, kv_side=("packed", r.integers(0, 9, 1024).tolist(), 1, 2))
    assert c.dp.dp_attention_workspace_bytes(c.desc, c.dp.DP_PASS_DGRAD) == 0
    c.check_forward(c.forward())


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 1, 20000, 8, 2, 128, 2047, 0), (1, 1, 9000, 4, 4, 64, 1000, 500), (2, 1, 7001, 6, 2, 40, 1300, 0), (1, 1, 5000, 2, 1, 96, 1600, -1)], ids=str)
def test_keys_of_a_window_dealt_out(env, case, bf16):
    """One token, few of its keys: every block that the keys are dealt out to has some of them (it writes its part of o into the workspace, [part][head][row][channel] fp32)."""
    c = Case(env, *case, bf16)
    dp, need = c.dp, c.dp.dp_attention_workspace_bytes(c.desc, c.dp.DP_PASS_FWD)
    per = 4 * c.heads * c.q_rows * (c.dim + 2)
    parts, rest = divmod(need, per)
    assert rest == 0 and parts >= 2
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    o, lse = torch.full((c.q_rows, c.widths[0]), 7.0, dtype=c.tdt, device="cuda"), torch.full((c.heads, c.q_rows), 7.0, device="cuda")
    dp.dp_attention_fwd(c.desc, c.wide(c.q), c.wide(c.k), c.wide(c.v), o, lse, c.seqs, ws)
    c.check_forward((o, lse))
    written = ws[:parts * c.heads * c.q_rows * c.dim].reshape(parts, -1).isfinite().all(dim=1)
    assert written.all(), written


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 2), (6, 2), (5, 1), (80, 2)], ids=str)
@pytest.mark.parametrize("window", [(1500, 0), (1100, 700), (1900, -1), (-1, 300)], ids=str)
def test_few_queries_with_windows_over_many_keys(env, heads, window, bf16):
    """Blocks that see different keys, split; padded and packed sequences with fewer keys than a window has, or none."""
    Case(env, 1, 37, 5000, *heads, 64, *window, bf16).check()
    Case(env, 5, 3, 5000, *heads, 40, *window, bf16, q_side=[3, 1, 0, 2, 3], kv_side=[5000, 900, 3000, 0, 2]).check()
    Case(env, 4, 9, 5000, *heads, 72, *window, bf16, q_side=("packed", [9, 0, 1, 4], 1, 2), kv_side=("packed", [4100, 20, 1999, 5000], 2, 1)).check(True, True)


@pytest.mark.parametrize("dim", [64, 96, 112, 128])
@pytest.mark.parametrize("case", [(16, 512, 8), (12, 640, 8), (13, 600, 7), (3, 1100, 12), (16, 1024, 5)], ids=str)
def test_causal_blocks_that_share_compute_units(env, case, dim):
    """512 blocks of 128 columns, 480, 455, 324 and 640, forward and for dq: those behind the first 256 in reverse."""
    n, length, heads = case
    Case(env, n, length, length, heads, heads, dim, -1, 0).check()


def test_lse_of_any_element(env):
    """lse inside a larger buffer, not at a multiple of 16 bytes: the bits of a call with one of its own."""
    c = Case(env, 2, 61, 90, 4, 2, 64, -1, 0)
    dp = c.dp
    o, lse = c.forward()
    grads = c.backward(o, lse)
    for shift in (1, 2, 3):
        room = torch.full((lse.numel() + 8,), 7.0, device="cuda")
        inside = room[shift:shift + lse.numel()].view(lse.shape)
        dp.dp_attention_fwd(c.desc, c.wide(c.q), c.wide(c.k), c.wide(c.v), torch.empty_like(o), inside, c.seqs)
        assert torch.equal(inside, lse) and (room[:shift] == 7).all() and (room[shift + lse.numel():] == 7).all()
        assert all(torch.equal(a, b) for a, b in zip(c.backward(o, inside), grads))
