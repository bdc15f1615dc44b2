"""A layer of attention as a user runs it: projection, norm and rotation of its queries and keys in place, attention, projection back, and the gradient through all of them; against the same
in 64 bits.  Each step's bf16 results are rounded (2^-8 of a value at most); errors of independent roundings are compared as a whole, in the 2-norm: a chain of
`steps` roundings of that size is off by less than steps 2^-8 of the norm, and is usually a third of one."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    from paper_2112_10065_amd import binding as dp
    from oracle import attention_ops
    assert torch.cuda.is_available()
    return dp, attention_ops


def rel(a, b):
    a = a.double().cpu().numpy().reshape(b.shape)
    return np.linalg.norm(a - b) / np.linalg.norm(b)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("n,grid,heads,kv_heads,dim,right", [(2, (6, 7), 4, 4, 32, -1), (1, (50,), 8, 2, 64, 0), (3, (2, 3, 5), 6, 3, 48, -1)], ids=str)
def test_layer(env, n, grid, heads, kv_heads, dim, right, halves):
    dp, O = env
    r = np.random.default_rng(dim)
    tokens, width, qw, kw = int(np.prod(grid)), 128, heads * dim, kv_heads * dim
    rows, total = n * tokens, qw + 2 * kw
    up = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().bfloat16()   # noqa: E731
    x, w1, w2, dy = up(r.normal(size=(rows, width))), up(r.normal(size=(total, width)) / width ** 0.5), up(r.normal(size=(width, qw)) / qw ** 0.5), up(r.normal(size=(rows, width)))
    gamma = [torch.from_numpy(r.uniform(0.5, 1.5, dim).astype(np.float32)).cuda() for _ in range(2)]
    pairs = [dim // 2 // len(grid)] * len(grid)
    places = np.stack(np.meshgrid(*(np.arange(g) for g in grid), indexing="ij"), axis=-1).reshape(-1, len(grid))
    pos, freq = torch.from_numpy(np.tile(places, (n, 1)).astype(np.float32)).cuda(), torch.from_numpy(10000.0 ** -r.uniform(0, 1, sum(pairs))).cuda()
    empty = lambda *s, dtype=torch.bfloat16: torch.full(s, 7.0, dtype=dtype, device="cuda")   # noqa: E731
    p1, p2 = dp.linear_desc(rows, width, total), dp.linear_desc(rows, qw, width)
    flags = dp.DP_QK_NORM | (dp.DP_ROTARY_HALVES if halves else 0)
    rot = dp.qk_rotary_desc(rows, heads, kv_heads, dim, pairs, flags=flags, q_stride=total, k_stride=total, dq_stride=total, dk_stride=total)
    att = dp.attention_desc(n, tokens, tokens, heads, kv_heads, dim, right=right, v_stride=total)
    ws = torch.empty(max(dp.dp_linear_workspace_bytes(p1), dp.dp_linear_workspace_bytes(p2), dp.dp_qk_rotary_workspace_bytes(rot, dp.DP_PASS_DGRAD),
                         *(dp.dp_attention_workspace_bytes(att, p) for p in (0, 1))) + 256, dtype=torch.uint8, device="cuda")
    qkv, q, k, o, lse, y = empty(rows, total), empty(rows, qw), empty(rows, kw), empty(rows, qw), empty(heads, rows, dtype=torch.float32), empty(rows, width)
    dp.dp_linear_fwd_bwd(p1, x=x, W=w1, y=qkv, ws=ws)
    parts = lambda t: (t[:, :qw], t[:, qw:qw + kw], t[:, qw + kw:])   # noqa: E731
    qi, ki, v = parts(qkv)
    dp.dp_qk_rotary_fwd(rot, qi, ki, *gamma, pos, freq, q, k)
    dp.dp_attention_fwd(att, q, k, v, o, lse, None, ws)
    dp.dp_linear_fwd_bwd(p2, x=o, W=w2, y=y, ws=ws)
    do, dw2, dqkv, dq, dk, dx, dw1 = empty(rows, qw), empty(width, qw, dtype=torch.float32), empty(rows, total), empty(rows, qw), empty(rows, kw), empty(rows, width), empty(total, width, dtype=torch.float32)
    dgamma = [empty(dim, dtype=torch.float32) for _ in range(2)]
    dp.dp_linear_fwd_bwd(p2, x=o, W=w2, dy=dy, dx=do, dW=dw2, ws=ws)
    dqi, dki, dv = parts(dqkv)
    dp.dp_attention_bwd(att, q, k, v, o, do, lse, dq, dk, dv, None, ws)
    dp.dp_qk_rotary_bwd(rot, qi, ki, *gamma, pos, freq, dq, dk, dqi, dki, *dgamma, ws)
    dp.dp_linear_fwd_bwd(p1, x=x, W=w1, dy=dqkv, dx=dx, dW=dw1, ws=ws)

    # the same in 64 bits
    h = lambda t: t.double().cpu().numpy()   # noqa: E731
    X, W1, W2, DY, G, F, P = h(x), h(w1), h(w2), h(dy), [h(g) for g in gamma], h(freq), h(pos)
    QKV = X @ W1.T
    Q0, K0, V0 = (t.reshape(rows, -1, dim) for t in parts(QKV))
    Q, K = (O.qk_rotary(t, g, P, F, pairs, halves, True, 1e-6) for t, g in ((Q0, G[0]), (K0, G[1])))
    seqs = [(b * tokens, tokens, b * tokens, tokens) for b in range(n)]
    OUT, LSE, _ = O.attention(Q, K, V0, seqs, dim ** -0.5, -1, right)
    Y = OUT.reshape(rows, qw) @ W2.T
    DO = (DY @ W2).reshape(rows, heads, dim)
    (DQ, DK, DV), _, _ = O.attention_bwd(Q, K, V0, OUT, DO, seqs, dim ** -0.5, -1, right)
    (DQ0, DG0), (DK0, DG1) = (O.qk_rotary_bwd(t, g, P, F, pairs, halves, True, 1e-6, d) for t, g, d in ((Q0, G[0], DQ), (K0, G[1], DK)))
    DQKV = np.concatenate([t.reshape(rows, -1) for t in (DQ0, DK0, DV)], axis=1)
    step = 2.0 ** -8
    for name, got, want, steps in (("qkv", qkv, QKV, 1), ("q", q, Q, 2), ("o", o, OUT, 4), ("y", y, Y, 5), ("do", do, DO, 1), ("dqkv", dqkv, DQKV, 7), ("dgamma", torch.cat(dgamma), np.concatenate([DG0, DG1]), 7),
                                   ("dx", dx, DQKV @ W1, 8), ("dw1", dw1, DQKV.T @ X, 8), ("dw2", dw2, DY.T @ OUT.reshape(rows, qw), 5)):
        assert rel(got, want) <= steps * step, (name, rel(got, want))
    assert np.abs(h(lse) - LSE).max() <= 8 * step * np.abs(h(q)).max()
