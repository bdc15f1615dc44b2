"""Host-side checks of the head norm with rotary positions and of attention: every refusal comes before any launch (no GPU needed)."""
import ctypes as C

import pytest

A = 0x1000   # made-up aligned addresses: validation fails first


@pytest.fixture(scope="module")
def dp():
    from paper_2112_10065_amd import binding
    return binding


def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on the addresses made up here")


def test_struct_sizes(dp):
    assert C.sizeof(dp.dp_qk_rotary_desc) == 96 and C.sizeof(dp.dp_attention_desc) == 88 and C.sizeof(dp.dp_attention_seqs) == 32


def rot(dp, **kw):
    args = dict(rows=7, heads=4, kv_heads=2, dim=32, pairs=[8, 8], flags=dp.DP_QK_NORM)
    args.update(kw)
    return dp.qk_rotary_desc(**args)


def test_qk_rotary_refusals(dp):
    lib = dp.lib
    good = rot(dp)
    need = dp.dp_qk_rotary_workspace_bytes(good, dp.DP_PASS_DGRAD)
    assert need > 0 and dp.dp_qk_rotary_workspace_bytes(good, dp.DP_PASS_FWD) == 0 and dp.dp_qk_rotary_workspace_bytes(good, 9) == 0

    def fwd(d=good, q=A, k=A, gq=A, gk=A, pos=A, freq=A, qo=A + 64, ko=A + 64):
        return lib.dp_qk_rotary_fwd(C.byref(d) if d is not None else None, q, k, gq, gk, pos, freq, qo, ko, None)

    def bwd(d=good, q=A, k=A, gq=A, gk=A, pos=A, freq=A, dqo=A + 64, dko=A + 64, dq=A + 128, dk=A + 128, dgq=A, dgk=A, ws=A, nbytes=1 << 30):
        return lib.dp_qk_rotary_bwd(C.byref(d) if d is not None else None, q, k, gq, gk, pos, freq, dqo, dko, dq, dk, dgq, dgk, ws, nbytes, None)

    assert fwd(d=None) == bwd(d=None) == dp.DP_ERR_NULL
    for name in ("q", "k", "pos", "freq", "qo", "ko"):
        assert fwd(**{name: None}) == dp.DP_ERR_NULL
        assert fwd(**{name: A + 8}) == dp.DP_ERR_BAD_DESC
    for name in ("q", "k", "pos", "freq", "dqo", "dko", "dq", "dk"):
        assert bwd(**{name: None}) == dp.DP_ERR_NULL
    for name in ("gq", "gk", "dgq", "dgk", "ws", "dq"):
        assert bwd(**{name: A + 4}) == dp.DP_ERR_BAD_DESC
    assert bwd(ws=None) == bwd(nbytes=need - 1) == dp.DP_ERR_WORKSPACE
    for bad in (dict(rows=-1), dict(heads=0), dict(kv_heads=-1), dict(dim=4), dict(dim=36), dict(dim=264), dict(pairs=[]), dict(pairs=[8, -1]), dict(pairs=[8, 9]),
                dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_stride=120), dict(q_stride=132), dict(k_stride=56), dict(k_out_stride=1 << 41),
                dict(dq_stride=4), dict(dk_stride=-64), dict(heads=1 << 27)):
        assert fwd(d=rot(dp, **bad)) == bwd(d=rot(dp, **bad)) == dp.DP_ERR_BAD_DESC, bad
        assert dp.dp_qk_rotary_workspace_bytes(rot(dp, **bad), dp.DP_PASS_DGRAD) == 0
    over = rot(dp)
    over.axes = 4
    assert fwd(d=over) == dp.DP_ERR_BAD_DESC
    for bad in (dict(io_dtype=2), dict(flags=dp.DP_RELU)):
        assert fwd(d=rot(dp, **bad)) == bwd(d=rot(dp, **bad)) == dp.DP_ERR_UNSUPPORTED
    assert bwd(d=rot(dp, flags=0)) == dp.DP_ERR_UNSUPPORTED                  # dgamma without a norm
    assert fwd(d=rot(dp, q_out_stride=256), qo=A) == dp.DP_ERR_BAD_DESC      # in place with another stride
    assert bwd(d=rot(dp, dq_stride=256), dq=A + 64) == dp.DP_ERR_BAD_DESC
    assert b"rotary" in lib.dp_last_error()


def test_qk_rotary_valid_calls(dp):
    no_gpu()
    assert dp.lib.dp_qk_rotary_fwd(C.byref(rot(dp, rows=0)), None, None, None, None, None, None, None, None, None) == dp.DP_OK
    for d in (rot(dp), rot(dp, kv_heads=0), rot(dp, io_dtype=dp.DP_F32, q_stride=132, flags=dp.DP_ROTARY_HALVES), rot(dp, dim=256, pairs=[128]), rot(dp, pairs=[0])):
        keys = A if d.kv_heads else None
        assert dp.lib.dp_qk_rotary_fwd(C.byref(d), A, keys, None, None, A, A, A + 64, A + 64, None) == dp.DP_ERR_HIP
        x = A if d.flags & dp.DP_QK_NORM else None
        assert dp.lib.dp_qk_rotary_bwd(C.byref(d), x, x and keys, None, None, A, A, A, keys, A + 64, A + 64, None, None, None, 0, None) == dp.DP_ERR_HIP


def att(dp, **kw):
    args = dict(n=2, q_len=5, kv_len=7, heads=4, kv_heads=2, dim=32)
    args.update(kw)
    return dp.attention_desc(**args)


def test_attention_refusals(dp):
    lib = dp.lib
    good = att(dp)
    back = dp.dp_attention_workspace_bytes(good, dp.DP_PASS_DGRAD)
    assert back > 0 and dp.dp_attention_workspace_bytes(good, 7) == 0
    long = att(dp, n=1, q_len=1, kv_len=100000)
    split = dp.dp_attention_workspace_bytes(long, dp.DP_PASS_FWD)
    assert split > 0

    def seqs(**kw):
        return dp.attention_seqs(**kw)

    def fwd(d=good, q=A, k=A, v=A, o=A + 64, lse=A, s=None, ws=A, nbytes=1 << 40):
        return lib.dp_attention_fwd(C.byref(d) if d is not None else None, q, k, v, o, lse, C.byref(s) if s is not None else None, ws, nbytes, None)

    def bwd(d=good, q=A, k=A, v=A, o=A, do=A, lse=A, dq=A + 64, dk=A + 128, dv=A + 192, s=None, ws=A, nbytes=1 << 40):
        return lib.dp_attention_bwd(C.byref(d) if d is not None else None, q, k, v, o, do, lse, dq, dk, dv, C.byref(s) if s is not None else None, ws, nbytes, None)

    assert fwd(d=None) == bwd(d=None) == dp.DP_ERR_NULL
    for name in ("q", "k", "v", "o"):
        assert fwd(**{name: None}) == dp.DP_ERR_NULL
        assert fwd(**{name: A + 8}) == dp.DP_ERR_BAD_DESC
    for name in ("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == dp.DP_ERR_NULL
        assert bwd(**{name: A + 2}) == dp.DP_ERR_BAD_DESC
    assert fwd(lse=A + 2) == fwd(ws=A + 8) == dp.DP_ERR_BAD_DESC
    assert fwd(d=long, ws=None) == fwd(d=long, nbytes=split - 1) == bwd(nbytes=back - 1) == bwd(ws=None) == dp.DP_ERR_WORKSPACE
    for bad in (dict(n=-1), dict(q_len=-1), dict(kv_len=-1), dict(q_len=1 << 29), dict(heads=0), dict(kv_heads=0), dict(heads=5), dict(dim=4), dict(dim=20), dict(dim=136),
                dict(left=-2), dict(right=-2), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2e38), dict(q_stride=64), dict(q_stride=132), dict(o_stride=-128),
                dict(v_stride=60), dict(k_stride=1 << 23), dict(q_rows=9), dict(kv_rows=13), dict(q_rows=-1), dict(kv_rows=1 << 32), dict(n=1 << 16, q_len=1 << 20),
                dict(n=1 << 30, q_len=1, kv_len=1), dict(n=1 << 22, q_len=1, kv_len=1), dict(n=1 << 12, q_len=1 << 17), dict(q_len=1 << 28, heads=16)):
        assert fwd(d=att(dp, **bad)) == bwd(d=att(dp, **bad)) == dp.DP_ERR_BAD_DESC, bad
    assert fwd(d=att(dp, io_dtype=2)) == bwd(d=att(dp, io_dtype=2)) == dp.DP_ERR_UNSUPPORTED
    for bad in (seqs(q_starts=A, q_lens=A), seqs(kv_starts=A, kv_lens=A)):
        assert fwd(s=bad) == bwd(s=bad) == dp.DP_ERR_UNSUPPORTED
    assert fwd(s=seqs(q_lens=A + 2)) == bwd(s=seqs(kv_starts=A + 1)) == dp.DP_ERR_BAD_DESC
    assert fwd(d=att(dp, q_rows=9), s=seqs(kv_starts=A)) == dp.DP_ERR_BAD_DESC     # only packed rows may be fewer than n q_len
    for name in ('q', 'k', 'v'):
        assert fwd(o=A, **{name: A}) == dp.DP_ERR_BAD_DESC                       # in place
    for name in ('dq', 'dk', 'dv'):
        assert bwd(**{name: A}) == dp.DP_ERR_BAD_DESC
    assert b"attention" in lib.dp_last_error()
    import torch
    with pytest.raises(ValueError, match="int32"):
        seqs(q_lens=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="not on the current GPU"):
        seqs(kv_lens=torch.zeros(2, dtype=torch.int32))


def test_tensors_of_the_host_are_refused(dp):
    """A kernel would fault on them."""
    import torch
    t = torch.zeros(4096)
    with pytest.raises(ValueError, match="not on the current GPU"):
        dp.dp_attention_fwd(att(dp), A, A, t, A)
    with pytest.raises(ValueError, match="not on the current GPU"):
        dp.dp_attention_bwd(att(dp), A, A, A, A, A, A, A, A, A, ws=t)
    with pytest.raises(ValueError, match="not on the current GPU"):
        dp.dp_qk_rotary_fwd(rot(dp), A, A, None, None, t, A, A, A)
    with pytest.raises(ValueError, match="not on the current GPU"):
        dp.dp_qk_rotary_bwd(rot(dp), A, A, None, None, A, A, A, A, A, A, dgamma_q=t)


class OnGpu:
    """A tensor that says it is on the current GPU; calls without rows look at its type alone."""

    def __init__(self, t):
        self.t, self.dtype, self.nbytes = t, t.dtype, t.nbytes

    def get_device(self):
        import torch
        return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else None

    def data_ptr(self):
        return A

    def is_contiguous(self):
        return self.t.is_contiguous()


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
def test_tensors_of_another_type_are_refused(dp, bf16):
    """A kernel would read past the end of a smaller type's memory, or other numbers than are there."""
    import torch
    io, other = (torch.bfloat16, torch.float32) if bf16 else (torch.float32, torch.bfloat16)
    made = lambda t: OnGpu(torch.zeros(64, dtype=t))   # noqa: E731
    x, f32, f64 = made(io), made(torch.float32), made(torch.float64)
    empty = dict(io_dtype=dp.DP_BF16 if bf16 else dp.DP_F32)
    calls = ((dp.dp_qk_rotary_fwd, rot(dp, rows=0, **empty), dict(q=x, k=x, gamma_q=f32, gamma_k=f32, pos=f32, freq=f64, q_out=x, k_out=x)),
             (dp.dp_qk_rotary_bwd, rot(dp, rows=0, **empty), dict(q=x, k=x, gamma_q=f32, gamma_k=f32, pos=f32, freq=f64, dq_out=x, dk_out=x, dq=x, dk=x, dgamma_q=f32, dgamma_k=f32)),
             (dp.dp_attention_fwd, att(dp, n=0, **empty), dict(q=x, k=x, v=x, o=x, lse=f32)),
             (dp.dp_attention_bwd, att(dp, n=0, **empty), dict(q=x, k=x, v=x, o=x, dout=x, lse=f32, dq=x, dk=x, dv=x)))
    for call, desc, args in calls:
        if "dgamma_q" not in args:
            call(desc, **args, stream=A)
        for name, right in args.items():
            for t in {torch.float16, torch.int64, torch.float64, torch.float32, other} - {right.dtype}:
                with pytest.raises(ValueError, match=f"{t} where the call takes {right.dtype}"):
                    call(desc, **{**args, name: made(t)}, stream=A)
            if right is not x:
                with pytest.raises(ValueError, match="not contiguous"):
                    call(desc, **{**args, name: OnGpu(torch.zeros(128, dtype=right.dtype)[::2])}, stream=A)


def test_attention_valid_calls(dp):
    no_gpu()
    lib = dp.lib
    for d in (att(dp, n=0), att(dp, q_len=0)):
        assert lib.dp_attention_fwd(C.byref(d), None, None, None, None, None, None, None, 0, None) == dp.DP_OK
    assert lib.dp_attention_bwd(C.byref(att(dp, q_len=0, kv_len=0)), *[None] * 9, None, None, 0, None) == dp.DP_OK
    packed = dp.attention_seqs(q_starts=A, kv_starts=A)
    for d, s in ((att(dp), None), (att(dp, kv_len=0), None), (att(dp, q_rows=3, kv_rows=2), packed), (att(dp, left=1 << 30, right=(1 << 31) - 1, io_dtype=dp.DP_F32), None),
                 (att(dp, n=1, q_len=1, kv_len=200000), None), (att(dp, n=64, q_len=1000, kv_len=1000, heads=32, kv_heads=8, dim=128, right=0), None)):
        byref = C.byref(s) if s is not None else None
        need = dp.dp_attention_workspace_bytes(d, dp.DP_PASS_FWD), dp.dp_attention_workspace_bytes(d, dp.DP_PASS_DGRAD)
        assert lib.dp_attention_fwd(C.byref(d), A, A, A, A + 64, None, byref, A, need[0], None) == dp.DP_ERR_HIP
        assert lib.dp_attention_bwd(C.byref(d), A, A, A, A, A, A, A + 64, A + 128, A + 192, byref, A, need[1], None) == dp.DP_ERR_HIP


def test_keys_limit_the_gradient_alone(dp):
    """The forward pass launches nothing for each tile of keys: next tokens of many sequences, the longest of which may be very long."""
    s = dp.attention_seqs(kv_starts=A)
    for d in (att(dp, n=1024, q_len=1, kv_len=131072, heads=32, kv_heads=8, dim=128, kv_rows=1 << 20), att(dp, n=1000, q_len=1, kv_len=1 << 28, heads=16, kv_heads=16, kv_rows=5000)):
        need = dp.dp_attention_workspace_bytes(d, dp.DP_PASS_FWD)
        assert dp.lib.dp_attention_fwd(C.byref(d), A, A, None, A + 64, None, C.byref(s), A, need, None) == dp.DP_ERR_NULL     # what comes behind the limits
        assert dp.lib.dp_attention_bwd(C.byref(d), A, A, None, A, A, A, A + 64, A + 128, A + 192, C.byref(s), A, 1 << 40, None) == dp.DP_ERR_BAD_DESC
        assert dp.dp_attention_workspace_bytes(d, dp.DP_PASS_DGRAD) == 0


RULES = """
#include "attention_common.h"
extern "C" bool wide(const dp_attention_desc *d, long long len, long long rows, long long mult, long long other) { return attn_wide(*d, len, rows, mult, other); }
extern "C" double share(const dp_attention_desc *d) { return attn_share(*d); }
extern "C" int second(int block, int of) { return second_reversed(block, of); }
"""


@pytest.fixture(scope="module")
def rules(dp, tmp_path_factory):
    """The rules that choose a call's blocks, built by themselves for the host."""
    import os
    import shutil
    import subprocess
    if shutil.which("hipcc") is None:
        pytest.skip("no compiler")
    path = tmp_path_factory.mktemp("rules")
    (path / "rules.hip").write_text(RULES)
    csrc = os.path.join(os.path.dirname(dp.__file__), "csrc")
    subprocess.check_call(["hipcc", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "-shared", "-I", csrc, str(path / "rules.hip"), "-o", str(path / "rules.so")])
    lib = C.CDLL(str(path / "rules.so"))
    lib.wide.argtypes, lib.wide.restype = [C.POINTER(dp.dp_attention_desc)] + [C.c_longlong] * 4, C.c_bool
    lib.share.argtypes, lib.share.restype = [C.POINTER(dp.dp_attention_desc)], C.c_double
    return lib


def test_a_chunk_behind_many_keys_takes_the_blocks_of_all_keys(dp, rules):
    """A causal mask hides nearly nothing from few queries at the end of many keys: the choice is that of a call without a mask.  Queries' blocks, then keys'."""
    for q, kv, heads, kv_heads, dim, io in ((512, 32768, 32, 8, 128, dp.DP_BF16), (700, 50000, 32, 8, 96, dp.DP_BF16), (512, 8192, 8, 8, 128, dp.DP_F32), (1024, 65536, 16, 2, 64, dp.DP_F32),
                                            (256, 16384, 32, 8, 128, dp.DP_BF16)):
        args = dict(n=1, q_len=q, kv_len=kv, heads=heads, kv_heads=kv_heads, dim=dim, io_dtype=io)
        masked, whole = att(dp, right=0, **args), att(dp, **args)
        shared = heads // kv_heads
        assert rules.wide(masked, q, q, shared, kv) == rules.wide(whole, q, q, shared, kv), args
        assert rules.wide(masked, kv, kv, 1, q * shared) == rules.wide(whole, kv, kv, 1, q * shared), args


def test_the_share_of_pairs_that_a_mask_leaves(dp, rules):
    """Beside a count; as an area it is off by less than one key of every query.  At least a half."""
    for q, kv in ((1, 1), (1, 50), (50, 1), (40, 40), (30, 100), (100, 30), (7, 90)):
        for left, right in ((-1, 0), (-1, 5), (-1, 33), (-1, 200), (0, -1), (9, -1), (64, -1), (300, -1), (3, 3), (-1, -1)):
            seen = sum(sum((left < 0 or j >= i + kv - q - left) and (right < 0 or j <= i + kv - q + right) for j in range(kv)) for i in range(q)) / (q * kv)
            got = rules.share(att(dp, q_len=q, kv_len=kv, left=left, right=right))
            one_side = (left < 0) != (right < 0)
            assert abs(got - max(0.5, seen)) <= 1 / kv + 1e-12 if one_side else got == 1, (q, kv, left, right, got, seen)
    for n in (1, 197, 4096):
        assert rules.share(att(dp, q_len=n, kv_len=n, right=0)) == rules.share(att(dp, q_len=n, kv_len=n, left=0)) == 0.5


def test_second_blocks_of_a_die_in_reverse(rules):
    """Each of 256 ... 511 once, on the die that it was on, the last first; however many there are."""
    for of in range(257, 769):
        for die in range(8):
            blocks = list(range(256 + die, min(of, 512), 8))
            assert [rules.second(b, of) for b in blocks] == blocks[::-1], (of, die)


def test_nothing_to_turn_needs_no_places(dp):
    """Without pairs freq has no elements, whose address is NULL: the call goes on to its other checks."""
    for pairs in ([0], [0, 0], [0, 0, 0]):
        d = rot(dp, pairs=pairs)
        assert dp.lib.dp_qk_rotary_fwd(C.byref(d), A, A, A + 4, A, None, None, A + 64, A + 64, None) == dp.DP_ERR_BAD_DESC
        assert dp.lib.dp_qk_rotary_bwd(C.byref(d), A, A, A, A, A, None, A + 64, A + 64, A + 128, A + 128, A, A, None, 0, None) == dp.DP_ERR_WORKSPACE
    d = rot(dp, pairs=[0, 4])
    assert dp.lib.dp_qk_rotary_fwd(C.byref(d), A, A, A + 4, A, A, None, A + 64, A + 64, None) != dp.DP_OK
    assert dp.lib.dp_qk_rotary_fwd(C.byref(d), A, A, A, A, A, None, A + 64, A + 64, None) == dp.DP_ERR_NULL
    assert dp.lib.dp_qk_rotary_fwd(C.byref(d), A, A, A, A, None, A, A + 64, A + 64, None) == dp.DP_ERR_NULL


def test_lse_has_the_alignment_of_its_elements(dp):
    """In the gradient as in the forward call: what one writes the other takes."""
    for lse, status in ((A + 4, dp.DP_ERR_WORKSPACE), (A + 12, dp.DP_ERR_WORKSPACE), (A + 1, dp.DP_ERR_BAD_DESC), (None, dp.DP_ERR_NULL)):
        assert dp.lib.dp_attention_bwd(C.byref(att(dp)), A, A, A, A, A, lse, A + 64, A + 128, A + 192, None, None, 0, None) == status, lse
