"""Host-side checks of group norm, gradient norm, AdamW and log-probabilities: every refusal comes before any launch (no GPU needed)."""
import ctypes as C

import pytest

A = 0x1000   # made-up aligned addresses: validation fails first


@pytest.fixture(scope="module")
def dp():
    from paper_2112_10065_amd import binding
    return binding


def no_gpu(dp):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on the addresses made up here")


def test_struct_sizes(dp):
    assert C.sizeof(dp.dp_group_norm_desc) == 32
    assert C.sizeof(dp.dp_param) == 72 and C.sizeof(dp.dp_param_list) == 40
    assert C.sizeof(dp.dp_adamw_hyper) == 48 and C.sizeof(dp.dp_logprobs_desc) == 24


def test_group_norm_refusals(dp):
    lib = dp.lib
    good = dp.group_norm_desc(2, 5, 7, 24, 3)
    need = dp.dp_group_norm_workspace_bytes(good, dp.DP_PASS_FWD)
    back = dp.dp_group_norm_workspace_bytes(good, dp.DP_PASS_DGRAD)
    assert need > 0 and back > 0 and dp.dp_group_norm_workspace_bytes(good, 7) == 0

    def fwd(d=good, x=A, y=A, ws=A, nbytes=1 << 30, gamma=A, mean=A):
        return lib.dp_group_norm_fwd(C.byref(d) if d is not None else None, x, gamma, A, y, mean, A, ws, nbytes, None)

    def bwd(d=good, x=A, dy=A, mean=A, dx=A, dg=A, db=A, ws=A, nbytes=1 << 30):
        return lib.dp_group_norm_bwd(C.byref(d) if d is not None else None, x, dy, None, A, A, mean, A, dx, dg, db, ws, nbytes, None)

    assert fwd(d=None) == bwd(d=None) == dp.DP_ERR_NULL
    for bad in (dict(x=None), dict(y=None)):
        assert fwd(**bad) == dp.DP_ERR_NULL
    for bad in (dict(x=None), dict(dy=None), dict(mean=None), dict(dx=None, dg=None, db=None)):
        assert bwd(**bad) == dp.DP_ERR_NULL
    for bad in (dict(x=A + 2), dict(y=A + 8), dict(gamma=A + 4), dict(mean=A + 4), dict(ws=A + 4)):
        assert fwd(**bad) == dp.DP_ERR_BAD_DESC
    assert fwd(ws=None) == fwd(nbytes=need - 1) == dp.DP_ERR_WORKSPACE or need == 0
    assert bwd(nbytes=back - 1) == dp.DP_ERR_WORKSPACE
    desc = dp.group_norm_desc
    for bad in (desc(0, 5, 7, 24, 3), desc(2, 0, 7, 24, 3), desc(2, 5, -1, 24, 3), desc(2, 5, 7, 0, 1), desc(2, 5, 7, 24, 5), desc(2, 5, 7, 24, 0),
                desc(2, 5, 7, 24, 3, eps=0.0), desc(2, 5, 7, 24, 3, eps=float("nan")), desc(64, 1024, 1024, 32, 4), desc(1, 1 << 16, 1 << 15, 1, 1),
                desc(1 << 24, 1, 1, 8, 1)):
        assert fwd(d=bad) == bwd(d=bad) == dp.DP_ERR_BAD_DESC
        assert dp.dp_group_norm_workspace_bytes(bad, dp.DP_PASS_FWD) == 0
    for bad in (desc(2, 5, 7, 24, 3, io_dtype=2), desc(2, 5, 7, 24, 3, flags=dp.DP_BIAS), desc(2, 5, 7, 24, 3, flags=dp.DP_RELU | dp.DP_SILU)):
        assert fwd(d=bad) == bwd(d=bad) == dp.DP_ERR_UNSUPPORTED
    assert b"group norm" in lib.dp_last_error()


def test_convolutions_still_refuse_the_new_flag(dp):
    d = dp.conv_desc(2, 8, 8, 16, 16, 3, 3, (1, 1), (1, 1), dp.DP_BF16, dp.DP_SILU)
    assert dp.lib.dp_conv2d_fwd(C.byref(d), A, A, A, A, A, 1 << 30, None) == dp.DP_ERR_UNSUPPORTED


def test_group_norm_valid_calls_reach_the_missing_gpu(dp):
    no_gpu(dp)
    for d in (dp.group_norm_desc(2, 5, 7, 24, 3), dp.group_norm_desc(1, 1, 1, 1, 1, dp.DP_F32, dp.DP_SILU), dp.group_norm_desc(3, 2, 2, 5000, 1, dp.DP_F32)):
        need = max(dp.dp_group_norm_workspace_bytes(d, p) for p in (0, 1))
        assert dp.lib.dp_group_norm_fwd(C.byref(d), A, None, None, A, None, None, A, need, None) == dp.DP_ERR_HIP
        assert dp.lib.dp_group_norm_bwd(C.byref(d), A, A, None, None, None, A, A, None, None, A, A, need, None) == dp.DP_ERR_HIP


def param(dp, count=1000, base=0x100000, **kw):
    p = dp.dp_param()
    p.count = count
    for i, f in enumerate(("grad", "w32", "w_bf16", "m", "v", "m_scale", "v_scale")):
        setattr(p, f, base + 0x10000 * i)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def build(dp, params, state=0, nbytes=None, host=True, device=A):
    arr = (dp.dp_param * max(1, len(params)))(*params)
    need = int(dp.lib.dp_param_table_bytes(arr, len(params)))
    buf = (C.c_uint8 * max(need, 1))()
    lst = dp.dp_param_list()
    st = dp.lib.dp_param_table_build(arr, len(params), state, buf if host else None, need if nbytes is None else nbytes, device, C.byref(lst))
    return st, lst, need, bytes(buf)


def test_param_table(dp):
    st, lst, need, _ = build(dp, [param(dp, 4096), param(dp, 4097, 0x10000000), param(dp, 0, 0), param(dp, 1, 0x20000000)])
    assert st == dp.DP_OK and lst.n_chunks == 4 and need == 4 * 64 and lst.n_elements == 4096 + 4097 + 1 and lst.n_params == 4 and lst.updates == 1
    st, lst, need, _ = build(dp, [])
    assert st == dp.DP_OK and lst.n_chunks == 0 and need == 0
    only = dict(w32=None, w_bf16=None, m=None, v=None, m_scale=None, v_scale=None)
    st, lst, _, _ = build(dp, [param(dp, **only)])
    assert st == dp.DP_OK and lst.updates == 0


def test_param_table_refusals(dp):
    assert build(dp, [param(dp, grad=None)])[0] == dp.DP_ERR_NULL
    for missing in ("w32", "m", "v"):
        assert build(dp, [param(dp, **{missing: None})])[0] == dp.DP_ERR_NULL
    assert build(dp, [param(dp, m_scale=None)])[0] == dp.DP_OK
    for missing in ("m_scale", "v_scale"):
        assert build(dp, [param(dp, **{missing: None})], state=1)[0] == dp.DP_ERR_NULL
    for f in ("grad", "w32", "w_bf16", "m", "v", "m_scale", "v_scale"):
        assert build(dp, [param(dp, **{f: 0x50000008})], state=1)[0] == dp.DP_ERR_BAD_DESC
    assert build(dp, [param(dp, weight_decay=-0.1)])[0] == build(dp, [param(dp, weight_decay=float("inf"))])[0] == dp.DP_ERR_BAD_DESC
    assert build(dp, [param(dp, count=-1)])[0] == dp.DP_ERR_BAD_DESC
    assert build(dp, [param(dp)], state=2)[0] == dp.DP_ERR_UNSUPPORTED
    assert build(dp, [param(dp)], nbytes=63)[0] == dp.DP_ERR_WORKSPACE
    assert build(dp, [param(dp)], host=False)[0] == build(dp, [param(dp)], device=None)[0] == dp.DP_ERR_NULL
    assert build(dp, [param(dp)], device=A + 16)[0] == dp.DP_ERR_BAD_DESC
    # a tensor listed twice, and one that begins inside another
    assert build(dp, [param(dp), param(dp)])[0] == dp.DP_ERR_BAD_DESC
    assert build(dp, [param(dp), param(dp, 8, 0x9000000, w32=0x110000 + 3984)])[0] == dp.DP_ERR_BAD_DESC
    assert build(dp, [param(dp), param(dp, 8, 0x9000000, w32=0x110000 + 4000)])[0] == dp.DP_OK
    assert b"share" in dp.lib.dp_last_error()
    too_many = param(dp, count=(1 << 36), base=0)
    assert dp.lib.dp_param_table_bytes(C.byref(too_many), 1) > 0
    lst = dp.dp_param_list()
    too_many = param(dp, count=(1 << 36), grad=1 << 40, w32=2 << 40, w_bf16=None, m=3 << 40, v=4 << 40)
    assert dp.lib.dp_param_table_build(C.byref(too_many), 1, 0, A, 1 << 40, A, C.byref(lst)) == dp.DP_ERR_BAD_DESC


def test_norm_and_adamw_refusals(dp):
    lib = dp.lib
    lst = build(dp, [param(dp, 5000)])[1]
    lst.table = A
    need = int(lib.dp_grad_norm_workspace_bytes(C.byref(lst)))
    assert need > 0

    def norm(l=lst, most=1.0, out=A, ws=A, nbytes=1 << 20):
        return lib.dp_grad_norm(C.byref(l) if l is not None else None, most, out, ws, nbytes, None)

    def adam(l=lst, h=None, scale=A, **kw):
        h = h or dp.adamw_hyper(**{**dict(lr=1e-3), **kw})
        return lib.dp_adamw_step(C.byref(l) if l is not None else None, C.byref(h), scale, None)

    assert norm(l=None) == norm(out=None) == adam(l=None) == dp.DP_ERR_NULL
    assert lib.dp_adamw_step(C.byref(lst), None, A, None) == dp.DP_ERR_NULL
    for most in (0.0, -1.0, float("nan")):
        assert norm(most=most) == dp.DP_ERR_BAD_DESC
    assert norm(out=A + 8) == norm(ws=A + 8) == dp.DP_ERR_BAD_DESC
    assert norm(ws=None) == norm(nbytes=need - 1) == dp.DP_ERR_WORKSPACE
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(lr=float("inf")), dict(eps=0.0), dict(eps=1e-60),
                dict(eps=-1e-8), dict(step=0), dict(step=-5), dict(scale=A + 2)):
        assert adam(**bad) == dp.DP_ERR_BAD_DESC
    no_table = build(dp, [param(dp)])[1]
    no_table.table = None
    assert norm(l=no_table) == adam(l=no_table) == dp.DP_ERR_NULL
    bad = build(dp, [param(dp)])[1]
    bad.table, bad.state = A, 9
    assert norm(l=bad) == adam(l=bad) == dp.DP_ERR_BAD_DESC
    only = dict(w32=None, w_bf16=None, m=None, v=None, m_scale=None, v_scale=None)
    grads = build(dp, [param(dp, **only)])[1]
    grads.table = A
    assert adam(l=grads) == dp.DP_ERR_NULL


def test_gradients_in_memory_that_a_step_writes(dp):
    """Another block may have written there before the gradient is read."""
    for state in (0, 1):
        assert build(dp, [param(dp), param(dp, 8, 0x9000000, grad=0x110000 + 3984)], state)[0] == dp.DP_ERR_BAD_DESC   # inside the first's w32
        assert b"share" in dp.lib.dp_last_error()
        assert build(dp, [param(dp, grad=0x110000)], state)[0] == dp.DP_ERR_BAD_DESC
        # the written memory begins inside a gradient, behind another gradient that ends before it
        assert build(dp, [param(dp, 4096, 0x4000000), param(dp, 4, 0x5000000, grad=0x4000000), param(dp, 4, 0x6000000, v=0x4000000 + 16368)], state)[0] == dp.DP_ERR_BAD_DESC
        assert build(dp, [param(dp, 4096, 0x4000000), param(dp, 4, 0x5000000, grad=0x4000000), param(dp, 4, 0x6000000, v=0x4000000 + 16384)], state)[0] == dp.DP_OK
    only = dict(w32=None, w_bf16=None, m=None, v=None, m_scale=None, v_scale=None)
    assert build(dp, [param(dp, **only), param(dp, **only)])[0] == dp.DP_OK


def test_adamw_refuses_subnormal_eps(dp):
    """Its reciprocal is infinite in fp32: an element that never had a gradient would become 0 * inf."""
    lst = build(dp, [])[1]   # an empty list: what is not refused launches nothing
    for eps, want in ((1e-39, dp.DP_ERR_BAD_DESC), (2.0 ** -126, dp.DP_OK), (1e-8, dp.DP_OK)):
        assert dp.lib.dp_adamw_step(C.byref(lst), C.byref(dp.adamw_hyper(lr=1e-3, eps=eps)), None, None) == want


def test_param_list_checks_tensors(dp):
    import torch
    g = torch.zeros(1000)
    ok = dict(grad=g, w32=torch.zeros(1000), m=torch.zeros(1000), v=torch.zeros(1000))
    for bad in (dict(grad=g.double()), dict(w32=torch.zeros(999)), dict(w32=torch.zeros(2000)[::2]), dict(m=torch.zeros(1000, dtype=torch.uint8)),
                dict(w_bf16=torch.zeros(1000)), dict(momentum=g)):
        with pytest.raises(ValueError):
            dp.param_list([{**ok, **bad}])


def test_logprobs_refusals(dp):
    lib = dp.lib
    good = dp.logprobs_desc(4, 100, 5)

    def fwd(d=good, z=A, ids=A, logp=A, ent=A, lse=A, top=A, at=A, ws=A, nbytes=1 << 30):
        return lib.dp_logprobs_fwd(C.byref(d) if d is not None else None, z, ids, logp, ent, lse, top, at, ws, nbytes, None)

    def bwd(d=good, z=A, ids=A, lse=A, ent=A, dlogp=A, dent=A, dz=A):
        return lib.dp_logprobs_bwd(C.byref(d) if d is not None else None, z, ids, lse, ent, dlogp, dent, dz, None)

    assert fwd(d=None) == bwd(d=None) == dp.DP_ERR_NULL
    for bad in (dict(z=None), dict(ids=None), dict(top=None), dict(at=None), dict(d=dp.logprobs_desc(4, 100), logp=None, ent=None, lse=None)):
        assert fwd(**bad) == dp.DP_ERR_NULL
    for bad in (dict(z=None), dict(ids=None), dict(lse=None), dict(ent=None), dict(dlogp=None, dent=None), dict(dz=None)):
        assert bwd(**bad) == dp.DP_ERR_NULL
    for bad in (dict(z=A + 1), dict(logp=A + 2), dict(at=A + 1)):
        assert fwd(**bad) == dp.DP_ERR_BAD_DESC
    assert bwd(dz=A + 1) == bwd(lse=A + 2) == dp.DP_ERR_BAD_DESC
    desc = dp.logprobs_desc
    for bad in (desc(-1, 100, 5), desc(4, 0, 0), desc(4, 100, 65), desc(4, 100, -1), desc(4, 3, 5), desc(4, 100, 5, row_stride=99),
                desc(4, 100, 5, row_stride=-100), desc(1 << 24, 100, 5), desc(4, (1 << 30) + 1, 5), desc(4, 100, 5, row_stride=1 << 41)):
        assert fwd(d=bad) == bwd(d=bad) == dp.DP_ERR_BAD_DESC
    assert fwd(d=desc(4, 100, 5, io_dtype=3)) == dp.DP_ERR_UNSUPPORTED
    assert fwd(d=desc(4, 100, 5, dp.DP_F32), z=A + 2) == dp.DP_ERR_BAD_DESC
    assert fwd(d=desc(0, 100, 5), z=None) == bwd(d=desc(0, 100, 5), z=None) == dp.DP_OK   # no rows: nothing to do
    assert b"log-prob" in lib.dp_last_error()


def test_logprobs_valid_calls_reach_the_missing_gpu(dp):
    no_gpu(dp)
    for d in (dp.logprobs_desc(4, 100, 5), dp.logprobs_desc(1, 131072, 64), dp.logprobs_desc(3, 1, 1, dp.DP_F32)):
        need = dp.dp_logprobs_workspace_bytes(d)
        assert dp.lib.dp_logprobs_fwd(C.byref(d), A + 4, A, A, None, None, A, A, A, need, None) == dp.DP_ERR_HIP
    assert dp.lib.dp_logprobs_bwd(C.byref(d), A + 4, None, A, A, None, A, A, None) == dp.DP_ERR_HIP


def test_many_narrow_groups_have_blocks_for_the_whole_card(dp):
    """The forward workspace holds 8 bytes for each split of the pixels and group: norms of a channel or two of large images are cut into slabs of down to a cache line of
    channels, of which a block of the second kernel reads 2048 partials: 32 splits of 64 groups, or 64 of 32."""
    for io, line in ((dp.DP_BF16, 64), (dp.DP_F32, 32)):
        for n, h, w, c, groups in ((1, 224, 224, 2048, 2048), (1, 128, 128, 512, 512), (1, 112, 112, 256, 256), (4, 112, 112, 256, 256), (1, 224, 224, 1024, 512), (1, 160, 160, 250, 250)):
            d = dp.group_norm_desc(n, h, w, c, groups, io)
            splits = dp.dp_group_norm_workspace_bytes(d, dp.DP_PASS_FWD) // (8 * n * groups)
            assert n * splits * -(-c // line) >= min(256, n * -(-c // line) * (2048 // line)), (n, h, w, c, groups, io)


def test_param_list_is_on_one_gpu(dp):
    """A kernel reads every address of the table: parameters of two devices are refused, and host memory before anything is launched."""
    import torch
    def tensors(device):
        return {k: torch.zeros(1000, device=device) for k in ("grad", "w32", "m", "v")}
    here = tensors("cpu")
    for params, device in (([here, tensors("meta")], None), ([tensors("meta"), here], None), ([here], "meta"), ([here], "cuda"), ([dict(grad=here["grad"]), dict(grad=tensors("meta")["grad"])], None)):
        with pytest.raises(ValueError, match=" on "):
            dp.param_list(params, device=device)
    lst = dp.param_list([here, dict(grad=torch.zeros(0, device="meta"), w32=None, m=None, v=None)])   # without elements: no address
    assert lst.desc.n_chunks == 1 and lst.desc.updates == 1 and lst.table.device == here["grad"].device
    out, ws = torch.zeros(4), torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        dp.dp_grad_norm(lst, 1.0, out, ws, stream=0)
    with pytest.raises(ValueError, match="GPU"):
        dp.dp_adamw_step(lst, dp.adamw_hyper(lr=1e-3), stream=0)
