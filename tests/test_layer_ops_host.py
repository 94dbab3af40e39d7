"""Refusals of the layer-norm, rotary and attention-core entry points, all before anything touches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2505_01068_amd import binding as B

P = C.c_void_p(256)      # never dereferenced: validation fails first
ODD = C.c_void_p(257)
BIG = 1 << 30
F32, BF16 = B.IM_DTYPE_F32, B.IM_DTYPE_BF16


def err():
    return B.lib().im_last_error().decode()


def view(ptr=256, batch=4096, row=64, head=16):
    return B.ImView(ptr, batch, row, head)


NORM = dict(rows=8, d=64, dtype=F32, x=P, ldx=64, gamma=P, beta=P, eps=1e-5, y=P, ldy=64, mean=None, rstd=None)
NORM_BWD = dict(rows=4096, d=64, dtype=F32, x=P, ldx=64, gamma=P, mean=P, rstd=P, dy=P, lddy=64, dx=P, lddx=64, dgamma=P, dbeta=P, ws=P, nbytes=BIG)


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(rows=(1 << 31) + 1), -1, "rows"), (dict(d=0), -1, "d must"), (dict(d=16385), -2, "16384"), (dict(dtype=2), -1, "dtype"),
    (dict(x=None), -1, "x is NULL"), (dict(y=None), -1, "y is NULL"), (dict(x=ODD), -1, "aligned"), (dict(gamma=ODD), -1, "aligned"),
    (dict(ldx=63), -1, "row distance of x"), (dict(ldy=0), -1, "row distance of y"), (dict(eps=0.0), -1, "eps"), (dict(eps=float("nan")), -1, "eps"),
    (dict(eps=float("inf")), -1, "eps"), (dict(mean=P), -1, "both or neither")])
def test_layernorm_forward_refuses(kw, code, text):
    a = {**NORM, **kw}
    assert B.lib().im_layernorm_fwd(*a.values(), None) == code and text in err()


@pytest.mark.parametrize("kw,code,text", [
    (dict(dx=None, dgamma=None, dbeta=None), -1, "all NULL"), (dict(mean=None), -1, "mean and rstd"), (dict(dy=None), -1, "dy is NULL"),
    (dict(lddx=3), -1, "row distance of dx"), (dict(ws=None), -3, "workspace"), (dict(nbytes=8), -3, "workspace"), (dict(ws=ODD), -1, "workspace must be"),
    (dict(d=20000, ldx=20000, lddy=20000, lddx=20000), -2, "16384")])
def test_layernorm_backward_refuses(kw, code, text):
    a = {**NORM_BWD, **kw}
    assert B.lib().im_layernorm_bwd(*a.values(), None) == code and text in err()


def test_layernorm_sizes():
    assert B.im_layernorm_sizes(0, 8, "fp32") == 0 and B.im_layernorm_sizes(1, 8, "bf16") == 0
    assert 0 < B.im_layernorm_sizes(1 << 30, 16384, "bf16") <= 4 * 256 * 2 * 16384 * 4
    with pytest.raises(B.ImAttnError):
        B.im_layernorm_sizes(5, 0, "fp32")


def rotary(axes=1, pairs=(4,), **kw):
    a = dict(batch=2, rows=3, n_axes=axes, pairs=(C.c_int32 * 4)(*pairs), q_heads=2, k_heads=2, head_dim=16, interleaved=0, inverse=0, dtype=F32)
    a.update(kw)
    return B.ImRotary(*a.values())


@pytest.mark.parametrize("shape,args,text", [
    (dict(axes=0), {}, "n_axes"), (dict(axes=5), {}, "n_axes"), (dict(pairs=(9,)), {}, "together"), (dict(pairs=(0,)), {}, "together"),
    (dict(axes=2, pairs=(8, 1)), {}, "together"), (dict(axes=2, pairs=(9, -1)), {}, "pairs[1]"), (dict(head_dim=1), {}, "head_dim"), (dict(head_dim=1026), {}, "head_dim"),
    (dict(q_heads=0), {}, "q_heads"), (dict(k_heads=-1), {}, "k_heads"), (dict(batch=-1), {}, "batch"), (dict(dtype=5), {}, "dtype"),
    ({}, dict(q=view(0)), "q has a NULL"), ({}, dict(q=None), "q is NULL"), ({}, dict(k_out=view(0)), "k_out has a NULL"), ({}, dict(q_out=view(row=0)), "stride of 0"),
    ({}, dict(q=view(258)), "aligned"), ({}, dict(q=view(row=-64)), "outside"), ({}, dict(pos=None), "pos"), ({}, dict(inv_freq=None), "inv_freq"),
    ({}, dict(pos_batch=-1), "pos_batch"), (dict(batch=65536, rows=32768), {}, "2^31")])
def test_rotary_refuses(shape, args, text):
    a = {**dict(pos=P, pos_batch=3, inv_freq=P, q=view(), q_out=view(), k=view(), k_out=view()), **args}
    assert B.lib().im_rotary_apply(C.byref(rotary(**shape)), *a.values(), None) == -1 and text in err()


def core(**kw):
    a = dict(batch=2, q_len=(8, 8), k_len=(8, 8), n_heads=4, n_kv_heads=2, head_dim=16, live_mask=0xF, scale=0.25, dtype="fp32")
    a.update(kw)
    return B.make_core(**a)


@pytest.mark.parametrize("kw,code,text", [
    (dict(batch=0), -1, "batch"), (dict(batch=65536), -1, "batch"), (dict(n_kv_heads=3), -1, "multiple"), (dict(n_kv_heads=0), -1, "multiple"),
    (dict(n_heads=0), -1, "multiple"), (dict(head_dim=0), -1, "head_dim"), (dict(head_dim=129), -2, "head_dim"), (dict(q_len=(8, -1)), -1, "q_len"),
    (dict(k_len=(1 << 24, 8)), -1, "too many rows"), (dict(live_mask=1 << 4), -1, "live_mask"), (dict(scale=float("nan")), -1, "scale"),
    (dict(scale=-1.0), -1, "scale"), (dict(scale=float("inf")), -1, "scale"), (dict(cap=-1.0), -1, "cap"), (dict(cap=0.001), -1, "cap"), (dict(cap=2000.0), -1, "cap"),
    (dict(cap=float("nan")), -1, "cap"), (dict(batch=65535, q_len=(1 << 20, 0), k_len=(1 << 20, 0)), -1, "workgroups")])
def test_core_shapes_are_refused(kw, code, text):
    with pytest.raises(B.ImAttnError) as e:
        B.im_core_attention_sizes(core(**kw))
    assert e.value.code == code and text in str(e.value)


def rules(**kw):
    r = B.ImCoreRules()
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def forward(c, r=None, **kw):
    a = {**dict(q=view(), k=view(), v=view(), o=view(), lse=None, saved=None, ws=P, nbytes=BIG), **kw}
    return B.lib().im_core_attention_fwd(C.byref(c), C.byref(r) if r else None, *a.values(), None)


def backward(c, r=None, **kw):
    a = {**dict(q=view(), k=view(), v=view(), saved=P, d_o=view(), dq=view(), dk=view(), dv=view(), dslope=None, ws=P, nbytes=BIG), **kw}
    return B.lib().im_core_attention_bwd(C.byref(c), C.byref(r) if r else None, *a.values(), None)


@pytest.mark.parametrize("shape,rule,args,code,text", [
    (dict(causal=True), None, {}, -1, "q_pos and k_pos"), ({}, dict(slope=256), {}, -1, "q_pos and k_pos"), ({}, dict(slope=256, q_pos=256), {}, -1, "q_pos and k_pos"),
    ({}, dict(prefix=256), {}, -1, "prefix needs causal"), ({}, dict(q_doc=256), {}, -1, "both or neither"), ({}, dict(k_doc=256), {}, -1, "both or neither"),
    ({}, dict(valid_len=258), {}, -1, "not aligned"), ({}, None, dict(q=view(0)), -1, "q has a NULL"), ({}, None, dict(v=None), -1, "v is NULL"),
    ({}, None, dict(o=view(head=0)), -1, "stride of 0"), ({}, None, dict(k=view(257)), -1, "aligned"), ({}, None, dict(saved=C.c_void_p(264)), -1, "saved"),
    ({}, None, dict(lse=ODD), -1, "lse"), (dict(q_len=(1, 1), k_len=(5000, 9000)), None, dict(ws=None), -3, "workspace"),
    (dict(q_len=(1, 1), k_len=(5000, 9000)), None, dict(nbytes=64), -3, "workspace"), (dict(q_len=(1, 1), k_len=(5000, 9000)), None, dict(ws=C.c_void_p(260)), -1, "16-byte")])
def test_core_forward_refuses(shape, rule, args, code, text):
    assert forward(core(**shape), rules(**rule) if rule else None, **args) == code and text in err()


@pytest.mark.parametrize("rule,args,code,text", [
    (None, dict(saved=None), -1, "saved is NULL"), (None, dict(dslope=P), -1, "dslope without slope"), (None, dict(ws=None), -3, "workspace"),
    (None, dict(nbytes=16), -3, "workspace"), (None, dict(dk=view(row=0)), -1, "stride of 0"), (None, dict(d_o=view(0)), -1, "d_o has a NULL"),
    (dict(slope=256), {}, -1, "q_pos and k_pos")])
def test_core_backward_refuses(rule, args, code, text):
    assert backward(core(), rules(**rule) if rule else None, **args) == code and text in err()


def test_core_sizes():
    saved, fwd, bwd = B.im_core_attention_sizes(core())
    assert saved >= 2 * 16 * 4 * 16 * 4 + 2 * 4 * 16 * 4 and fwd == 0 and bwd >= 2 * 2 * 4 * 16 * 4
    assert B.im_core_attention_sizes(core(q_len=(0, 0))) == (0, 0, 0)
    assert B.im_core_attention_sizes(core(q_len=(1, 1), k_len=(9000, 9000)))[1] > 0


def test_the_binding_takes_tensors_of_the_current_gpu_only():
    x = torch.zeros(4, 8)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        B.im_layernorm_fwd(x)
    with pytest.raises(ValueError):
        B._rows("t", "x", torch.zeros(4, 8, 16)[:, :5], 16, torch.float32)
    assert B._rows("t", "x", torch.zeros(4, 8, 16)[..., :5], 5, torch.float32) == (32, 16)
    assert B._rows("t", "x", torch.zeros(4, 16)[1:2], 16, torch.float32) == (1, 16)
    with pytest.raises(ValueError):
        B._view("t", "q", torch.zeros(1, 2, 3, 8)[..., ::2], torch.Size((1, 2, 3, 4)), torch.float32)
    with pytest.raises(ValueError):
        B._dtype(torch.float16)
    with pytest.raises(ValueError):
        core(q_len=(1,))


def test_in_place_needs_the_same_places():
    """An operator that writes where it reads refuses a second layout of the same memory."""
    a = {**NORM, **dict(ldy=128)}
    assert B.lib().im_layernorm_fwd(*a.values(), None) == -1 and "in place" in err()
    a = {**NORM_BWD, **dict(dx=P, dy=P, lddx=128)}
    assert B.lib().im_layernorm_bwd(*a.values(), None) == -1 and "in place" in err()
    for q, q_out, k, k_out in ((view(), view(row=128), view(512), view(1024)), (view(), view(1024), view(512), view(512, head=32)),
                               (view(), view(batch=8192), view(512), view(1024))):
        assert B.lib().im_rotary_apply(C.byref(rotary()), P, 3, P, q, q_out, k, k_out, None) == -1 and "in place" in err()


@pytest.mark.parametrize("mask", [1 << 64, -1])
def test_block_patterns_behind_64_bits_are_refused(mask):
    with pytest.raises(ValueError, match="live_mask"):
        core(live_mask=mask)


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_outputs_of_the_core_are_apart_from_its_inputs(name):
    at = dict(q=view(1024), k=view(2048), v=view(4096), d_o=view(8192))
    assert forward(core(), **{n: at[n] for n in "qkv"}, o=at[name]) == -1 and f"o overlaps {name}" in err()
    outs = dict(dq=view(1 << 14), dk=view(1 << 15), dv=view(1 << 16))
    assert backward(core(), **at, **{**outs, "dv": at[name]}) == -1 and f"dv overlaps {name}" in err()
    assert backward(core(), **at, **{**outs, "dv": outs["dk"]}) == -1 and "dv overlaps dk" in err()


@pytest.mark.parametrize("views,text", [((256, 512, 512, 1024), "q_out overlaps k"), ((256, 512, 1024, 256), "k_out overlaps q"), ((256, 512, 1024, 512), "k_out overlaps q_out")])
def test_rotated_queries_and_keys_are_apart(views, text):
    q, q_out, k, k_out = (view(p) for p in views)
    assert B.lib().im_rotary_apply(C.byref(rotary()), P, 3, P, q, q_out, k, k_out, None) == -1 and text in err()
