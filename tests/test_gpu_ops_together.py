"""Layer norm, projection, rotary positions, attention and their backward passes as one step, on a stream of its own, against the
same step in fp64 with its gradients by differentiation.

Tolerance: every tensor of the chain is rounded once (half a step: 2^-24 in fp32), and the longest path from x to dx has nine roundings
or fp32 sums of at most 160 terms, each of which the following steps amplify by no more than their norms allow; measured
against the largest element, 1e-5 is 170 half steps for them together.  In bf16 the half step is 2^-8: nine of them, 4e-2."""
import math

import pytest
import torch

from paper_2505_01068_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-5), ("bf16", 4e-2)])
def test_one_step_of_a_layer(dtype, tol):
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[dtype]
    torch.manual_seed(1)
    seg, batch, heads, kv, dh, mask = (20, 75, 65), 2, 4, 2, 32, 0x0EE
    T, d, wide = sum(seg), heads * dh, (heads + 2 * kv) * dh
    pairs = (8, 4, 4)
    x, dy = torch.randn(batch, T, d).to(dt).cuda(), torch.randn(batch, T, heads, dh).to(dt).cuda()
    gamma, beta = (1 + 0.1 * torch.randn(d)).to(dt).cuda(), (0.1 * torch.randn(d)).to(dt).cuda()
    w = (torch.randn(d, wide) / math.sqrt(d)).to(dt).cuda()
    pos = torch.floor(torch.rand(batch, T, 3) * 50).cuda()
    freq = torch.cat([100.0 ** (-torch.arange(n).float() / n) for n in pairs]).cuda()
    time = torch.cat([torch.arange(n).float() * (10.0 / n) for n in seg]).expand(batch, -1).contiguous().cuda()
    slope = torch.tensor([0.5, 0.25, 0.1, 0.05], device="cuda")
    valid = torch.tensor([[20, 60, 30], [9, 75, 65]], dtype=torch.int32, device="cuda")
    core = B.make_core(batch, seg, seg, heads, kv, dh, mask, dh ** -0.5, dtype, cap=8.0)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mean, rstd = torch.empty(batch * T, device="cuda"), torch.empty(batch * T, device="cuda")
        u = B.im_layernorm_fwd(x, gamma, beta, mean=mean, rstd=rstd)
        qkv = (u.view(-1, d) @ w).view(batch, T, heads + 2 * kv, dh)
        q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:]
        B.im_rotary(pos, freq, pairs, q, k, q_out=q, k_out=k)
        n_saved, n_fwd, n_bwd = B.im_core_attention_sizes(core)
        saved, ws = (torch.empty(max(1, n), dtype=torch.uint8, device="cuda") for n in (n_saved, max(n_fwd, n_bwd)))
        rules = dict(valid_len=valid, q_pos=time, k_pos=time, slope=slope)
        o = B.im_core_attention_fwd(core, q, k, v, saved=saved, workspace=ws, **rules)
        g = torch.empty_like(qkv)
        gq, gk, gv = g[:, :, :heads], g[:, :, heads:heads + kv], g[:, :, heads + kv:]
        dslope = torch.empty_like(slope)
        B.im_core_attention_bwd(core, q, k, v, saved, dy, gq, gk, gv, dslope=dslope, workspace=ws, **rules)
        B.im_rotary(pos, freq, pairs, gq, gk, q_out=gq, k_out=gk, inverse=True)
        du = (g.view(-1, wide) @ w.t()).view(batch, T, d)
        dw = u.view(-1, d).t() @ g.view(-1, wide)
        dgamma, dbeta = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        lws = torch.empty(max(1, B.im_layernorm_sizes(batch * T, d, dt)), dtype=torch.uint8, device="cuda")
        dx = B.im_layernorm_bwd(x, gamma, mean, rstd, du, dx=du, dgamma=dgamma, dbeta=dbeta, workspace=lws)
    stream.synchronize()

    f = lambda t: t.detach().double().cpu().requires_grad_()  # noqa: E731
    X, Ga, Be, W, Sl = f(x), f(gamma), f(beta), f(w), f(slope)
    U = (X - X.mean(-1, keepdim=True)) / torch.sqrt(X.var(-1, unbiased=False, keepdim=True) + 1e-5) * Ga + Be
    Q, K, V = (U @ W).view(batch, T, heads + 2 * kv, dh).split((heads, kv, kv), 2)
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(pairs))
    ang = (pos.double().cpu()[..., axis] * freq.double().cpu())[:, :, None]
    turn = lambda z: torch.cat((z[..., :16] * ang.cos() - z[..., 16:] * ang.sin(), z[..., :16] * ang.sin() + z[..., 16:] * ang.cos()), -1)  # noqa: E731
    Q, K, V = turn(Q).transpose(1, 2), turn(K).transpose(1, 2).repeat_interleave(2, 1), V.transpose(1, 2).repeat_interleave(2, 1)
    t = time.double().cpu()
    s = 8 * torch.tanh(Q @ K.transpose(2, 3) * dh ** -0.5 / 8) - Sl.view(1, -1, 1, 1) * (t[:, None, :, None] - t[:, None, None, :]).abs()
    which = torch.repeat_interleave(torch.arange(3), torch.tensor(seg))
    place = torch.cat([torch.arange(n) for n in seg])
    seen = (which[:, None] != which[None])[None] & (place[None] < valid.cpu()[:, which])[:, None]
    O = torch.softmax(s.masked_fill(~seen[:, None], -math.inf), -1) @ V
    want = torch.autograd.grad(O, (X, Ga, Be, W, Sl), dy.double().cpu().transpose(1, 2))
    for name, got, ref in [("o", o.transpose(1, 2), O)] + list(zip(("dx", "dgamma", "dbeta", "dw", "dslope"), (dx, dgamma, dbeta, dw, dslope), want)):
        off = (got.double().cpu() - ref.detach()).abs().max() / ref.detach().abs().max()
        print(name, float(off), flush=True)
        assert off <= tol, (name, float(off))
