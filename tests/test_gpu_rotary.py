"""im_rotary against the fp64 definition.  Bound: the cosine and sine are rounded to fp32 after an angle that is exact to 2^-24 of
a half turn (pi u, and the functions' own 2 u), each product and the sum once: (pi + 5) u times |x0| + |x1|, and the result's rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from paper_2505_01068_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def np64(t):
    return t.detach().double().cpu().numpy()


def check(x, got, pos, freq, pairs, interleaved, inverse, dtype):
    p = np64(pos)
    want = L.rotary(np64(x), p if p.ndim == 3 else p[None], np64(freq), pairs, interleaved, inverse)
    mag = L.rotary(np.abs(np64(x)), np.zeros((1, x.shape[1], len(pairs))), np.zeros(sum(pairs)), pairs, interleaved)
    n = sum(pairs)
    i0, i1 = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    both = mag[..., i0] + mag[..., i1]
    bound = np.zeros_like(want)
    bound[..., i0] = bound[..., i1] = (math.pi + 5) * L.U * both
    bound += L.half_step(dtype) * (np.abs(want) + bound)
    bound[..., 2 * n:] = 0
    off = np.abs(np64(got) - want)
    assert np.all(off <= bound), (off - bound).max()


def case(seed, batch, rows, heads, kv, dh, pairs, dtype, span):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(batch, rows, h, dh, generator=g).to(TYPES[dtype]).cuda() for h in (heads, kv))
    pos = torch.floor(torch.rand(batch, rows, len(pairs), generator=g) * span).cuda()
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in pairs]).float().cuda()
    return q, k, pos, freq


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("batch,rows,heads,kv,dh,pairs,span", [
    (1, 1, 1, 1, 2, (1,), 10), (2, 24, 4, 4, 8, (2, 1, 1), 100), (16, 1, 8, 2, 64, (16, 8, 8), 1e5), (3, 77, 5, 5, 30, (7, 5), 1000),
    (2, 130, 8, 2, 128, (16, 8, 8), 5000), (1, 33, 2, 1, 7, (3,), 50), (2, 9, 3, 3, 72, (0, 20, 16, 0), 1e6), (1, 5, 1, 1, 1024, (512,), 1 << 24),
    (2, 3, 70, 70, 256, (64, 32, 32), 300), (1, 700, 1, 1, 4, (1, 1), 700)])
def test_against_the_definition(dtype, interleaved, inverse, batch, rows, heads, kv, dh, pairs, span):
    print("rotary", dtype, interleaved, inverse, batch, rows, heads, kv, dh, pairs, flush=True)
    q, k, pos, freq = case(1, batch, rows, heads, kv, dh, pairs, dtype, span)
    q_out, k_out = B.im_rotary(pos, freq, pairs, q, k, interleaved=interleaved, inverse=inverse)
    check(q, q_out, pos, freq, pairs, interleaved, inverse, dtype)
    check(k, k_out, pos, freq, pairs, interleaved, inverse, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("lead", [0, 3])
def test_slices_of_one_projection_in_place_and_alone(dtype, interleaved, lead):
    """q and k as heads of one [B, T, heads + 2 kv, dh] tensor (lead: not 16-byte aligned), turned where they are; v stays."""
    pairs, (batch, rows, heads, kv, dh) = (8, 4, 4), (2, 61, 4, 2, 40)
    q, k, pos, freq = case(2, batch, rows, heads, kv, dh, pairs, dtype, 500)
    qkv = torch.full((batch * rows * (heads + 2 * kv) * dh + 8,), 5.0, dtype=q.dtype, device="cuda")[lead:][:batch * rows * (heads + 2 * kv) * dh]
    qkv = qkv.view(batch, rows, heads + 2 * kv, dh)
    qs, ks = qkv[:, :, :heads], qkv[:, :, heads:heads + kv]
    qs.copy_(q)
    ks.copy_(k)
    B.im_rotary(pos, freq, pairs, qs, ks, q_out=qs, k_out=ks, interleaved=interleaved)
    check(q, qs, pos, freq, pairs, interleaved, False, dtype)
    check(k, ks, pos, freq, pairs, interleaved, False, dtype)
    assert torch.all(qkv[:, :, heads + kv:] == 5.0)
    alone, none = B.im_rotary(pos, freq, pairs, q, interleaved=interleaved)
    assert none is None and torch.equal(alone, qs)


def test_positions_shared_by_the_batch_and_heads_first_tensors():
    q, k, pos, freq = case(3, 3, 50, 4, 4, 32, (8, 8), "fp32", 90)
    one = pos[:1].expand(3, -1, -1).contiguous()
    want, _ = B.im_rotary(one, freq, (8, 8), q)
    got, _ = B.im_rotary(pos[0].contiguous(), freq, (8, 8), q)
    assert torch.equal(got, want)
    first = q.transpose(1, 2).contiguous().transpose(1, 2)      # [B, heads, T, dh] in memory
    got, _ = B.im_rotary(one, freq, (8, 8), first, q_out=torch.empty_like(first))
    assert torch.equal(got, want)


def test_the_gradient_is_the_inverse_rotation():
    """<turn(x), dy> = <x, inverse(dy)>, up to the rounding of both; and the inverse undoes the rotation."""
    q, k, pos, freq = case(4, 2, 30, 3, 3, 24, (6, 6), "fp32", 1e6)
    y, dy = B.im_rotary(pos, freq, (6, 6), q, k)
    back, _ = B.im_rotary(pos, freq, (6, 6), y, inverse=True)
    assert (back - q).abs().max() <= 2 * (math.pi + 6) * L.U * 2 * q.abs().max()
    dx, _ = B.im_rotary(pos, freq, (6, 6), k, inverse=True)
    a, b = (y.double() * k.double()).sum(), (q.double() * dx.double()).sum()
    assert abs(a - b) <= 2 * (math.pi + 6) * L.U * 2 * (q.abs().max() * k.double().abs().sum())


def test_nothing_to_turn():
    q = torch.empty(2, 0, 3, 8, device="cuda")
    out, _ = B.im_rotary(torch.empty(2, 0, 1, device="cuda"), torch.ones(4, device="cuda"), (4,), q)
    assert out.shape == q.shape


def test_rows_beyond_32_bits_of_offset():
    """Two rows whose distance is over 2^31 elements."""
    far = (1 << 31) + 24
    big = torch.zeros(far + 64, dtype=torch.bfloat16, device="cuda")
    q = big.as_strided((1, 2, 1, 16), (0, far, 16, 1))
    q.copy_(torch.arange(32, device="cuda").view(1, 2, 1, 16))
    pos, freq = torch.tensor([[[3.0], [5.0]]], device="cuda"), torch.linspace(0.1, 1, 8, device="cuda")
    x = q.clone()
    B.im_rotary(pos, freq, (8,), q, q_out=q)
    check(x, q, pos, freq, (8,), False, False, "bf16")
