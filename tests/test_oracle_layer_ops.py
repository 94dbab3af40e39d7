"""The fp64 definitions of layer norm, rotary positions and the attention core: gradients against differences, closed forms."""
import numpy as np
import pytest

import oracle
from oracle import layer_ops as L


def rng(seed):
    return np.random.default_rng(seed)


def differences(f, x, dy, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = ((f(a) - f(b)) * dy).sum() / (2 * h)
    return g


def test_layernorm_gradients_are_the_differences():
    r = rng(1)
    x, g, b, dy = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    out = L.layernorm(x, g, b, 1e-3, dy)
    assert np.allclose(out["dx"], differences(lambda z: L.layernorm(z, g, b, 1e-3)["y"], x, dy), atol=1e-8)
    assert np.allclose(out["dgamma"], differences(lambda z: L.layernorm(x, z, b, 1e-3)["y"], g, dy), atol=1e-8)
    assert np.allclose(out["dbeta"], differences(lambda z: L.layernorm(x, g, z, 1e-3)["y"], b, dy), atol=1e-8)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_rotation_that_its_inverse_undoes_and_that_depends_on_differences(interleaved):
    r = rng(2)
    q, k = r.normal(size=(1, 4, 2, 10)), r.normal(size=(1, 4, 2, 10))
    pos, f = r.integers(0, 50, size=(1, 4, 2)).astype(float), r.uniform(0, 1, 4)
    turn = lambda x, p, **kw: L.rotary(x, p, f, [3, 1], interleaved=interleaved, **kw)  # noqa: E731
    assert np.allclose(np.linalg.norm(turn(q, pos), axis=-1), np.linalg.norm(q, axis=-1))
    assert np.allclose(turn(turn(q, pos), pos, inverse=True), q)
    assert np.array_equal(turn(q, pos)[..., 8:], q[..., 8:])
    shift = pos + np.array([5.0, -3.0])
    dots = lambda p: np.einsum("btha,bsha->bhts", turn(q, p), turn(k, p))  # noqa: E731
    assert np.allclose(dots(pos), dots(shift))
    assert not np.allclose(turn(q, pos), turn(q, shift))


def problem(seed, B, q_len, k_len, H, Hkv, dh, masked=True):
    r = rng(seed)
    tq, tk = sum(q_len), sum(k_len)
    g = dict(q=r.normal(size=(B, tq, H, dh)), k=r.normal(size=(B, tk, Hkv, dh)), v=r.normal(size=(B, tk, Hkv, dh)), d_o=r.normal(size=(B, tq, H, dh)))
    g["q_pos"], g["k_pos"] = np.sort(r.integers(0, 6, (B, tq))).astype(float), np.sort(r.integers(0, 6, (B, tk))).astype(float)
    return g


@pytest.mark.parametrize("cap,bias,causal", [(0.0, False, False), (2.0, True, True), (1.5, False, True), (0.0, True, False)])
def test_core_gradients_are_the_differences(cap, bias, causal):
    B, ql, kl, H, Hkv, dh = 2, (2, 3), (3, 2), 4, 2, 3
    g = problem(3, B, ql, kl, H, Hkv, dh)
    slope = rng(4).uniform(0.1, 1, H) if bias else None
    seen = L.visible(B, ql, kl, 0b0111, valid_len=[[3, 1], [0, 2]], q_pos=g["q_pos"], k_pos=g["k_pos"], causal=causal, prefix=np.array([1.0, 2.0]))
    f = lambda **kw: L.core_attention(**{**dict(q=g["q"], k=g["k"], v=g["v"], seen=seen, scale=0.6, cap=cap, slope=slope, q_pos=g["q_pos"],  # noqa: E731
                                               k_pos=g["k_pos"]), **kw})[0]
    out = f(d_o=g["d_o"])
    for n in "qkv":
        assert np.allclose(out["d" + n], differences(lambda z: f(**{n: z})["o"], g[n], g["d_o"]), atol=1e-7), n
    if bias:
        assert np.allclose(out["dslope"], differences(lambda z: f(slope=z)["o"], slope, g["d_o"]), atol=1e-7)
    empty = ~seen.any(2)
    assert empty.any() and np.all(out["o"][empty] == 0) and np.all(np.isneginf(out["lse"].transpose(0, 2, 1)[empty])) and np.all(out["dq"][empty] == 0)


def test_core_against_the_interlaced_attention_without_projections():
    """Identity projections, no further rules: the core is the interlaced attention of the same inputs."""
    r = rng(5)
    seg, d, H = (3, 4, 2), 8, 2
    x, eye = r.normal(size=(2, 9, d)), np.eye(d)
    y = oracle.forward(x, eye, eye, eye, eye, seg, oracle.IM_IFM_FORWARD, H, 0.5)
    y = y[0] if isinstance(y, tuple) else y
    heads = x.reshape(2, 9, H, d // H)
    o = L.core_attention(heads, heads, heads, L.visible(2, seg, seg, oracle.IM_IFM_FORWARD), 0.5)[0]["o"]
    assert np.allclose(o.reshape(2, 9, d), y, atol=1e-12)


def test_visible_pair_by_pair():
    seen = L.visible(1, (2, 1), (2, 2), 0b1001, key_pad=[[0, 1, 0, 0]], q_doc=[[0, 1, 1]], k_doc=[[0, 0, 1, 2]])
    assert seen[0].astype(int).tolist() == [[1, 0, 0, 0], [0, 0, 0, 0], [0, 0, 1, 0]]
    pos = np.array([[0.0, 1.0, 2.0]])
    seen = L.visible(1, (3,), (3,), 1, q_pos=pos, k_pos=pos, causal=True)
    assert seen[0].astype(int).tolist() == [[1, 0, 0], [1, 1, 0], [1, 1, 1]]
    seen = L.visible(1, (3,), (3,), 1, q_pos=pos, k_pos=pos, causal=True, prefix=np.array([1.5]))
    assert seen[0].astype(int).tolist() == [[1, 1, 0], [1, 1, 0], [1, 1, 1]]
