"""The slopes' gradient and the gradients of rows of few keys within bounds that are well below their values.

In bf16 both rest on corrections: of the slopes' gradient by what the saved output's rounding leaves of a row's sum of dS, and of the saved output by
a second product of probabilities that carry a row.  An emulation of the kernels' roundings without either is outside the bounds (on the CPU), the
kernels are inside."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from paper_2505_01068_amd import binding as B

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(TYPES[dtype]).double().numpy()


def far_keys(dtype):
    """Keys a thousand steps away from every query: the row's sum of dS, 0 but for rounding, is multiplied by a thousand."""
    rng = np.random.default_rng(1)
    n = lambda *s: rng.standard_normal(s)  # noqa: E731
    q, k, v, do = (rounded(x, dtype) for x in (1.5 * n(2, 37, 4, 16), n(2, 40, 2, 16), n(2, 40, 2, 16), n(2, 37, 4, 16)))
    steps = lambda m: np.float32(0.1) * np.arange(m, dtype=np.float32)[None].repeat(2, 0)  # noqa: E731
    return dict(q=q, k=k, v=v, do=do, q_pos=steps(37), k_pos=steps(40) + np.float32(1000.0), slope=np.float32(2.0) ** -(7 + np.arange(4, dtype=np.float32)), doc=None)


def near_keys(dtype, batch, rows, heads, dh, seed):
    rng = np.random.default_rng(seed)
    n = lambda: rounded(rng.standard_normal((batch, rows, heads, dh)), dtype)  # noqa: E731
    pos = np.float32(0.1) * np.arange(rows, dtype=np.float32)[None].repeat(batch, 0)
    return dict(q=rounded(1.5 * n(), dtype), k=n(), v=n(), do=n(), q_pos=pos, k_pos=pos, slope=np.float32(2.0) ** -(1 + np.arange(heads, dtype=np.float32)), doc=None)


def pairs_of_keys(dtype, rows, dh, seed):
    """Documents of two rows, whose keys, values and gradients have much in common: dP is nearly the same for both keys and delta as large."""
    rng = np.random.default_rng(seed)
    n = lambda heads: rng.standard_normal((2, rows, heads, dh))  # noqa: E731
    q, k, v, do = (rounded(x, dtype) for x in (0.3 * n(4), 2 + 0.5 * n(2), 2 + 0.1 * n(2), 1 + 0.2 * n(4)))
    return dict(q=q, k=k, v=v, do=do, q_pos=None, k_pos=None, slope=None, doc=(np.arange(rows, dtype=np.int32) // 2)[None].repeat(2, 0))


def reference(x, dtype, second=False):
    tq, tk = x["q"].shape[1], x["k"].shape[1]
    seen = L.visible(x["q"].shape[0], (tq,), (tk,), 1, q_doc=x["doc"], k_doc=x["doc"])
    return L.core_attention(x["q"], x["k"], x["v"], seen, float(np.float32(x["q"].shape[3] ** -0.5)), 0.0, x["slope"], x["q_pos"], x["k_pos"], x["do"], dtype, second), seen


def emulated(x, seen, second, row_sum):
    """dslope and dq in 64 bits but for the bf16 rounding of probabilities (second: and of what that leaves of heavy ones) and dS."""
    group = x["q"].shape[2] // x["k"].shape[2]
    q, k, v, do = (t.transpose(0, 2, 1, 3) for t in (x["q"], np.repeat(x["k"], group, 2), np.repeat(x["v"], group, 2), x["do"]))
    scale = x["q"].shape[3] ** -0.5
    s = scale * (q @ k.transpose(0, 1, 3, 2))
    if x["slope"] is not None:
        gap = np.abs(x["q_pos"].astype(np.float64)[:, :, None] - x["k_pos"].astype(np.float64)[:, None])[:, None]
        s = s - x["slope"].astype(np.float64)[:, None, None] * gap
    s = np.where(seen[:, None], s, -np.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    total = p.sum(-1, keepdims=True)
    kept = rounded(p, "bf16")
    if second:
        kept = kept + np.where(p > total / 8, rounded(p - kept, "bf16"), 0.0)
    delta = (do * (kept @ v) / total).sum(-1, keepdims=True)
    p = p / total
    ds = p * (do @ v.transpose(0, 1, 3, 2) - delta)
    out = {"dq": scale * (rounded(ds, "bf16") @ k).transpose(0, 2, 1, 3)}
    if x["slope"] is not None:
        left = ds.sum(-1, keepdims=True) * p if row_sum else 0.0
        out["dslope"] = -((ds - left) * gap).sum((0, 2, 3))
    return out


def over(got, want, bound):
    return np.abs(got - want) > bound


NEAR = [(1, 235, 4, 64, 2), (2, 65, 4, 128, 2), (8, 634, 2, 64, 4)]


def test_the_slopes_bound_needs_the_row_sums():
    x = far_keys("bf16")
    (ref, bound), seen = reference(x, "bf16")
    assert np.all(bound["dslope_sharp"] < 0.5 * np.abs(ref["dslope"]))
    for second in (False, True):
        assert not over(emulated(x, seen, second, True)["dslope"], ref["dslope"], bound["dslope_sharp"]).any()
        assert over(emulated(x, seen, second, False)["dslope"], ref["dslope"], bound["dslope_sharp"]).any()


@pytest.mark.parametrize("shape", NEAR)
def test_the_slopes_bound_is_below_their_gradient(shape):
    (ref, bound), _ = reference(near_keys("bf16", *shape), "bf16")
    assert np.linalg.norm(bound["dslope_sharp"]) < 0.25 * np.linalg.norm(ref["dslope"])


@pytest.mark.parametrize("rows,dh", [(64, 16), (130, 64), (64, 128)])
def test_the_bound_of_rows_of_two_keys_needs_the_second_product(rows, dh):
    x = pairs_of_keys("bf16", rows, dh, 4)
    (ref, bound), seen = reference(x, "bf16", second=True)
    assert not over(emulated(x, seen, True, True)["dq"], ref["dq"], bound["dq"]).any()
    assert over(emulated(x, seen, False, True)["dq"], ref["dq"], bound["dq"]).mean() > 0.5


def run(x, dtype):
    dev = lambda t, to=None: None if t is None else torch.from_numpy(np.ascontiguousarray(t)).to(to or torch.from_numpy(np.ascontiguousarray(t)).dtype).cuda()  # noqa: E731
    q, k, v, do = (dev(x[n], TYPES[dtype]) for n in ("q", "k", "v", "do"))
    batch, tq, heads, dh = q.shape
    core = B.make_core(batch, (tq,), (k.shape[1],), heads, k.shape[2], dh, 1, dh ** -0.5, dtype)
    rules = dict(q_pos=dev(x["q_pos"]), k_pos=dev(x["k_pos"]), slope=dev(x["slope"]), q_doc=dev(x["doc"]), k_doc=dev(x["doc"]))
    saved, fwd, bwd = (torch.empty(max(1, n), dtype=torch.uint8, device="cuda") for n in B.im_core_attention_sizes(core))
    B.im_core_attention_fwd(core, q, k, v, saved=saved, workspace=fwd, **rules)
    out = dict(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v), dslope=None if x["slope"] is None else torch.empty_like(rules["slope"]))
    B.im_core_attention_bwd(core, q, k, v, saved, do, workspace=bwd, **out, **rules)
    return {n: t.double().cpu().numpy() for n, t in out.items() if t is not None}


def inside(name, got, want, bound):
    off = np.abs(got - want)
    assert np.all(off <= bound), f"{name}: off by up to {(off / bound).max():.2f} of its bound"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [None] + NEAR)
def test_slopes_gradient(dtype, shape):
    print("sharp slopes", dtype, shape, flush=True)
    x = far_keys(dtype) if shape is None else near_keys(dtype, *shape)
    (ref, bound), _ = reference(x, dtype)
    got = run(x, dtype)
    inside("dslope", got["dslope"], ref["dslope"], bound["dslope_sharp"])
    for n in ("dq", "dk", "dv"):
        inside(n, got[n], ref[n], bound[n])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,dh", [(64, 16), (130, 64), (64, 128)])
def test_rows_of_two_keys(dtype, rows, dh):
    print("sharp pairs", dtype, rows, dh, flush=True)
    x = pairs_of_keys(dtype, rows, dh, 4)
    (ref, bound), _ = reference(x, dtype, second=True)
    got = run(x, dtype)
    for n in ("dq", "dk", "dv"):
        inside(n, got[n], ref[n], bound[n])
