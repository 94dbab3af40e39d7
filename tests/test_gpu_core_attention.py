"""im_core_attention_fwd / im_core_attention_bwd against the fp64 definition, within its elementwise bounds."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import layer_ops as L
from paper_2505_01068_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
IFM, IEM, SELF, DENSE = oracle.IM_IFM_FORWARD, oracle.IM_IEM, B.NAMED_MASKS["self_only"], oracle.IM_DENSE


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Case:
    """One problem with its inputs on the GPU."""

    def __init__(self, dtype, batch, q_len, k_len, heads, kv, dh, mask=DENSE, cap=0.0, bias=False, causal=False, prefix=False, docs=0, pad="none",
                 seed=1, gain=1.5):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.batch, self.q_len, self.k_len, self.heads, self.kv, self.dh = dtype, batch, q_len, k_len, heads, kv, dh
        self.mask, self.cap, self.causal, self.scale = mask, cap, causal, 1.0 / math.sqrt(dh)
        tq, tk = sum(q_len), sum(k_len)
        n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        dev = lambda t: t.to(TYPES[dtype]).cuda()  # noqa: E731
        self.q, self.k, self.v, self.d_o = dev(gain * n(batch, tq, heads, dh)), dev(n(batch, tk, kv, dh)), dev(n(batch, tk, kv, dh)), dev(n(batch, tq, heads, dh))
        u = lambda *s: torch.rand(*s, generator=g)  # noqa: E731
        r = dict.fromkeys(("valid_len", "key_pad", "q_pos", "k_pos", "slope", "prefix", "q_doc", "k_doc"))
        if bias or causal:
            span = 0.1 * max(tk, 1)
            times = lambda lens: torch.cat([torch.arange(x).float() * (span / max(x, 1)) for x in lens]).expand(batch, -1).contiguous()  # noqa: E731
            r["q_pos"], r["k_pos"] = times(q_len), times(k_len)
            if q_len != k_len and tq:
                r["q_pos"] = r["q_pos"] + span / 2
            if prefix:
                r["prefix"] = u(batch) * span / 2
        if bias:
            r["slope"] = 2.0 ** (-8.0 * (torch.arange(heads).float() + 1) / heads)
        if docs:
            r["q_doc"], r["k_doc"] = ((u(batch, x).sort(1).values * docs).int() for x in (tq, tk))
        if pad == "valid_len":
            r["valid_len"] = (torch.tensor(k_len) * u(batch, len(k_len)) * 1.2).int()
            r["valid_len"][0, 0] = 0
        elif pad == "key_pad":
            r["key_pad"] = (u(batch, tk) < 0.3).to(torch.uint8)
        self.rules = {k: None if t is None else t.contiguous().cuda() for k, t in r.items()}
        self.core = B.make_core(batch, q_len, k_len, heads, kv, dh, mask, self.scale, dtype, cap=cap, causal=causal)

    def seen(self):
        r = {k: None if t is None else t.cpu().numpy() for k, t in self.rules.items() if k != "slope"}
        return L.visible(self.batch, self.q_len, self.k_len, self.mask, causal=self.causal, **r)

    def reference(self, seen=None):
        r = self.rules
        with np.errstate(invalid="ignore", over="ignore"):
            return L.core_attention(np64(self.q), np64(self.k), np64(self.v), self.seen() if seen is None else seen, self.scale, self.cap, np64(r["slope"]),
                                    np64(r["q_pos"]), np64(r["k_pos"]), np64(self.d_o), self.dtype)

    def buffers(self):
        saved, fwd, bwd = B.im_core_attention_sizes(self.core)
        full = lambda n: torch.full((max(1, n),), 255, dtype=torch.uint8, device="cuda")  # noqa: E731  (255: NaN in what is read before it is written)
        return full(saved), full(max(fwd, bwd))

    def run(self, backward=True, outs=None, buffers=None):
        nan = lambda t: torch.full(t.shape, float("nan"), dtype=t.dtype, device="cuda")  # noqa: E731
        saved, ws = buffers or self.buffers()
        out = outs or dict(o=nan(self.q), lse=torch.full((self.batch, self.heads, sum(self.q_len)), float("nan"), device="cuda"), dq=nan(self.q), dk=nan(self.k),
                           dv=nan(self.v), dslope=None if self.rules["slope"] is None else nan(self.rules["slope"]))
        B.im_core_attention_fwd(self.core, self.q, self.k, self.v, o=out["o"], lse=out["lse"], saved=saved if backward else None, workspace=ws, **self.rules)
        if backward:
            B.im_core_attention_bwd(self.core, self.q, self.k, self.v, saved, self.d_o, out["dq"], out["dk"], out["dv"], dslope=out["dslope"], workspace=ws,
                                    **self.rules)
        return {n: t for n, t in out.items() if t is not None and (backward or n in ("o", "lse"))}


def inside(out, ref, bound, rows=None):
    for n, t in out.items():
        got, want, b = np64(t), ref[n], bound[n]
        if rows is not None and n in rows:
            got, want, b = (np.where(rows[n], x, 0.0) for x in (got, want, b))
        same = np.isneginf(got) & np.isneginf(want)
        assert np.all(np.isfinite(got) | same), f"{n}: not finite"
        off = np.where(same, 0.0, np.abs(np.where(same, 0, got) - np.where(same, 0, want)))
        assert np.all(off <= b), f"{n}: {(off - b).max():.3e} over its bound, {off.max():.3e} off at most (bound there {b.flat[off.argmax()]:.3e})"


def check(case, backward=True):
    ref, bound = case.reference()
    out = case.run(backward)
    torch.cuda.synchronize()
    inside(out, ref, bound)
    return out


SHAPES = [
    # batch, q_len, k_len, heads, kv heads
    (1, (1,), (1,), 1, 1),
    (2, (8, 8, 8), (8, 8, 8), 4, 4),
    (2, (31, 1, 33), (31, 1, 33), 2, 1),
    (1, (65, 130, 40), (65, 130, 40), 4, 2),
    (3, (5, 0, 7), (64, 32, 0), 3, 3),
    (1, (150,), (300,), 6, 2),
]
RULES = [
    dict(),
    dict(cap=5.0),
    dict(bias=True, pad="valid_len"),
    dict(cap=2.0, bias=True, causal=True),
    dict(causal=True, prefix=True, docs=3),
    dict(docs=2, pad="key_pad", cap=30.0),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("rules", range(len(RULES)))
@pytest.mark.parametrize("dh", [8, 64, 128])
def test_forward_and_backward(dtype, shape, rules, dh):
    batch, ql, kl, heads, kv = SHAPES[shape]
    print("core", dtype, SHAPES[shape], RULES[rules], dh, flush=True)
    mask = [DENSE, IFM, IEM, SELF][(shape + rules) % 4] if len(ql) == 3 else 1
    check(Case(dtype, batch, ql, kl, heads, kv, dh, mask, seed=shape + 10 * rules, **RULES[rules]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh", [1, 2, 5, 7, 16, 24, 31, 32, 33, 40, 48, 63, 80, 96, 100, 127])
def test_every_kind_of_width(dtype, dh):
    print("core width", dtype, dh, flush=True)
    check(Case(dtype, 2, (37, 70, 9), (37, 70, 9), 4, 2, dh, SELF, cap=10.0, bias=True, pad="key_pad", seed=dh))


@pytest.mark.parametrize("dtype,dh", [("fp32", 8), ("fp32", 64), ("bf16", 16), ("bf16", 64), ("bf16", 128), ("fp32", 128)])
@pytest.mark.parametrize("rules", range(len(RULES)))
def test_tiles_of_128_rows(dtype, dh, rules):
    """Enough rows for the kernels whose waves share a streamed tile."""
    print("core wide", dtype, dh, RULES[rules], flush=True)
    case = Case(dtype, 8, (128, 250, 256), (128, 250, 256), 8, 8, dh, IFM, seed=rules, **RULES[rules])
    ref, bound = case.reference()
    inside(case.run(), ref, bound)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv,dh", [(8, 2, 64), (4, 4, 16), (40, 1, 128)])
@pytest.mark.parametrize("rules", [0, 2, 3, 5])
def test_single_tokens_against_a_long_cache(dtype, heads, kv, dh, rules):
    print("core token", dtype, heads, kv, dh, RULES[rules], flush=True)
    case = Case(dtype, 2, (1, 1, 0), (700, 5000, 33), heads, kv, dh, DENSE, seed=rules, **RULES[rules])
    check(case)
    saved, fwd, _ = B.im_core_attention_sizes(case.core)
    assert fwd > 0      # the keys are split


def test_queries_that_see_nothing_and_keys_that_nobody_sees():
    """valid_len 0 and a document without keys: o and gradients 0, lse -inf; NaN and infinities where nobody looks change no bit."""
    for dtype in ("fp32", "bf16"):
        for dh in (16, 64):
            case = Case(dtype, 2, (40, 70, 20), (40, 70, 20), 4, 2, dh, IEM, cap=5.0, bias=True, docs=2, pad="valid_len", seed=5)
            case.rules["valid_len"] = torch.tensor([[0, 50, 20], [40, 0, 7]], dtype=torch.int32, device="cuda")
            case.rules["q_doc"][:, 45:60] = 9
            good = check(case)
            seen = case.seen()
            assert (~seen.any(2)).any()
            nobody = torch.from_numpy(~seen.any(1)).cuda()
            for bad in (float("nan"), float("inf"), -float("inf")):
                case.k[nobody] = bad
                case.v[nobody] = bad
                out = case.run()
                for n, t in good.items():
                    assert torch.equal(out[n], t), (dtype, dh, n, bad)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rules", [dict(causal=True), dict(docs=4), dict(causal=True, prefix=True, cap=5.0, bias=True)])
@pytest.mark.parametrize("dh,few", [(64, True), (64, False), (24, True), (128, False)])
def test_values_that_are_not_finite_stay_with_those_who_see_them(dtype, rules, dh, few):
    """NaN or infinity in a value or key (and in a query, for the gradients): the rows that see it are not finite, every other row has the bits
    it had."""
    print("core bad values", dtype, rules, dh, few, flush=True)
    case = Case(dtype, 1 if few else 8, (70, 128, 100), (70, 128, 100), 4 if few else 16, 2 if few else 16, dh, DENSE, seed=9, **rules)
    seen = case.seen()
    good = {n: t.clone() for n, t in case.run().items()}
    key = max(range(298), key=lambda j: (0 < seen[0, :, j].sum() < 298) * seen[0, :, j].sum())
    for tensor, bad in ((case.v, float("nan")), (case.v, float("inf")), (case.k, float("nan")), (case.k, -float("inf"))):
        keep = tensor[0, key, 0, 0].clone()
        tensor[0, key, 0, 0] = bad
        out = case.run()
        tensor[0, key, 0, 0] = keep
        G = case.heads // case.kv
        sees = torch.from_numpy(seen[0, :, key]).cuda()
        for n in ("o", "dq"):
            t = out[n][0][:, :G]
            assert torch.equal(t[~sees], good[n][0][:, :G][~sees]), n
            assert torch.equal(out[n][0][:, G:], good[n][0][:, G:]) and torch.equal(out[n][1:], good[n][1:]), n
        # a key of -inf may give a score of -inf, exp(-inf) = 0: as if the key were not there
        assert (tensor is case.k and bad == -float("inf")) or not torch.isfinite(out["o"][0][sees][:, :G]).all(dim=-1).any()
        # keys that no query of the bad key's shares keep their gradients
        touched = torch.from_numpy(seen[0][seen[0, :, key]].any(0)).cuda()
        for n in ("dk", "dv"):
            assert torch.equal(out[n][0][~touched][:, 0], good[n][0][~touched][:, 0]), n
            assert torch.equal(out[n][0][:, 1:], good[n][0][:, 1:]), n
    row = 150
    for tensor in (case.q, case.d_o):
        keep = tensor[0, row, 0, 0].clone()
        tensor[0, row, 0, 0] = float("nan")
        out = case.run()
        tensor[0, row, 0, 0] = keep
        unseen = torch.from_numpy(~seen[0, row]).cuda()
        for n in ("dk", "dv"):
            assert torch.equal(out[n][0][unseen], good[n][0][unseen]), n


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_extreme_scores(dtype):
    """Scores of some hundreds, far keys with a bias of thousands, a cap at its limits."""
    for kw in (dict(gain=200.0), dict(gain=200.0, cap=1000.0), dict(gain=50.0, cap=0.01), dict(bias=True, gain=1.0)):
        case = Case(dtype, 1, (60, 90), (60, 90), 2, 2, 32, 0b1111, seed=3, **kw)
        if kw.get("bias"):
            case.rules["k_pos"] += 4000.0
            case.rules["slope"] *= 10
        check(case)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,lead", [(64, 0), (64, 1), (20, 0), (128, 0)])
def test_views_of_one_projection_and_heads_first(dtype, dh, lead):
    """q, k, v as slices of [B, T, heads + 2 kv, dh] (lead: not 16-byte aligned), results into slices and heads-first tensors: the same bits
    as from dense tensors; what lies between stays."""
    case = Case(dtype, 2, (30, 61, 45), (30, 61, 45), 4, 2, dh, IFM, cap=5.0, seed=6)
    want = {n: t.clone() for n, t in check(case).items()}
    T, H, K = 136, 4, 2
    packed = lambda: torch.full((lead + 2 * T * (H + 2 * K) * dh,), 3.0, dtype=TYPES[dtype], device="cuda")[lead:].view(2, T, H + 2 * K, dh)  # noqa: E731
    cut = lambda t: (t[:, :, :H], t[:, :, H:H + K], t[:, :, H + K:])  # noqa: E731
    qkv, grads = packed(), packed()
    for dst, src in zip(cut(qkv), (case.q, case.k, case.v)):
        dst.copy_(src)
    case.q, case.k, case.v = cut(qkv)
    case.d_o = case.d_o.transpose(1, 2).contiguous().transpose(1, 2)
    out = dict(o=torch.empty(2, H, T, dh, dtype=TYPES[dtype], device="cuda").transpose(1, 2), lse=torch.empty(2, H, T, device="cuda"), dslope=None)
    out["dq"], out["dk"], out["dv"] = cut(grads)
    got = case.run(outs=out)
    for n, t in want.items():
        assert torch.equal(got[n], t), n


def test_keys_shared_by_the_batch():
    """A batch stride of 0: one cache for all batch elements."""
    case = Case("bf16", 3, (5,), (200,), 4, 2, 64, 1, seed=7)
    case.k, case.v = case.k[:1].expand(3, -1, -1, -1), case.v[:1].expand(3, -1, -1, -1)
    ref, bound = case.reference()
    inside(case.run(backward=False), ref, bound)


def test_no_queries_or_no_keys():
    case = Case("bf16", 2, (0, 0), (30, 20), 2, 2, 16, 0b1111, bias=True, seed=1)
    out = case.run()
    assert torch.all(out["dk"] == 0) and torch.all(out["dv"] == 0) and torch.all(out["dslope"] == 0)
    case = Case("fp32", 2, (30, 20), (0, 0), 2, 2, 16, 0b1111, bias=True, seed=1)
    out = case.run()
    assert torch.all(out["o"] == 0) and torch.all(torch.isneginf(out["lse"])) and torch.all(out["dq"] == 0) and torch.all(out["dslope"] == 0)


def test_rows_beyond_32_bits_of_offset():
    """A cache whose rows are 2^25 elements apart (over 2^32 bytes from its first row to its last) and one whose batch elements are."""
    case = Case("bf16", 1, (3,), (90,), 2, 1, 64, 1, seed=8)
    want = {n: t.clone() for n, t in case.run(backward=False).items()}
    far = 1 << 25
    big = torch.empty(89 * far + 128, dtype=torch.bfloat16, device="cuda")
    k, v = big.as_strided((1, 90, 1, 64), (0, far, 64, 1)), big.as_strided((1, 90, 1, 64), (0, far, 64, 1), 64)
    k.copy_(case.k)
    v.copy_(case.v)
    case.k, case.v = k, v
    for n, t in case.run(backward=False).items():
        assert torch.equal(t, want[n]), n


@pytest.mark.parametrize("dtype,few", [("bf16", True), ("bf16", False), ("fp32", True), ("fp32", False)])
def test_the_same_bits_again_and_in_two_graphs(dtype, few):
    """Two captured steps that share their workspaces, replayed in turn with eager work between."""
    kw = dict(cap=10.0, bias=True, pad="valid_len")
    if few:
        cases = [Case(dtype, 2, (1, 1, 1), (2000, 3000, 100), 8, 2, 64, DENSE, seed=s, **kw) for s in (1, 2)]
    else:
        cases = [Case(dtype, 4, (256, 300, 128), (256, 300, 128), 16, 16, 64, SELF, seed=s, **kw) for s in (1, 2)]
    first = [{n: t.clone() for n, t in c.run().items()} for c in cases]
    buffers = cases[0].buffers()
    outs = [dict({n: torch.empty_like(t) for n, t in f.items()}) for f in first]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for c, o in zip(cases, outs):
        with torch.cuda.stream(side):
            c.run(outs=o, buffers=buffers)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            c.run(outs=o, buffers=buffers)
    for rep in range(3):
        for o in outs:
            for t in o.values():
                t.fill_(float("nan"))
        for b in buffers:
            b.fill_(255)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        again = cases[rep % 2].run()
        for o, f in zip(outs, first):
            for n, t in f.items():
                assert torch.equal(o[n], t), (rep, n)
        for n, t in again.items():
            assert torch.equal(t, first[rep % 2][n]), (rep, n)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rules", range(len(RULES)))
@pytest.mark.parametrize("few", [True, False])
def test_eight_segments(dtype, rules, few):
    """Any block pattern over the most segments: neighbours with the same partners, with others, empty ones."""
    print("core segments", dtype, rules, few, flush=True)
    ql = (3, 1, 0, 33, 20, 20, 64, 5) if few else (130, 1, 0, 128, 40, 200, 64, 129)
    kl = (40, 7, 9, 0, 64, 31, 1, 2)
    mask = sum(row << (8 * i) for i, row in enumerate((0x35, 0x35, 0xFF, 0x00, 0xC3, 0xC3, 0xC3, 0x80)))
    check(Case(dtype, 2, ql, kl, 4 if few else 16, 2 if few else 16, 24, mask, seed=70 + rules, **RULES[rules]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cap,causal,docs", [(0.0, True, 0), (3.0, True, 4), (0.0, False, 4)])
def test_positions_and_documents_in_any_order(dtype, cap, causal, docs):
    """Times that run backwards or jump, document numbers up to the type's ends, slopes of both signs."""
    print("core order", dtype, cap, causal, docs, flush=True)
    case = Case(dtype, 2, (70, 40), (90, 160), 4, 2, 16, DENSE & 0xF, cap=cap, bias=True, causal=causal, docs=docs, seed=91)
    g = torch.Generator().manual_seed(92)
    for name in ("q_pos", "k_pos", "q_doc", "k_doc"):
        t = case.rules[name]
        if t is not None:
            t = torch.gather(t.cpu(), 1, torch.rand(t.shape, generator=g).argsort(1))
            if t.dtype == torch.int32:
                t = torch.tensor([-(1 << 31), -1, 0, (1 << 31) - 1], dtype=torch.int32)[t.long()]
            else:
                t = t - 4.0
            case.rules[name] = t.contiguous().cuda()
    case.rules["slope"] = torch.tensor([0.25, -0.25, 0.0, 1.0], device="cuda")
    check(case)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_a_scale_of_zero_is_the_mean(dtype, cap):
    case = Case(dtype, 2, (40,), (70,), 2, 1, 16, 1, cap=cap, pad="key_pad", seed=5)
    case.scale = 0.0
    case.core = B.make_core(case.batch, case.q_len, case.k_len, 2, 1, 16, 1, 0.0, dtype, cap=cap)
    check(case)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_calls_at_once(dtype):
    """Calls on two streams, each with its own workspace, give what they give one after the other."""
    cases = [Case(dtype, 1, (4,), (9000,), 4, 2, 64, 1, cap=8.0, seed=3), Case(dtype, 2, (200,), (300,), 4, 2, 64, 1, bias=True, seed=4)]
    want = [{n: t.clone() for n, t in c.run().items()} for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s, c in zip(streams, cases):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(c.run())
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for n in a:
            assert torch.equal(a[n], b[n]), n
