"""Timed operators of a multimodal encoder layer, in plain form and as the library's own calls.

A case is a dict of plain values.  `op` says which operator it takes:
  norm       layer norm over rows [rows, d]: "fwd" (inference), "train" (forward with statistics + backward)
  rotary     rotary positions with several axes (time, height, width) on queries and keys: "fwd", or "bwd" (the
             rotation of the gradients); the first `axes` entries of p0, p1, p2 are the rotated pairs of each axis
  attention  attention of projected heads on the live blocks of an interlaced mask, with capped scores (`cap`),
             a bias that falls with the distance in time (`bias`), causal visibility with a free prefix (`causal`,
             `prefix`) and documents (`docs`: about that many per sample): "fwd", or "train" (forward + backward)
Lengths t / v / a are those of the three query segments, kt / kv / ka those of the key segments (text, vision,
audio; 0: no such segment).  `pad`: "none", "valid_len" (per-sample lengths between half and all of a segment) or
"key_pad" (a tenth of the keys masked one by one).
"""
import math

import torch

own = False

MASKS = {"ifm_forward": 0x062, "ifm_backward": 0x08C, "iem": 0x111, "self_only": 0x0EE, "dense": 0x1FF}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    def norm(name, way, dtype, rows, d):
        return dict(name=name, op="norm", way=way, dtype=dtype, rows=rows, d=d)

    def rotary(name, way, dtype, batch, rows, heads, kv_heads, dh, pairs, interleaved=False, span=100.0):
        p = tuple(pairs) + (0, 0)
        return dict(name=name, op="rotary", way=way, dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dh=dh,
                    axes=len(pairs), p0=p[0], p1=p[1], p2=p[2], interleaved=interleaved, span=span)

    def attention(name, way, dtype, batch, seg, keys, heads, kv_heads, dh, mask, pad="none", cap=0.0, bias=False, causal=False,
                  prefix=False, docs=0):
        return dict(name=name, op="attention", way=way, dtype=dtype, batch=batch, t=seg[0], v=seg[1], a=seg[2], kt=keys[0], kv=keys[1],
                    ka=keys[2], heads=heads, kv_heads=kv_heads, dh=dh, mask=mask, pad=pad, cap=cap, bias=bias, causal=causal, prefix=prefix,
                    docs=docs)

    c5 = (512, 2048, 2048)
    return [
        # one small request: two samples of 8 + 8 + 8 steps at width 32, where only the latency of a call counts
        norm("norm_fp32_tiny", "fwd", "fp32", 48, 32),
        # training at width 40, 32 samples of 50 + 500 + 375 steps
        norm("norm_fp32_train", "train", "fp32", 29600, 40),
        # training at the doubled width of the intra-modal encoder, 8 samples of 4608 steps
        norm("norm_bf16_train_wide", "train", "bf16", 36864, 1024),
        # one new token for each of 16 running requests, far along their streams, four query heads to a key head
        rotary("rotary_bf16_token", "fwd", "bf16", 16, 1, 8, 2, 64, (16, 8, 8), span=100000.0),
        # long sequences with time, height and width of each step
        rotary("rotary_bf16_long", "fwd", "bf16", 8, 4608, 8, 8, 64, (16, 8, 8), span=4608.0),
        # gradients at the narrow fp32 model, one time axis, neighbouring elements as pairs
        rotary("rotary_fp32_bwd", "bwd", "fp32", 32, 925, 8, 8, 8, (4,), interleaved=True, span=925.0),
        # one small call, as an example or an online request makes it
        attention("attention_fp32_tiny", "fwd", "fp32", 2, (8, 8, 8), (8, 8, 8), 4, 4, 8, "ifm_forward", cap=20.0, bias=True),
        # training with unaligned features: the keys' distance in seconds, per-sample lengths
        attention("attention_fp32_train", "train", "fp32", 32, (50, 500, 375), (50, 500, 375), 8, 8, 5, "ifm_forward", pad="valid_len", bias=True),
        # packed training rows of several documents, a prefix of each sample seen by all, two query heads to a key head
        attention("attention_bf16_documents", "train", "bf16", 3, (333, 1501, 1290), (333, 1501, 1290), 4, 2, 128, "dense", pad="key_pad",
                  causal=True, prefix=True, docs=4),
        # one token for each of 16 requests against the long caches of its own and the two other modalities
        attention("attention_bf16_token", "fwd", "bf16", 16, (1, 1, 1), (1024, 8192, 8192), 8, 2, 64, "dense", pad="valid_len", cap=30.0),
        # inference on long sequences, intra-modal, scores capped
        attention("attention_bf16_infer", "fwd", "bf16", 8, c5, c5, 8, 8, 64, "iem", cap=50.0),
        # the largest: training on long sequences at width 512, scores capped, bias by distance
        attention("attention_bf16_large", "train", "bf16", 8, c5, c5, 8, 8, 64, "ifm_forward", cap=50.0, bias=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.4))))))

    dtype = rng.choice(("fp32", "bf16"))
    op = rng.choice(("norm", "rotary", "attention", "attention", "attention"))
    if op == "norm":
        d = log_int(5, 8192)
        return dict(op=op, way=rng.choice(("fwd", "train")), dtype=dtype, rows=log_int(1, max(1, min(200000, 40000000 // d))), d=d)
    if op == "rotary":
        axes = rng.randint(1, 3)
        dh = rng.choice((6, 8, 16, 30, 32, 64, 72, 96, 128))
        total = rng.choice((dh // 2, max(axes, dh // 4)))
        cut = [total // axes] * axes
        cut[0] += total - sum(cut)
        cut += [0, 0]
        kv = log_int(1, 8)
        heads = kv * rng.choice((1, 1, 2, 4))
        batch = log_int(1, 32)
        return dict(op=op, way=rng.choice(("fwd", "bwd")), dtype=dtype, batch=batch, rows=log_int(1, max(1, 20000000 // (batch * heads * dh))),
                    heads=heads, kv_heads=kv, dh=dh, axes=axes, p0=cut[0], p1=cut[1], p2=cut[2], interleaved=rng.random() < 0.5,
                    span=float(log_int(10, 100000)))
    kv = rng.choice((1, 2, 3, 4, 8))
    heads = kv * rng.choice((1, 1, 2, 4))
    dh = rng.choice((5, 8, 16, 24, 32, 40, 64, 64, 80, 128, rng.randint(1, 128)))
    token = rng.random() < 0.25
    train = not token and rng.random() < 0.6
    top = (9000 if token else 2000) if dtype == "bf16" else 1000
    keys = [log_int(1, top) for _ in range(3)]
    seg = [1, 1, 1] if token else keys if rng.random() < 0.7 else [log_int(1, top) for _ in range(3)]
    batch = log_int(1, 32)
    most = (4.0e10 if dtype == "bf16" else 1.0e10) if train else 4.0e10
    while batch > 1 and batch * heads * sum(seg) * sum(keys) * max(dh, 32) > most:
        batch = (batch + 1) // 2
    while heads * sum(seg) * sum(keys) * max(dh, 32) > most:
        keys = [max(1, n // 2) for n in keys]
        seg = [max(1, n // 2) for n in seg]
    causal = rng.random() < 0.4
    return dict(op=op, way="train" if train else "fwd", dtype=dtype, batch=batch, t=seg[0], v=seg[1], a=seg[2], kt=keys[0], kv=keys[1],
                ka=keys[2], heads=heads, kv_heads=kv, dh=dh, mask=rng.choice(sorted(MASKS)), pad=rng.choice(("none", "valid_len", "key_pad")),
                cap=rng.choice((0.0, 0.0, 10.0, 30.0, 50.0)), bias=rng.random() < 0.5, causal=causal, prefix=causal and rng.random() < 0.5,
                docs=rng.choice((0, 0, 3)))


def segments(case):
    return (case["t"], case["v"], case["a"]), (case["kt"], case["kv"], case["ka"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, dtype=dt, gain=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(gain).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    st = {"case": case}
    if case["op"] == "norm":
        rows, d = case["rows"], case["d"]
        # activations of a residual stream: every channel has a level and a spread of its own
        st["x"] = (torch.randn(rows, d, generator=g, device="cuda") * (0.5 + uniform(d)) + normal(d, dtype=torch.float32, gain=0.5)).to(dt)
        st["gamma"], st["beta"] = (1 + normal(d, dtype=torch.float32, gain=0.1)).to(dt), normal(d, gain=0.1)
        if case["way"] == "train":
            st["dy"] = normal(rows, d)
        return st
    if case["op"] == "rotary":
        batch, rows, axes, dh = case["batch"], case["rows"], case["axes"], case["dh"]
        st["pairs"] = [case["p0"], case["p1"], case["p2"]][:axes]
        st["axis"] = torch.tensor([a for a, n in enumerate(st["pairs"]) for _ in range(n)], device="cuda")
        # queries and keys where the projection left them: side by side in one row
        qkv = normal(batch, rows, case["heads"] + 2 * case["kv_heads"], dh)
        st["q"], st["k"] = qkv[:, :, :case["heads"]], qkv[:, :, case["heads"]:case["heads"] + case["kv_heads"]]
        st["pos"] = torch.floor(uniform(batch, rows, axes) * case["span"])  # frame, line and column numbers
        st["inv_freq"] = torch.cat([10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / max(n, 1)) for n in st["pairs"]]).float()
        return st
    seg, keys = segments(case)
    batch, heads, kv_heads, dh, tq, tk = case["batch"], case["heads"], case["kv_heads"], case["dh"], sum(seg), sum(keys)
    # which rows of queries and keys may meet at all, and each key's place in its segment
    which_q, which_k = (torch.tensor([i for i, n in enumerate(lengths) for _ in range(n)], device="cuda") for lengths in (seg, keys))
    live = torch.tensor([[bool(MASKS[case["mask"]] >> (3 * i + j) & 1) for j in range(3)] for i in range(3)], device="cuda")
    st["blocks"], st["which_k"] = live[which_q][:, which_k], which_k
    st["place"] = torch.tensor([p for n in keys for p in range(n)], device="cuda")
    st["q"] = normal(batch, tq, heads, dh, gain=1.5)
    st["k"], st["v"] = normal(batch, tk, kv_heads, dh), normal(batch, tk, kv_heads, dh)
    if case["way"] == "train":
        st["do"] = normal(batch, tq, heads, dh)
    # times in seconds: the modalities are sampled at rates of their own over the same clip; a single new step comes at its end
    span = 0.1 * max(keys)

    def times(lengths, at_end):
        one = [torch.full((1,), span, device="cuda") if at_end and n == 1 else torch.arange(n, device="cuda", dtype=torch.float32) * (span / n)
               for n in lengths]
        return torch.cat(one).expand(batch, -1).contiguous()

    st["k_pos"], st["q_pos"] = times(keys, False), times(seg, seg != keys)
    st["slope"] = 2.0 ** (-8.0 * (torch.arange(heads, device="cuda", dtype=torch.float32) + 1) / heads) if case["bias"] else None
    st["prefix"] = span * 0.5 * uniform(batch) if case["prefix"] else None
    st["valid_len"] = st["key_pad"] = st["q_doc"] = st["k_doc"] = None
    if case["pad"] == "valid_len":
        n = torch.tensor(keys, device="cuda")
        st["valid_len"] = torch.ceil(n * (0.5 + 0.5 * uniform(batch, 3))).to(torch.int32)
    elif case["pad"] == "key_pad":
        st["key_pad"] = (uniform(batch, tk) < 0.1).to(torch.uint8)
    if case["docs"]:
        ends = span * uniform(batch, case["docs"] - 1).sort(1).values  # where in time a sample's documents end
        st["q_doc"], st["k_doc"] = (torch.searchsorted(ends, p, right=True).to(torch.int32) for p in (st["q_pos"], st["k_pos"]))
    return st


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ----

def plain_norm(st, eps=1e-5):
    case, dt = st["case"], st["x"].dtype
    x, gamma, beta = st["x"].float(), st["gamma"].float(), st["beta"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / torch.sqrt((centred * centred).mean(1, keepdim=True) + eps)
    xhat = centred * rstd
    out = {"y": (xhat * gamma + beta).to(dt)}
    if case["way"] == "train":
        dy = st["dy"].float()
        out["mean"], out["rstd"] = mean[:, 0], rstd[:, 0]
        out["dgamma"], out["dbeta"] = (dy * xhat).sum(0), dy.sum(0)
        w = dy * gamma
        out["dx"] = (rstd * (w - w.mean(1, keepdim=True) - xhat * (w * xhat).mean(1, keepdim=True))).to(dt)
    return out


def plain_rotary(st):
    case = st["case"]
    axis = st["axis"]
    # far positions times frequencies: the angle's integer part would eat a 32-bit fraction
    angle = st["pos"].double()[..., axis] * st["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if case["way"] == "bwd":
        sin = -sin
    n = axis.numel()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["interleaved"] else (slice(0, n), slice(n, 2 * n))

    def turn(x):
        y = x.float()
        a, b = y[..., first], y[..., second]
        out = y.clone()
        out[..., first], out[..., second] = a * cos - b * sin, a * sin + b * cos
        return out.to(x.dtype)

    return {"q": turn(st["q"]), "k": turn(st["k"])}


def plain_visible(st):
    """[batch, queries, keys]: who sees whom."""
    case = st["case"]
    seen = st["blocks"][None]
    if st["valid_len"] is not None:
        seen = seen & (st["place"] < st["valid_len"][:, st["which_k"]])[:, None]
    if st["key_pad"] is not None:
        seen = seen & (st["key_pad"] == 0)[:, None]
    if st["q_doc"] is not None:
        seen = seen & (st["q_doc"][:, :, None] == st["k_doc"][:, None])
    if case["causal"]:
        before = st["k_pos"][:, None] <= st["q_pos"][:, :, None]
        seen = seen & ((before | (st["k_pos"] < st["prefix"][:, None])[:, None]) if st["prefix"] is not None else before)
    return seen.expand(case["batch"], -1, -1)


def plain_attention(st):
    case, dt = st["case"], st["q"].dtype
    batch, heads, kv_heads, dh, cap = case["batch"], case["heads"], case["kv_heads"], case["dh"], case["cap"]
    group, scale = heads // kv_heads, 1.0 / math.sqrt(dh)
    heads_first = lambda x: x.float().transpose(1, 2)  # noqa: E731
    q = heads_first(st["q"])
    k, v = (heads_first(x).repeat_interleave(group, 1).contiguous() for x in (st["k"], st["v"]))
    hidden = ~plain_visible(st)[:, None]
    s = torch.matmul(q, k.transpose(2, 3)) * scale
    if cap:
        t = torch.tanh(s / cap)
        s = cap * t
    if st["slope"] is not None:
        far = (st["q_pos"][:, :, None] - st["k_pos"][:, None]).abs()[:, None]
        s = s - st["slope"][:, None, None] * far
    s = s.masked_fill(hidden, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(s - top)
    del s
    total = p.sum(3, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v)
    out = {"o": o.transpose(1, 2).to(dt), "lse": lse}
    if case["way"] == "train":
        do = heads_first(st["do"])
        ds = torch.matmul(do, v.transpose(2, 3))
        ds = p * (ds - (do * o).sum(3, keepdim=True))
        if st["slope"] is not None:
            out["dslope"] = -(ds * far).sum((0, 2, 3), dtype=torch.float64).float()
        if cap:
            ds = ds * (1 - t * t)
        shared = lambda x: x.reshape(batch, kv_heads, group, -1, dh).sum(2).transpose(1, 2).to(dt)  # noqa: E731
        out["dq"] = (torch.matmul(ds, k) * scale).transpose(1, 2).to(dt)
        out["dk"] = shared(torch.matmul(ds.transpose(2, 3), q) * scale)
        out["dv"] = shared(torch.matmul(p.transpose(2, 3), do))
    return out


# ---- the library's calls ----

def buffers(*sizes):
    return [torch.empty(max(1, n), dtype=torch.uint8, device="cuda") for n in sizes]


def own_norm(st):
    from paper_2505_01068_amd import binding as B
    case, x = st["case"], st["x"]
    if "y" not in st:  # what a program keeps between its steps: outputs and a workspace
        st["y"], st["mean"], st["rstd"] = torch.empty_like(x), x.new_empty(case["rows"], dtype=torch.float32), x.new_empty(case["rows"], dtype=torch.float32)
        if case["way"] == "train":
            st["dx"], st["dgamma"], st["dbeta"] = torch.empty_like(x), *(x.new_empty(case["d"], dtype=torch.float32) for _ in range(2))
            st["ws"], = buffers(B.im_layernorm_sizes(case["rows"], case["d"], x.dtype))
    if case["way"] == "fwd":
        return {"y": B.im_layernorm_fwd(x, st["gamma"], st["beta"], 1e-5, y=st["y"])}
    B.im_layernorm_fwd(x, st["gamma"], st["beta"], 1e-5, y=st["y"], mean=st["mean"], rstd=st["rstd"])
    B.im_layernorm_bwd(x, st["gamma"], st["mean"], st["rstd"], st["dy"], dx=st["dx"], dgamma=st["dgamma"], dbeta=st["dbeta"], workspace=st["ws"])
    return {n: st[n] for n in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}


def own_rotary(st):
    from paper_2505_01068_amd import binding as B
    case = st["case"]
    if "q_out" not in st:
        st["q_out"], st["k_out"] = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (st["q"], st["k"]))
    B.im_rotary(st["pos"], st["inv_freq"], st["pairs"], st["q"], st["k"], q_out=st["q_out"], k_out=st["k_out"],
                interleaved=case["interleaved"], inverse=case["way"] == "bwd")
    return {"q": st["q_out"], "k": st["k_out"]}


def own_attention(st):
    from paper_2505_01068_amd import binding as B
    case, q = st["case"], st["q"]
    train = case["way"] == "train"
    if "core" not in st:
        seg, keys = segments(case)
        st["core"] = core = B.make_core(case["batch"], seg, keys, case["heads"], case["kv_heads"], case["dh"], MASKS[case["mask"]],
                                        1.0 / math.sqrt(case["dh"]), case["dtype"], cap=case["cap"], causal=case["causal"])
        saved, forward, backward = B.im_core_attention_sizes(core)
        st["ws"], = buffers(max(forward, backward) if train else forward)
        st["saved"], = buffers(saved) if train else (None,)
        st["o"], st["lse"] = torch.empty_like(q), q.new_empty(case["batch"], case["heads"], sum(seg), dtype=torch.float32)
        if train:
            st["dq"], st["dk"], st["dv"] = (torch.empty_like(st[n]) for n in "qkv")
            st["dslope"] = torch.empty_like(st["slope"]) if case["bias"] else None
        st["rules"] = {n: st[n] for n in ("valid_len", "key_pad", "slope", "prefix", "q_doc", "k_doc")}
        if case["bias"] or case["causal"]:
            st["rules"].update(q_pos=st["q_pos"], k_pos=st["k_pos"])
    B.im_core_attention_fwd(st["core"], q, st["k"], st["v"], o=st["o"], lse=st["lse"], saved=st["saved"], workspace=st["ws"], **st["rules"])
    out = {"o": st["o"], "lse": st["lse"]}
    if train:
        B.im_core_attention_bwd(st["core"], q, st["k"], st["v"], st["saved"], st["do"], st["dq"], st["dk"], st["dv"], dslope=st["dslope"],
                                workspace=st["ws"], **st["rules"])
        out.update((n, st[n]) for n in ("dq", "dk", "dv"))
        if case["bias"]:
            out["dslope"] = st["dslope"]
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return own_norm(state) if op == "norm" else own_rotary(state) if op == "rotary" else own_attention(state)
    return plain_norm(state) if op == "norm" else plain_rotary(state) if op == "rotary" else plain_attention(state)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "norm":
        n, rows, d = case["rows"] * case["d"], case["rows"], case["d"]
        if case["way"] == "fwd":
            return {"bytes": size * (2 * n + 2 * d), "flops": 8 * n}
        return {"bytes": size * (5 * n + 3 * d) + 16 * rows + 8 * d, "flops": 24 * n}
    if case["op"] == "rotary":
        n = case["batch"] * case["rows"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * size * n * case["dh"] + 4 * case["batch"] * case["rows"] * case["axes"], "flops": 6 * n * (case["p0"] + case["p1"] + case["p2"])}
    seg, keys = segments(case)
    share = 1.0 if case["pad"] == "none" else 0.75 if case["pad"] == "valid_len" else 0.9
    share *= (0.5 if case["causal"] and seg == keys else 1.0) / max(1, case["docs"])
    pairs = sum(seg[i] * keys[j] for i in range(3) for j in range(3) if MASKS[case["mask"]] >> (3 * i + j) & 1)
    pairs *= share * case["batch"] * case["heads"]
    tq, tk = (case["batch"] * case["dh"] * size * n for n in (sum(seg) * case["heads"], sum(keys) * case["kv_heads"]))
    tk_seen = tk * (0.75 if case["pad"] == "valid_len" else 1.0)
    stats = 4 * case["batch"] * case["heads"] * sum(seg)
    if case["way"] == "fwd":
        return {"bytes": int(2 * tq + 2 * tk_seen + stats), "flops": int(4 * case["dh"] * pairs)}
    return {"bytes": int(5 * tq + 4 * tk_seen + 2 * tk + 2 * stats), "flops": int(14 * case["dh"] * pairs)}


# ---- the operators' definitions in 64 bits, gradients by differentiation of the forward ----

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        x, gamma, beta = (st[n].double().requires_grad_() for n in ("x", "gamma", "beta"))
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = torch.rsqrt(var + 1e-5)
        y = torch.addcmul(beta, (x - mean[:, None]) * rstd[:, None], gamma)
        out = {"y": y.detach()}
        if case["way"] == "train":
            out["dx"], out["dgamma"], out["dbeta"] = torch.autograd.grad(y, (x, gamma, beta), st["dy"].double())
            out["mean"], out["rstd"] = mean.detach(), rstd.detach()
        return out
    if case["op"] == "rotary":
        out = {}
        for name in "qk":
            x = st[name].double()
            y = x.clone()
            p, total = 0, sum(st["pairs"])
            for axis, n in enumerate(st["pairs"]):
                for _ in range(n):
                    a, b = (2 * p, 2 * p + 1) if case["interleaved"] else (p, p + total)
                    angle = st["pos"][:, :, axis].double() * st["inv_freq"][p].double()
                    turn = torch.polar(torch.ones_like(angle), -angle if case["way"] == "bwd" else angle)[:, :, None]
                    z = torch.complex(x[..., a], x[..., b]) * turn
                    y[..., a], y[..., b] = z.real, z.imag
                    p += 1
            out[name] = y
        return out
    seg, keys = segments(case)
    heads, kv_heads, dh, train = case["heads"], case["kv_heads"], case["dh"], case["way"] == "train"
    slope = st["slope"].double().requires_grad_() if case["bias"] else None
    parts = {n: [] for n in ("o", "lse", "dq", "dk", "dv")}
    dslope = 0.0
    for b in range(case["batch"]):
        q, k, v = (st[n][b].double().permute(1, 0, 2).reshape(kv_heads, -1, st[n].shape[1], dh).contiguous().requires_grad_() for n in "qkv")
        rows_o, rows_l = [], []
        for i in range(3):
            qs = slice(sum(seg[:i]), sum(seg[:i + 1]))
            at = [torch.arange(sum(keys[:j]), sum(keys[:j]) + (int(st["valid_len"][b, j]) if case["pad"] == "valid_len" else keys[j]))
                  for j in range(3) if MASKS[case["mask"]] >> (3 * i + j) & 1]
            at = torch.cat(at).cuda() if at else torch.zeros(0, dtype=torch.long, device="cuda")
            if case["pad"] == "key_pad":
                at = at[st["key_pad"][b, at] == 0]
            score = q[:, :, qs] @ k[:, :, at].transpose(2, 3) / math.sqrt(dh)
            if case["cap"]:
                score = case["cap"] * torch.tanh(score / case["cap"])
            gap = st["k_pos"][b, at].double() - st["q_pos"][b, qs, None].double()
            if case["bias"]:
                score = score - slope.view(kv_heads, -1, 1, 1) * gap.abs()
            seen = torch.ones_like(gap, dtype=torch.bool)
            if case["docs"]:
                seen &= ~(st["k_doc"][b, at] - st["q_doc"][b, qs, None]).bool()
            if case["causal"]:
                ahead = gap > 0
                if case["prefix"]:
                    ahead &= st["k_pos"][b, at] >= st["prefix"][b]
                seen &= ~ahead
            some = seen.any(1)
            score = score + torch.where(seen | ~some[:, None], 0.0, -math.inf)
            weight = torch.softmax(score, 3) * some[:, None] if at.numel() else score
            rows_o.append(weight @ v[:, :, at])
            lse = torch.logsumexp(score, 3) if at.numel() else torch.full(score.shape[:3], -math.inf, device="cuda", dtype=torch.float64)
            rows_l.append(torch.where(some, lse, -math.inf).detach())
        o = torch.cat(rows_o, 2)
        back = lambda x, h: x.reshape(h, -1, dh).permute(1, 0, 2).detach()  # noqa: E731
        parts["o"].append(back(o, heads))
        parts["lse"].append(torch.cat(rows_l, 2).reshape(heads, -1))
        if train:
            do = st["do"][b].double().permute(1, 0, 2).reshape(o.shape)
            grads = torch.autograd.grad(o, (q, k, v) + ((slope,) if case["bias"] else ()), do)
            for n, x, h in zip(("dq", "dk", "dv"), grads, (heads, kv_heads, kv_heads)):
                parts[n].append(back(x, h))
            if case["bias"]:
                dslope = dslope + grads[3]
    out = {n: torch.stack(x) for n, x in parts.items() if x}
    if train and case["bias"]:
        out["dslope"] = dslope
    return out
