"""Layer norm, rotary positions and the attention core in fp64 numpy, from their definitions (include/imattn.h), with elementwise
bounds on what the GPU's arithmetic may differ by.

Bounds.  u = 2^-24 is half a step of fp32, `half` half a step of the tensors' type relative to the value (2^-8 for bf16,
2^-24 for fp32).  A sum of n products in fp32 is off by at most (n + 2) u times the sum of the products' magnitudes, in any
order.  Numbers below TINY = 2^-126, the smallest normal one, may be flushed to 0 wherever they occur: each probability, dS, product and
sum may be off by TINY more.  bf16 operands of the second products (probabilities, dS) are rounded once, by at most 2^-8 of each.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def layernorm(x, gamma, beta, eps, dy=None):
    """x [R, d] -> dict y, mean, rstd and, given dy, dx, dgamma, dbeta."""
    x = np.asarray(x, np.float64)
    d = x.shape[1]
    g = np.ones(d) if gamma is None else np.asarray(gamma, np.float64)
    b = np.zeros(d) if beta is None else np.asarray(beta, np.float64)
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    xhat = (x - mean) * rstd
    out = {"y": xhat * g + b, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if dy is not None:
        dy = np.asarray(dy, np.float64)
        w = dy * g
        out["dx"] = rstd * (w - w.mean(1, keepdims=True) - xhat * (w * xhat).mean(1, keepdims=True))
        out["dgamma"], out["dbeta"] = (dy * xhat).sum(0), dy.sum(0)
    return out


def layernorm_bounds(x, gamma, beta, eps, dy, dtype):
    """Elementwise bounds of layernorm's outputs as the GPU computes them (sums in fp32, one rounding of the result)."""
    x = np.asarray(x, np.float64)
    r, d = x.shape
    g = np.ones(d) if gamma is None else np.asarray(gamma, np.float64)
    b = np.zeros(d) if beta is None else np.asarray(beta, np.float64)
    ref = layernorm(x, gamma, beta, eps, dy)
    h = half_step(dtype)
    mean, rstd = ref["mean"][:, None], ref["rstd"][:, None]
    xhat = (x - mean) * rstd
    e_mean = (d + 3) * U * np.abs(x).mean(1, keepdims=True)
    e_c = e_mean + U * np.abs(x - mean)                       # of a centred value
    # of rstd, relative: half of the variance's error; its first-order term in e_mean cancels (centred values sum to 0)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    e_r = 0.5 * rstd ** 2 * ((d + 6) * U * var + e_mean ** 2 + 2 * U * np.abs(x - mean).mean(1, keepdims=True) * np.sqrt(var)) + 8 * U
    e_xhat = e_c * rstd + np.abs(xhat) * (e_r + 2 * U)
    out = {"mean": e_mean[:, 0], "rstd": (rstd * e_r)[:, 0],
           "y": e_xhat * np.abs(g) + 3 * U * (np.abs(xhat * g) + np.abs(b)) + h * np.abs(ref["y"])}
    if dy is not None:
        dy = np.asarray(dy, np.float64)
        w = np.abs(dy * g)
        m1, m2 = w.mean(1, keepdims=True), (w * np.abs(xhat)).mean(1, keepdims=True)
        e_m1 = (d + 3) * U * m1
        e_m2 = (d + 4) * U * m2 + (w * e_xhat).mean(1, keepdims=True)
        out["dx"] = rstd * (3 * U * w + e_m1 + np.abs(xhat) * e_m2 + e_xhat * m2 + 3 * U * np.abs(xhat) * m2) + np.abs(ref["dx"]) * (e_r + 3 * U + h)
        out["dgamma"] = (r + 3) * U * (np.abs(dy * xhat)).sum(0) + (np.abs(dy) * e_xhat).sum(0)
        out["dbeta"] = (r + 3) * U * np.abs(dy).sum(0)
    return out


def rotary(x, pos, inv_freq, pairs, interleaved=False, inverse=False):
    """x [B, T, H, dh], pos [B, T, axes] -> turned x."""
    x = np.asarray(x, np.float64)
    axis = np.repeat(np.arange(len(pairs)), pairs)
    n = len(axis)
    angle = np.asarray(pos, np.float64)[..., axis] * np.asarray(inv_freq, np.float64)
    c, s = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None] * (-1 if inverse else 1)
    i0, i1 = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y = x.copy()
    y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
    return y


def visible(B, q_len, k_len, live_mask, valid_len=None, key_pad=None, q_pos=None, k_pos=None, causal=False, prefix=None, q_doc=None, k_doc=None):
    """[B, Tq, Tk] booleans, pair by pair as the definition says it."""
    n = len(q_len)
    seen = np.zeros((B, sum(q_len), sum(k_len)), bool)
    qo, ko = np.concatenate([[0], np.cumsum(q_len)]).astype(int), np.concatenate([[0], np.cumsum(k_len)]).astype(int)
    for b in range(B):
        for i in range(n):
            for j in range(n):
                if not live_mask >> (i * n + j) & 1:
                    continue
                stop = ko[j] + (k_len[j] if valid_len is None else int(np.clip(valid_len[b][j], 0, k_len[j])))
                seen[b, qo[i]:qo[i + 1], ko[j]:stop] = True
    if key_pad is not None:
        seen &= (np.asarray(key_pad) == 0)[:, None]
    if q_doc is not None:
        seen &= np.asarray(q_doc)[:, :, None] == np.asarray(k_doc)[:, None]
    if causal:
        ok = np.asarray(k_pos)[:, None] <= np.asarray(q_pos)[:, :, None]
        if prefix is not None:
            ok |= (np.asarray(k_pos) < np.asarray(prefix)[:, None])[:, None]
        seen &= ok
    return seen


def core_attention(q, k, v, seen, scale, cap=0.0, slope=None, q_pos=None, k_pos=None, d_o=None, dtype="fp32", second=False):
    """q [B, Tq, H, dh], k, v [B, Tk, Hkv, dh], seen [B, Tq, Tk] -> (values, bounds): o, lse and, given d_o, dq, dk, dv, dslope.

    second: what rounding takes off every visible probability is known to enter the saved output too (rows of a few keys), rounded in its turn:
    2^-16 of a probability is missing there, not 2^-8.
    bounds["dslope_sharp"]: as dslope's bound, but with the part of dS's errors that is the same for a whole row taken back, as the kernel does."""
    q, k, v = (np.asarray(t, np.float64).transpose(0, 2, 1, 3) for t in (q, k, v))
    B, H, Tq, dh = q.shape
    Hkv, Tk = k.shape[1], k.shape[2]
    G = H // Hkv
    # values nobody sees take no part: 0 in their place
    k, v = (np.where(seen.any(1)[:, None, :, None], t, 0.0) for t in (k, v))
    k, v = np.repeat(k, G, 1), np.repeat(v, G, 1)
    hid = ~seen[:, None]
    raw = scale * (q @ k.transpose(0, 1, 3, 2))
    e_s = scale * (dh + 4) * U * (np.abs(q) @ np.abs(k).transpose(0, 1, 3, 2))
    s = raw
    if cap:
        t = np.tanh(raw / cap)
        s = cap * t
        # |tanh'| <= 1; the function itself to 8 u relative in fp32.  bf16 takes the same polynomial and exponential; 2^-21 of the cap is more than
        # they need (a bound in the cap, not in the score), and still far below what bf16 operands leave.
        e_s = e_s + (cap * 2.0 ** -21 if dtype == "bf16" else 8 * U * np.abs(s)) + 4 * U * np.abs(s)
    gap = None
    if slope is not None:
        gap = np.abs(np.asarray(q_pos, np.float64)[:, :, None] - np.asarray(k_pos, np.float64)[:, None])[:, None]
        bias = np.asarray(slope, np.float64)[:, None, None] * gap
        s = s - bias
        e_s = e_s + 4 * U * np.abs(bias)
    e_s = e_s + 6 * U * np.abs(s) + 4 * U
    s = np.where(hid, -np.inf, s)
    e_s = np.where(hid, 0.0, e_s)
    top = s.max(-1, keepdims=True, initial=-np.inf)
    top = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(s - top)
    total = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(total))[..., 0]
    p = p / np.where(total > 0, total, 1.0)
    # relative error of a probability: its own score's and the row's sum's, which averages the scores' errors
    e_row = (p * e_s).sum(-1, keepdims=True)
    e_p = p * (e_s + e_row + (Tk + 8) * U + 6 * U * np.abs(top)) + TINY
    half, hp = half_step(dtype), (2.0 ** -8 if dtype == "bf16" else 0.0)
    av = np.abs(v)
    o = p @ v
    e_o = (e_p + hp * p + (Tk + 4) * U * p) @ av
    out = {"o": o, "lse": lse}
    err = {"o": e_o + half * np.abs(o) + 2 * Tk * TINY, "lse": np.where(np.isfinite(lse), e_row[..., 0] + (Tk + 8) * U + 8 * U * np.abs(np.where(np.isfinite(lse), lse, 0)) + 6 * U * np.abs(top[..., 0]), 0.0)}
    if d_o is not None:
        do = np.asarray(d_o, np.float64).transpose(0, 2, 1, 3)
        vt = v.transpose(0, 1, 3, 2)
        dp, e_dp = do @ vt, (dh + 4) * U * (np.abs(do) @ np.abs(vt))
        delta = (do * o).sum(-1, keepdims=True)
        # the saved o is fp32, but formed from rounded probabilities
        e_saved = (e_p + 2.0 ** -16 * p + 2 * (Tk + 4) * U * p) @ av if second and dtype == "bf16" else e_o
        e_delta = (np.abs(do) * (e_saved + U * np.abs(o))).sum(-1, keepdims=True) + (dh + 4) * U * (np.abs(do) * np.abs(o)).sum(-1, keepdims=True)
        ds = p * (dp - delta)
        e_ds = e_p * np.abs(dp - delta) + p * (e_dp + e_delta) + 4 * U * np.abs(ds)
        if slope is not None:
            out["dslope"] = -(ds * gap).sum((0, 2, 3))
            err["dslope"] = ((e_ds + 4 * U * np.abs(ds)) * gap).sum((0, 2, 3)) + (Tk + 8) * U * (np.abs(ds) * gap).sum((0, 2, 3)) + half_step("fp32") * np.abs(out["dslope"])
            # What the kernel sums is -sum (dS - R P) gap with R = sum dS, the row's sum, and G = sum P gap:  -sum dS gap + R G.  An error x of a
            # pair's dS so counts x (gap - G), and delta's, which is P times one number for the whole row, only by what sum P misses of 1.
            # (Tk + 10) U for each sum, its products and the distance's own rounding.
            g_row = (p * gap).sum(-1, keepdims=True)
            e_one = e_p * np.abs(dp - delta) + p * e_dp + 4 * U * (np.abs(ds) + p * e_delta)
            e_rest = e_delta + e_one.sum(-1, keepdims=True)
            pairs = e_one * np.abs(gap - g_row) + (Tk + 10) * U * (np.abs(ds) + p * e_rest) * (gap + g_row)
            rows_left = e_rest * g_row * (e_p.sum(-1, keepdims=True) + (Tk + 10) * U)
            err["dslope_sharp"] = pairs.sum((0, 2, 3)) + rows_left.sum((0, 2, 3)) + half_step("fp32") * np.abs(out["dslope"])
        if cap:
            f = 1 - t * t
            # the derivative's own error: twice the tangent's, and the score's.  A product of x +- ex and f +- ef is off by at most
            # ex f + |x| ef + ex ef; the last term is what is left where f and x are 0 (scores at the cap, rows of one key), and scale multiplies it
            e_f = 2 * np.where(hid, 0.0, e_s) / cap + 2.0 ** -20
            e_ds = e_ds * (f + e_f) + np.abs(ds) * e_f
            ds = ds * f
        e_ds = e_ds + hp * np.abs(ds) + TINY
        fold = lambda x: x.reshape(B, Hkv, G, Tk, dh).sum(2)  # noqa: E731
        n_k, n_v = scale * (ds.transpose(0, 1, 3, 2) @ q), p.transpose(0, 1, 3, 2) @ do
        out.update(dq=scale * (ds @ k), dk=fold(n_k), dv=fold(n_v))
        aq, ak, ado = np.abs(q), np.abs(k), np.abs(do)
        ads = np.abs(ds)
        err["dq"] = scale * ((e_ds + (Tk + 4) * U * ads) @ ak) + (half + 2 * U) * np.abs(out["dq"])
        err["dk"] = fold(scale * ((e_ds + (G * Tq + 4) * U * ads).transpose(0, 1, 3, 2) @ aq)) + (half + 2 * U) * np.abs(out["dk"])
        err["dq"], err["dk"] = err["dq"] + 2 * (Tk + 1) * TINY, err["dk"] + 2 * (G * Tq + 1) * TINY
        err["dv"] = 2 * (G * Tq + 1) * TINY + fold((e_p + hp * p + (G * Tq + 4) * U * p).transpose(0, 1, 3, 2) @ ado) + half * np.abs(out["dv"])
    rows = lambda n, x: x.transpose(0, 2, 1, 3) if n in ("o", "dq", "dk", "dv") else x  # noqa: E731
    return {n: rows(n, x) for n, x in out.items()}, {n: rows(n, x) for n, x in err.items()}
