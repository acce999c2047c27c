"""The layer operators' definitions in 64 bits on the CPU, and the error bounds that the
tests of the kernels allow.

Bounds. u is the unit roundoff of an output's type, 2^-p for p significant bits (bfloat16 8,
half 11 with half a spacing of 2^-25 below its normal range, float 24): one rounding costs
u |exact|. Arithmetic in
32 bits costs at most EPS = 2^-23 per operation (twice the unit roundoff, which also covers
sums that a tensor core truncates). A sum of n products then errs by at most (n + 2) EPS
sum |a b|. Longer expressions are bounded with the row's largest magnitudes, at OPS = 64
operations a row statistic and its use (16 sequential additions, ten levels of a tree, a
reciprocal root of 2 ulp, and the handful of products around it).
"""
import math

import numpy as np
import torch

EPS = 2.0 ** -23
OPS = 64
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}


def d64(t):
    return None if t is None else t.detach().cpu().double()


def assert_within(got, exact, bound, what):
    """got (an output tensor) within one rounding of exact +- bound, elementwise."""
    g = d64(got)
    assert g.shape == exact.shape, (what, g.shape, exact.shape)
    u = UNIT[got.dtype]
    allowed = u * (exact.abs() + bound) + bound + TINY[got.dtype] + 1e-300
    assert bool(torch.isfinite(g).all()), f"{what}: not finite"
    bad = (g - exact).abs() > allowed
    if bool(bad.any()):
        i = int(((g - exact).abs() / allowed).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst at {i}: "
                             f"{g.flatten()[i].item()} for {exact.flatten()[i].item()} "
                             f"+- {allowed.flatten()[i].item()}")


# ------------------------------------------------------------------- expert products
def clean_offsets(offsets, rows):
    out, top = [], 0
    for v in offsets:
        top = max(top, min(max(int(v), 0), rows))
        out.append(top)
    return out


def expert_products(x, w, dy, offsets, rows):
    """(y, dx, dw) and their bounds' sums of magnitudes; x, w, dy double or None."""
    o = clean_offsets(offsets, rows)
    E = len(o) - 1
    res = {}

    def put(name, shape, f):
        val, mag, n = torch.zeros(shape).double(), torch.zeros(shape).double(), torch.zeros(shape).double()
        for e in range(E):
            lo, hi = o[e], o[e + 1]
            a, b, terms = f(e, lo, hi)
            where = e if name == "dw" else slice(lo, hi)
            val[where], mag[where], n[where] = a @ b, a.abs() @ b.abs(), terms
        res[name] = (val, (n + 2) * EPS * mag)

    if x is not None and w is not None:
        put("y", (rows, w.shape[1]), lambda e, lo, hi: (x[lo:hi], w[e].t(), w.shape[2]))
    if dy is not None and w is not None:
        put("dx", (rows, w.shape[2]), lambda e, lo, hi: (dy[lo:hi], w[e], w.shape[1]))
    if x is not None and dy is not None:
        put("dw", (E, dy.shape[1], x.shape[1]), lambda e, lo, hi: (dy[lo:hi].t(), x[lo:hi], hi - lo))
    return res


# ------------------------------------------------------------------------ gated unit
def gated(h, act):
    F = h.shape[1] // 2
    g, u = h[:, :F], h[:, F:]
    if act == "silu":
        s = torch.sigmoid(g)
        a, slope = g * s, s + g * s * (1 - s)
    else:
        cdf = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))  # keeps its digits in the tail
        a, slope = g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return a * u, a, slope, g, u


# --------------------------------------------------------------------------- dropout
def splitmix(seed, n):
    """SplitMix64's outputs number n (Steele, Lea, Flood 2014) for an array of numbers."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + np.asarray(n, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def keep_factor(rows, cols, p, seed, offset):
    """[rows, cols] double: 0 where dropped, 1 / (1 - q) where kept."""
    t = int(math.floor(p * 65536 + 0.5))
    r, c = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    n = offset + r * ((cols + 3) // 4) + c // 4 + 1
    field = (splitmix(seed, n) >> (16 * (c % 4)).astype(np.uint64)) & np.uint64(0xFFFF)
    f = np.where(field.astype(np.int64) >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)
    return torch.from_numpy(f)


# ----------------------------------------------------------------------- block norms
def norm_stats(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    var = ((v - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    return (v - mean) * rstd, rstd


def norm_forward(x, f, gate, post, pre, alpha, kind, eps, keep):
    """y, h from double operands; gate per row, keep a factor per element."""
    y = alpha * x + gate * keep * post * norm_stats(f, kind, eps)[0] if f is not None else x
    return y, pre * norm_stats(y, kind, eps)[0]


def rowmax(v):
    return v.abs().max(1, keepdim=True).values


def norm_forward_bounds(x, f, gate, post, pre, alpha, kind, eps, keep):
    y, _ = norm_forward(x, f, gate, post, pre, alpha, kind, eps, keep)
    by = torch.zeros_like(y)
    if f is not None:
        _, fr = norm_stats(f, kind, eps)
        by = OPS * EPS * ((alpha * x).abs() + (gate * keep * post).abs() * fr * (f.abs() + rowmax(f)))
    yhat, yr = norm_stats(y, kind, eps)
    bh = pre.abs() * yr * (OPS * EPS * (y.abs() + rowmax(y)) * (1 + yhat.abs())
                           + rowmax(by) * (2 + yhat.abs()))
    return by, bh


def norm_backward(dy, dh, y, f, gate, post, pre, alpha, kind, eps, keep):
    """Per-row pieces of the gradients and their bounds: t, df, and the terms that dgate,
    dw_post and dw_pre add over rows."""
    def back(d, hat, r):
        out = d - hat * (d * hat).mean(1, keepdim=True)
        return r * (out - (out.mean(1, keepdim=True) if kind == "layer" else 0.0))

    def spread(hat):
        return 1 + (1 + hat.abs()) * rowmax(hat)

    t, bt = dy.clone(), OPS * EPS * dy.abs()
    out = {}
    if dh is not None:
        yhat, yr = norm_stats(y, kind, eps)
        t = t + back(dh * pre, yhat, yr)
        ey = OPS * EPS * yr * (y.abs() + rowmax(y)) * (1 + yhat.abs())  # error of yhat
        bt = bt + yr * rowmax(dh * pre) * (OPS * EPS * spread(yhat) + 2 * rowmax(ey) * (1 + rowmax(yhat)))
        out["w_pre"] = (dh * yhat, dh.abs() * (ey + OPS * EPS * yhat.abs()))
    out["t"] = (t, bt)
    if f is not None:
        fhat, fr = norm_stats(f, kind, eps)
        ef = OPS * EPS * fr * (f.abs() + rowmax(f)) * (1 + fhat.abs())
        u, bu = t * gate * keep, bt * (gate * keep).abs()
        out["df"] = (back(u * post, fhat, fr),
                     fr * (rowmax(bu * post) * spread(fhat)
                           + rowmax(u * post) * (OPS * EPS * spread(fhat)
                                                 + 2 * rowmax(ef) * (1 + rowmax(fhat)))))
        out["gate"] = (t * keep * post * fhat,
                       (keep * post).abs() * (bt * fhat.abs() + t.abs() * (ef + OPS * EPS * fhat.abs())))
        out["w_post"] = (u * fhat, bu * fhat.abs() + u.abs() * (ef + OPS * EPS * fhat.abs()))
    return out


def add_rows(pair, groups=None):
    """Sum over rows (or over consecutive groups of `groups` rows) of (value, bound)."""
    v, b = pair
    R = v.shape[0]
    G = 1 if groups is None else -(-R // groups)
    step = R if groups is None else groups
    vs, bs = [], []
    for i in range(G):
        a, c = v[i * step:(i + 1) * step], b[i * step:(i + 1) * step]
        vs.append(a.sum(0))
        bs.append(c.sum(0) + (a.shape[0] + 2) * EPS * a.abs().sum(0))
    return torch.stack(vs), torch.stack(bs)
