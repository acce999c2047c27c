"""The definitions of head norms with rotation and of causal attention in 64 bits on the CPU, and
the error bounds that the tests of the kernels allow.

Bounds (u, EPS as in layer_oracle; a rounding to the operands' type T costs u of the value).
Attention, 16-bit types: scores are sums of D products in 32 bits, off by dS = (D + 4) EPS scale
|q| . |k|, and so is their exponential, relatively, with 8 EPS for the exponential itself. P = e^(S -
lse) and dS are rounded to T before the products with v, dy, k and q (u each; half as low as 2^-25
in its own scale), and those sums of n terms lose at most (n + 16) EPS of their terms' magnitudes.
Floats round neither (u = 2^-24). The gradient takes y as rounded to T, so that dy . y is off by w = |dy| . |y's
error|. Floats feel that as it is; for 16-bit types it is taken back by what a row of dS sums to, so that w is felt
through the rounding of P alone (3 u w), and the row's own errors once more.
"""
import math

import torch

import layer_oracle as lo

EPS = lo.EPS


# ------------------------------------------------------------------- norms and rotation
def _pairs(rotary, interleaved):
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def turn(x, positions, rotary, base, interleaved, sign=1.0):
    """x [tokens, heads, D] double, turned."""
    a = positions.double()[:, None] * torch.tensor([base ** (-2.0 * i / rotary) for i in range(rotary // 2)],
                                                        dtype=torch.float64)
    c, s = torch.cos(a)[:, None], sign * torch.sin(a)[:, None]
    e, f = _pairs(rotary, interleaved)
    y = x.clone()
    y[..., e] = x[..., e] * c - x[..., f] * s
    y[..., f] = x[..., f] * c + x[..., e] * s
    return y


def rotary_forward(x, w, positions, rotary, base, interleaved, norm, eps):
    n = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) if norm else x
    return turn(n * w, positions, rotary, base, interleaved)


def rotary_grad(dy, x, w, positions, rotary, base, interleaved, norm, eps):
    """dx, dw"""
    g = turn(dy, positions, rotary, base, interleaved, -1.0)
    rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) if norm else torch.ones_like(x[..., :1])
    n = x * rstd
    u = g * w
    dx = rstd * (u - (n * (u * n).mean(-1, keepdim=True) if norm else 0))
    return dx, (g * n).sum((0, 1))


def rotary_bounds(x, w, dy, positions, rotary, interleaved, norm, eps, base):
    """Of y, dx, dw: OPS operations a statistic; an element turned sums two products, whose angle is off
    by 2^-24 half turns and the binary fraction's and the definition's own 2^-52 |position|."""
    angle = 4 * EPS + positions.abs().double()[:, None, None] * 2.0 ** -50
    rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) if norm else torch.ones_like(x[..., :1])
    n = x.abs() * rstd
    wide = lambda t: t + _other(t, rotary, interleaved)
    y = wide(n * w.abs()) * (lo.OPS * EPS + angle)
    dx = dw = None
    if dy is not None:
        g = wide(dy.abs())
        u = g * w.abs()
        each = u + (n * (u * n).mean(-1, keepdim=True) if norm else 0)
        dx = rstd * (each * (2 * lo.OPS * EPS + (x.shape[-1] * EPS if norm else 0)) + angle * each)
        terms = x.shape[0] * x.shape[1]
        dw = ((g * n) * (lo.OPS * EPS + angle)).sum((0, 1)) + terms * EPS * (g * n).sum((0, 1))
    return y, dx, dw


def _other(t, rotary, interleaved):
    e, f = _pairs(rotary, interleaved)
    o = torch.zeros_like(t)
    o[..., e] = t[..., f]
    o[..., f] = t[..., e]
    return o


# ------------------------------------------------------------------------- attention
def attention(q, k, v, offsets, scale, dy=None, y_used=None, dtype=torch.float32):
    """name -> (value, bound) of y, lse and, with dy, of dq, dk, dv; q, k, v, dy double on any
    device. y_used: the y that the gradient's call takes (its own exact one if None)."""
    T, H, D = q.shape
    G = k.shape[1]
    u = lo.UNIT[dtype]
    half = dtype is torch.float16
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=q.device)
    val = {"y": z(T, H, D), "lse": z(H, T)}
    if dy is not None:
        val.update(dq=z(T, H, D), dk=z(T, G, D), dv=z(T, G, D))
    bound = {n: torch.zeros_like(t) for n, t in val.items()}
    o = lo.clean_offsets(offsets, T)
    big = 0.0
    if dy is not None and half and o[-1] > o[0]:
        rows = slice(o[0], o[-1])
        big = float(dy[rows].abs().max() * v[rows].abs().max()) * D
    for a, b in zip(o[:-1], o[1:]):
        if a == b:
            continue
        n = b - a
        later = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
        sum_eps = (n + 16) * EPS
        for h in range(H):
            g = h // (H // G)
            Q, K, V = q[a:b, h], k[a:b, g], v[a:b, g]
            s = (Q @ K.t() * scale).masked_fill(later, -math.inf)
            off = (D + 4) * EPS * abs(scale) * (Q.abs() @ K.abs().t())
            off = off.masked_fill(later, 0.0)
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[:, None])
            worst = off.amax(-1)  # of a row's scores: also its sum's relative error
            e = off + worst[:, None] + 16 * EPS + sum_eps  # of p, relatively
            e = e + EPS * (lse.abs()[:, None] + s.masked_fill(later, 0.0).abs())
            Y = p @ V
            val["y"][a:b, h], val["lse"][h, a:b] = Y, lse
            tiny = 2.0 ** -25 if half else 0.0
            bound["y"][a:b, h] = (p * (e + u + sum_eps)) @ V.abs() + tiny * ((~later).double() @ V.abs())
            bound["lse"][h, a:b] = worst + 8 * EPS * (1 + lse.abs()) + sum_eps
            if dy is None:
                continue
            d = dy[a:b, h]
            used = Y if y_used is None else y_used[a:b, h]
            dp = d @ V.t()
            delta = (d * Y).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            rounded = (d.abs() * (used - Y).abs()).sum(-1, keepdim=True)
            wrong = (D + 4) * EPS * (d.abs() @ V.abs().t()) \
                + (D + 4) * EPS * (d.abs() * Y.abs()).sum(-1, keepdim=True) + EPS * (dp.abs() + delta.abs())
            if dtype is torch.float32:
                wrong = wrong + rounded
            else:
                row = ((ds.abs() + p * rounded) * (e + sum_eps) + p * wrong).sum(-1, keepdim=True)
                wrong = wrong + (3 * u + tiny) * rounded + row
            ds_off = ds.abs() * (e + u) + p * wrong * (1 + e) + (tiny * big * 2.0 ** -13 * (~later).double() if half else 0.0)
            val["dv"][a:b, g] += p.t() @ d
            val["dq"][a:b, h] = scale * ds @ K
            val["dk"][a:b, g] += scale * ds.t() @ Q
            more = sum_eps * (H // G)
            bound["dv"][a:b, g] += (p * (e + u + more)).t() @ d.abs() + tiny * (~later).double().t() @ d.abs()
            bound["dq"][a:b, h] = abs(scale) * (ds_off + ds.abs() * sum_eps) @ K.abs()
            bound["dk"][a:b, g] += abs(scale) * (ds_off + ds.abs() * more).t() @ Q.abs()
    return {n: (val[n].cpu(), bound[n].cpu()) for n in val}
