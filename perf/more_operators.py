"""Performance cases of the attention half of a block (``paper_2101_07968_gb300.layers``),
whose forward and backward times are compute costs of a schedule as the experts' are.

Operators (``op``):

* ``rotary``     norms of queries and keys for each head and the rotation by position, in one
  pass over both: ``fwd``, and ``bwd`` their gradient with that of the norms' weights;
* ``attention``  causal attention of packed sequences, heads that share keys and values: ``fwd``,
  and ``train`` the forward pass with the gradient after it.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BASE, EPS = 10000.0, 1e-6


def _rotary(name, direction, dtype, tokens, heads, kv, D, rotary, interleaved=False, weights=True, first=0):
    return {"name": name, "op": "rotary", "dir": direction, "dtype": dtype, "tokens": tokens,
            "heads": heads, "kv": kv, "D": D, "rotary": rotary, "interleaved": interleaved,
            "weights": weights, "first": first}


def _attention(name, direction, dtype, tokens, sequences, spread, heads, kv, D, pad=0):
    return {"name": name, "op": "attention", "dir": direction, "dtype": dtype, "tokens": tokens,
            "sequences": sequences, "spread": spread, "heads": heads, "kv": kv, "D": D, "pad": pad}


def listed():
    return [
        # one token's queries and keys: latency
        _rotary("rotary_token", "fwd", "bf16", 1, 16, 4, 128, 128),
        # a training batch's, as slices of one projection's output
        _rotary("rotary_train", "fwd", "bf16", 32768, 32, 8, 128, 128),
        # its gradient
        _rotary("rotary_grad", "bwd", "bf16", 32768, 32, 8, 128, 128),
        # part of each head rotated, neighbours in pairs, an odd number of tokens far along
        _rotary("rotary_part", "bwd", "fp16", 16381, 16, 16, 80, 32, True, True, 500000),
        # odd-sized heads in floats, without weights
        _rotary("rotary_odd", "fwd", "fp32", 2049, 7, 1, 65, 64, False, False),
        # two prompts of a few tokens: latency
        _attention("attention_short", "fwd", "bf16", 9, 2, 0.5, 16, 4, 128),
        # a batch of prompts of many lengths, with spare rows at the buffer's end
        _attention("attention_packed", "fwd", "bf16", 16384, 48, 1.0, 16, 4, 128, 100),
        # one long prompt
        _attention("attention_long", "fwd", "bf16", 16384, 1, 0.0, 32, 8, 128),
        # a training step's packed batch, forward and gradient
        _attention("attention_train", "train", "bf16", 32768, 14, 0.6, 32, 8, 128),
        # long sequences, smaller heads, none shared
        _attention("attention_heads", "train", "fp16", 16384, 2, 0.2, 16, 16, 64),
        # sizes that are multiples of nothing
        _attention("attention_odd", "train", "fp16", 3001, 7, 0.8, 6, 2, 75, 3),
        # floats
        _attention("attention_float", "train", "fp32", 2000, 3, 0.5, 8, 2, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: from one token to 32,768, one sequence to one of a few tokens
    each, heads of up to 128 elements, most of them multiples of eight and some of nothing."""
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp16", "fp16", "fp32"])
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    heads = kv * rng.choice([n for n in (1, 2, 3, 4, 8) if n * kv <= 32])
    D = rng.choice([64, 128, 128, 128, 8 * rng.randint(4, 16), rng.randint(16, 128)])
    tokens = _log(rng, 1, 32768)
    if rng.random() < 0.4:
        c = _rotary("", rng.choice(["fwd", "bwd"]), dtype, tokens, heads, kv, D,
                    rng.choice([D // 2 * 2, D // 2 * 2, max(2, D // 4 * 2)]), rng.random() < 0.3,
                    rng.random() < 0.8, rng.choice([0, 0, 100000]))
    else:
        direction = rng.choice(["fwd", "train"])
        sequences = min(tokens, _log(rng, 1, max(1, tokens // 16)))
        spread = rng.choice([0.0, 0.5, 1.0])
        # floats have no tensor cores' rate, and rows off 16 bytes cost copies: smaller ones
        top = 1.5e12 if dtype != "fp32" else 6e10
        while True:
            c = _attention("", direction, dtype, tokens, sequences, spread, heads, kv, D,
                           rng.choice([0, 0, tokens // 20]))
            if work(c)["flops"] <= top:
                break
            tokens = tokens * 3 // 4
            sequences = min(tokens, sequences)
    del c["name"]
    return c


# ----------------------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the packed sequences, log-normal: the same for every seed, longest first; each
    has a token at least, and they fill all rows but the `pad` last."""
    n, used = case["sequences"], case["tokens"] - case["pad"]
    n = max(1, min(n, used))
    u = (np.arange(n) + 0.5) / n
    share = np.exp(-case["spread"] * _normal_quantile(u))
    cut = np.floor(np.cumsum(share) / share.sum() * (used - n) + 0.5).astype(np.int64)
    return np.diff(np.concatenate([[0], cut])) + 1


def _normal_quantile(u):
    """Logistic stand-in for the normal distribution's quantiles (within 0.1 in the bulk)."""
    return np.log(u / (1 - u)) / 1.702


def _offsets(case, seed):
    lengths = _lengths(case)
    np.random.default_rng([seed, 5]).shuffle(lengths)
    return [0] + [int(v) for v in np.cumsum(lengths)]


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        t = torch.empty(shape, dtype=dtype, device="cuda")
        t.normal_(shift, scale, generator=g)
        return t

    T, H, G, D = case["tokens"], case["heads"], case["kv"], case["D"]
    s = {"case": case}
    # queries, keys and values come from one projection, as neighbours in a row
    fused = normal(T, H + 2 * G, D, scale=1.2)
    if case["op"] == "rotary":
        s["q"], s["k"] = fused[:, :H], fused[:, H:H + G]
        # each sequence counts from `first` on
        n = min(T, 2048)
        s["positions"] = torch.arange(T, dtype=torch.int64, device="cuda") % n + case["first"]
        s["w_q"] = normal(D, scale=0.1, shift=1.0) if case["weights"] else None
        s["w_k"] = normal(D, scale=0.1, shift=1.0) if case["weights"] else None
        if case["dir"] == "bwd":
            s["dq"], s["dk"] = normal(T, H, D), normal(T, G, D)
        return s
    s["q"], s["k"] = normal(T, H, D, scale=1.3), normal(T, G, D, scale=1.3)
    s["v"] = fused[:, H + G:]
    s["host_offsets"] = _offsets(case, seed)
    s["offsets"] = torch.tensor(s["host_offsets"], dtype=torch.int64, device="cuda")
    s["scale"] = D ** -0.5
    if case["dir"] == "train":
        s["do"] = normal(T, H, D)
    return s


# ------------------------------------------------------------------- the plain forms
def _angles(positions, rotary):
    """cos and sin [tokens, 1, rotary / 2], the angles in 64 bits."""
    i = torch.arange(rotary // 2, dtype=torch.float64, device=positions.device)
    a = positions.double()[:, None] * torch.exp(i * (-2.0 * math.log(BASE) / rotary))
    a = torch.remainder(a, 2 * math.pi).float()[:, None, :]
    return torch.cos(a), torch.sin(a)


def _halves(x, rotary, interleaved):
    if interleaved:
        return x[..., 0:rotary:2], x[..., 1:rotary:2]
    return x[..., :rotary // 2], x[..., rotary // 2:rotary]


def _rotate(x, cos, sin, rotary, interleaved):
    a, b = _halves(x, rotary, interleaved)
    y = x.clone()
    ya, yb = _halves(y, rotary, interleaved)
    ya.copy_(a * cos - b * sin)
    yb.copy_(b * cos + a * sin)
    return y


def _plain_rotary(s):
    c, out = s["case"], {}
    dtype = DTYPES[c["dtype"]]
    cos, sin = _angles(s["positions"], c["rotary"])
    for name in ("q", "k"):
        x = s[name].float()
        w = s["w_" + name].float() if s["w_" + name] is not None else torch.ones(c["D"], device="cuda")
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * rstd
        if c["dir"] == "fwd":
            out[name] = _rotate(n * w, cos, sin, c["rotary"], c["interleaved"]).to(dtype)
            continue
        g = _rotate(s["d" + name].float(), cos, -sin, c["rotary"], c["interleaved"])
        u = g * w
        out["d" + name] = (rstd * (u - n * (u * n).mean(-1, keepdim=True))).to(dtype)
        if s["w_" + name] is not None:
            out["dw_" + name] = (g * n).sum((0, 1))
    return out


def _chunks(lo, hi, heads, most=1 << 28):
    """Row ranges of a sequence whose scores [heads, rows, keys] hold up to `most` elements."""
    n = max(1, min(hi - lo, most // (heads * (hi - lo))))
    for a in range(lo, hi, n):
        yield a, min(a + n, hi)


def _plain_attention(s):
    c, o = s["case"], s["host_offsets"]
    dtype, H, G = DTYPES[c["dtype"]], c["heads"], c["kv"]
    train = c["dir"] == "train"
    q = s["q"].float().transpose(0, 1)
    k, v = (s[n].float().transpose(0, 1).repeat_interleave(H // G, 0) for n in ("k", "v"))
    y = torch.zeros_like(q)
    lse = torch.zeros(q.shape[:2], device="cuda")
    if train:
        do = s["do"].float().transpose(0, 1)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for lo, hi in zip(o[:-1], o[1:]):
        for a, b in _chunks(lo, hi, H):
            kk, vv = k[:, lo:b], v[:, lo:b]
            later = torch.arange(lo, b, device="cuda")[None, :] > torch.arange(a, b, device="cuda")[:, None]
            p = (q[:, a:b] @ kk.transpose(1, 2)).mul_(s["scale"]).masked_fill_(later, -math.inf)
            top = p.amax(-1, keepdim=True)
            p = p.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            p = p.div_(total)
            lse[:, a:b] = (top + torch.log(total))[..., 0]
            y[:, a:b] = p @ vv
            if train:
                d = do[:, a:b]
                dv[:, lo:b] += p.transpose(1, 2) @ d
                ds = (d @ vv.transpose(1, 2)).sub_((d * y[:, a:b]).sum(-1, keepdim=True)).mul_(p)
                dq[:, a:b] = (ds @ kk) * s["scale"]
                dk[:, lo:b] += (ds.transpose(1, 2) @ q[:, a:b]) * s["scale"]
    out = {"o": y.transpose(0, 1).to(dtype).contiguous(), "lse": lse}
    if train:
        out["dq"] = dq.transpose(0, 1).to(dtype).contiguous()
        for name, t in (("dk", dk), ("dv", dv)):
            out[name] = t.view(G, H // G, *t.shape[1:]).sum(1).transpose(0, 1).to(dtype).contiguous()
    return out


def _kernels(s):
    from paper_2101_07968_gb300 import layers as ly
    c = s["case"]
    if c["op"] == "rotary":
        how = dict(w_q=s["w_q"], w_k=s["w_k"], rotary=c["rotary"], base=BASE, interleaved=c["interleaved"], eps=EPS)
        if c["dir"] == "fwd":
            q, k = ly.head_norm_rotary(s["q"], s["k"], s["positions"], **how)
            return {"q": q, "k": k}
        r = ly.head_norm_rotary_grad(s["dq"], s["dk"], s["q"], s["k"], s["positions"], **how)
        return {n: t for n, t in r.items() if t is not None}
    o, lse = ly.attention(s["q"], s["k"], s["v"], s["offsets"], scale=s["scale"])
    out = {"o": o, "lse": lse}
    if c["dir"] == "train":
        out["dq"], out["dk"], out["dv"] = ly.attention_grad(s["do"], s["q"], s["k"], s["v"], o, lse,
                                                            s["offsets"], scale=s["scale"])
    return out


def run(state):
    if own:
        return _kernels(state)
    return _plain_rotary(state) if state["case"]["op"] == "rotary" else _plain_attention(state)


# ----------------------------------------------------------------- the least work
def work(case):
    b, T, D = SIZE[case["dtype"]], case["tokens"], case["D"]
    H, G = case["heads"], case["kv"]
    if case["op"] == "rotary":
        w = 2 * D * b if case["weights"] else 0
        if case["dir"] == "fwd":
            return {"bytes": 2 * T * (H + G) * D * b + 8 * T + w, "flops": 8.0 * T * (H + G) * D}
        return {"bytes": 3 * T * (H + G) * D * b + 8 * T + 5 * w // b, "flops": 16.0 * T * (H + G) * D}
    n = _lengths(case).astype(np.float64)
    pairs = float((n * (n + 1) / 2).sum())
    used = T - case["pad"]
    if case["dir"] == "fwd":
        byte = (used * (H + 2 * G) + T * H) * D * b + 4 * T * H
        return {"bytes": byte, "flops": 4.0 * D * H * pairs}
    # q, k, v, do read; o, lse and the three gradients written
    byte = (used * (2 * H + 2 * G) + T * (2 * H + 2 * G)) * D * b + 4 * T * H
    return {"bytes": byte, "flops": 14.0 * D * H * pairs}


# ------------------------------------------------- the definition, in 64 bits
def _exact_rotary(case, s):
    r, out = case["rotary"], {}
    theta = [BASE ** (-2.0 * i / r) for i in range(r // 2)]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None, None] * torch.tensor(theta, dtype=torch.float64, device="cuda"))
    order = list(range(r))
    order = order[0::2] + order[1::2] if case["interleaved"] else order
    order = torch.tensor(order, device="cuda")

    def turned(x, by):
        z = torch.complex(x[..., order[:r // 2]], x[..., order[r // 2:]]) * by
        y = x.clone()
        y[..., order] = torch.cat([z.real, z.imag], -1)
        return y

    for name in ("q", "k"):
        x = s[name].double()
        w = s["w_" + name].double() if s["w_" + name] is not None else torch.ones(case["D"], dtype=torch.float64,
                                                                                 device="cuda")
        norm = torch.sqrt(x.square().sum(-1, keepdim=True) / case["D"] + EPS)
        if case["dir"] == "fwd":
            out[name] = turned(x / norm * w, turn)
            continue
        g = turned(s["d" + name].double(), turn.conj())
        u = g * w
        out["d" + name] = u / norm - x * (u * x).sum(-1, keepdim=True) / (case["D"] * norm ** 3)
        if s["w_" + name] is not None:
            out["dw_" + name] = torch.einsum("thd,thd->d", g, x / norm)
    return out


def exact(case, seed):
    if case["op"] == "attention":
        n = _lengths(case).astype(np.float64)
        units = 2.0 if case["dir"] == "fwd" else 6.0
        if units * 2 * case["D"] * case["heads"] * float((n * n).sum()) > 8e12:
            return None
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    T, H, G, D = case["tokens"], case["heads"], case["kv"], case["D"]

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")
    out = {"o": zeros(T, H, D), "lse": zeros(H, T)}
    train = case["dir"] == "train"
    if train:
        out.update(dq=zeros(T, H, D), dk=zeros(T, G, D), dv=zeros(T, G, D))
    o = s["host_offsets"]
    for lo, hi in zip(o[:-1], o[1:]):
        step = max(1, min(hi - lo, (1 << 27) // (hi - lo)))
        for h in range(H):
            g = h * G // H
            q, k, v = s["q"][lo:hi, h].double(), s["k"][lo:hi, g].double(), s["v"][lo:hi, g].double()
            for a in range(0, hi - lo, step):
                b = min(a + step, hi - lo)
                sc = q[a:b] @ k[:b].t() * s["scale"]
                sc += torch.full((b - a, b), -math.inf, dtype=torch.float64, device="cuda").triu(a + 1)
                z = torch.logsumexp(sc, -1)
                out["lse"][h, lo + a:lo + b] = z
                p = torch.exp(sc - z[:, None])
                y = p @ v[:b]
                out["o"][lo + a:lo + b, h] = y
                if train:
                    d = s["do"][lo + a:lo + b, h].double()
                    ds = p * (d @ v[:b].t() - (d * y).sum(-1)[:, None]) * s["scale"]
                    out["dv"][lo:lo + b, g] += p.t() @ d
                    out["dq"][lo + a:lo + b, h] = ds @ k[:b]
                    out["dk"][lo:lo + b, g] += ds.t() @ q[a:b]
    return out
