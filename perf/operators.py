"""Performance cases of the layer operators (``paper_2101_07968_gb300.layers``): the
training block of a mixture of experts, whose forward and backward times are the compute
costs of a schedule.

Operators (``op``):

* ``experts``  products grouped by expert over ragged rows: ``fwd`` y = W_e x, ``dx`` and
  ``dw`` its gradients, ``grads`` both of them, ``all`` the three;
* ``norm``     the norms after a block and before the next one in one pass, with the block's
  gate, its dropout and the residual's scale: ``fwd`` and ``bwd``;
* ``dropout``  dropout from the counter-based generator, with or without a residual (its
  gradient is the same call);
* ``gated``    the gated unit act(g) * u between the experts' two products: ``fwd``, ``bwd``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def _experts(name, direction, dtype, rows, experts, active, N, K, pad=0, skew=0.5):
    return {"name": name, "op": "experts", "dir": direction, "dtype": dtype, "rows": rows,
            "experts": experts, "active": active, "N": N, "K": K, "pad": pad, "skew": skew}


def _norm(name, direction, dtype, kind, rows, D, per_gate, p, alpha=1.0):
    return {"name": name, "op": "norm", "dir": direction, "dtype": dtype, "kind": kind,
            "rows": rows, "D": D, "per_gate": per_gate, "p": p, "alpha": alpha}


def _dropout(name, dtype, rows, D, p, residual):
    return {"name": name, "op": "dropout", "dtype": dtype, "rows": rows, "D": D, "p": p,
            "residual": residual}


def _gated(name, direction, dtype, act, rows, F):
    return {"name": name, "op": "gated", "dir": direction, "dtype": dtype, "act": act,
            "rows": rows, "F": F}


def listed():
    return [
        # one token through its two experts: latency, and the weights of two experts
        _experts("experts_token", "fwd", "bf16", 2, 16, 2, 4096, 2048),
        # a small batch answered token by token: skewed, some experts without a row
        _experts("experts_decode", "fwd", "fp16", 128, 32, 24, 2048, 2048, skew=1.0),
        # a training step's rows in a buffer with spare capacity at its end
        _experts("experts_train", "fwd", "bf16", 16384, 16, 16, 4096, 2048, pad=700),
        # the largest batch: both gradients
        _experts("experts_grads", "grads", "bf16", 65536, 32, 32, 2048, 4096),
        # sizes that are multiples of nothing, all three products
        _experts("experts_odd", "all", "bf16", 1234, 7, 6, 1001, 515, pad=3),
        # one token between two blocks: latency
        _norm("norm_token", "fwd", "bf16", "rms", 1, 2048, 1, 0.0),
        # a training batch of sequences, one gate a sequence, dropout on the branch
        _norm("norm_train", "fwd", "bf16", "rms", 32768, 2048, 2048, 0.1),
        # the largest batch's gradient: layer norm, an odd number of rows, one gate for all
        _norm("norm_grad", "bwd", "fp16", "layer", 32765, 4096, 1 << 30, 0.1, 0.5),
        # a short odd-sized activation with its residual
        _dropout("dropout_odd", "fp16", 257, 1001, 0.25, True),
        # a whole batch's activations
        _dropout("dropout_large", "bf16", 32768, 4096, 0.1, False),
        # between the two products of a training step
        _gated("gated_train", "fwd", "bf16", "silu", 16384, 2048),
        # the largest batch's gradient
        _gated("gated_grad", "bwd", "bf16", "gelu", 65536, 2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: rows from one to 65,536 and widths up to 4,096, spread over
    their logarithm, most widths multiples of eight and some of nothing."""
    op = rng.choice(["experts", "experts", "experts", "norm", "norm", "dropout", "gated"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    rows = _log(rng, 1, 65536)

    def width(lo, hi):
        w = _log(rng, lo, hi)
        w = max(8, w // 8 * 8) if rng.random() < 0.75 else w
        return w - 8 if w % 1024 == 0 and w < 4096 and w > 2048 else w

    if op == "experts":
        N, K = width(64, 4096), width(64, 4096)
        direction = rng.choice(["fwd", "dx", "dw", "grads", "all"])
        products = {"grads": 2, "all": 3}.get(direction, 1)
        # the library's wide products take aligned 16-bit operands; the others stay smaller
        top = 2e11 if dtype == "fp32" or N % 8 or K % 8 else 1e12
        rows = max(1, min(rows, int(top / (2.0 * N * K * products))))
        E = _log(rng, 1, 64)
        pad = rng.choice([0, 0, rows // 10])
        active = max(1, min(E, rows - pad, int(round(E * rng.uniform(0.5, 1.0)))))
        c = _experts("", direction, dtype, rows, E, active, N, K, pad, rng.choice([0.0, 0.5, 1.0]))
    elif op == "norm":
        c = _norm("", rng.choice(["fwd", "bwd"]), dtype, rng.choice(["rms", "layer"]), rows // 2 + 1,
                  width(64, 4096), rng.choice([1, 7, 256, 2048, 1 << 30]),
                  rng.choice([0.0, 0.1, 0.5]), rng.choice([1.0, 0.5]))
    elif op == "dropout":
        c = _dropout("", dtype, rows // 2 + 1, width(64, 4096), rng.choice([0.0, 0.1, 0.25, 0.5]),
                     rng.random() < 0.5)
    else:
        c = _gated("", rng.choice(["fwd", "bwd"]), dtype, rng.choice(["silu", "gelu"]), rows,
                   width(64, 2048))
    del c["name"]
    return c


# ----------------------------------------------------------------------------- inputs
def _offsets(case, seed):
    """First row of each expert and the end of the last: `active` experts get at least a row
    each and the rest by log-normal popularity; `pad` rows at the end belong to none."""
    rng = np.random.default_rng([seed, 77])
    E, active, used = case["experts"], case["active"], case["rows"] - case["pad"]
    who = rng.permutation(E)[:active]
    share = np.exp(case["skew"] * rng.standard_normal(active))
    count = np.zeros(E, dtype=np.int64)
    count[who] = 1 + rng.multinomial(used - active, share / share.sum())
    return [0] + [int(v) for v in np.cumsum(count)]


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, dt=dtype):
        t = torch.empty(shape, dtype=dt, device="cuda")
        t.normal_(shift, scale, generator=g)
        return t

    s = {"case": case}
    if case["op"] == "experts":
        E, N, K, R = case["experts"], case["N"], case["K"], case["rows"]
        s["host_offsets"] = _offsets(case, seed)
        s["offsets"] = torch.tensor(s["host_offsets"], dtype=torch.int64, device="cuda")
        if case["dir"] in ("fwd", "dw", "grads", "all"):
            s["x"] = normal(R, K)
        if case["dir"] != "dw":
            s["w"] = normal(E, N, K, scale=K ** -0.5)
        if case["dir"] != "fwd":
            s["dy"] = normal(R, N)
    elif case["op"] == "norm":
        R, D = case["rows"], case["D"]
        s["per_gate"] = min(case["per_gate"], R)
        G = (R + s["per_gate"] - 1) // s["per_gate"]
        s["gate"] = normal(G, D, scale=0.3, shift=0.5)
        s["w_post"] = normal(D, scale=0.1, shift=1.0)
        s["w_pre"] = normal(D, scale=0.1, shift=1.0)
        s["f"] = normal(R, D, scale=0.7, shift=0.1)
        s["seed"], s["offset"] = (seed * 0x9E3779B1 + 12345) & (2**63 - 1), 1000 * (seed % 7)
        if case["dir"] == "fwd":
            s["x"] = normal(R, D, scale=2.0)
        else:
            s["y"] = normal(R, D, scale=2.0)
            s["dy"], s["dh"] = normal(R, D), normal(R, D)
    elif case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["D"])
        s["residual"] = normal(case["rows"], case["D"]) if case["residual"] else None
        s["seed"], s["offset"] = (seed * 0x9E3779B1 + 54321) & (2**63 - 1), 4 * (seed % 5)
    else:
        s["h"] = normal(case["rows"], 2 * case["F"], scale=1.5)
        if case["dir"] == "bwd":
            s["da"] = normal(case["rows"], case["F"])
    return s


# ------------------------------------------------------------------- the plain forms
EPS = 1e-6
_M1, _M2, _GAMMA = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 0x9E3779B97F4A7C15


def _signed(v):
    v &= 2**64 - 1
    return v - 2**64 if v >= 2**63 else v


def _shift(z, n):
    return (z >> n) & (2 ** (64 - n) - 1)


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _factor(R, C, p, seed, offset, device):
    """What dropout multiplies a [R, C] tensor by: 0 or the inverse of the kept share. Four
    columns take the four 16-bit fields of one draw of the counter-based generator."""
    thr = _threshold(p)
    words = (C + 3) // 4
    z = torch.arange(offset + 1, offset + 1 + R * words, dtype=torch.int64, device=device)
    z = z * _signed(_GAMMA) + _signed(seed)
    z = (z ^ _shift(z, 30)) * _signed(_M1)
    z = (z ^ _shift(z, 27)) * _signed(_M2)
    z = z ^ _shift(z, 31)
    fields = torch.stack([_shift(z, 16 * j) & 0xFFFF if j else z & 0xFFFF for j in range(4)], 1)
    keep = fields.reshape(R, 4 * words)[:, :C] >= thr
    return keep, (65536.0 / (65536 - thr) if thr < 65536 else 0.0)


def _drop(v, p, seed, offset):
    if _threshold(p) == 0:
        return v
    keep, scale = _factor(v.shape[0], v.shape[1], p, seed, offset, v.device)
    return torch.where(keep, v * scale, torch.zeros_like(v))


def _normalise(v, kind):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * rstd, rstd


def _normalise_grad(d, hat, rstd, kind):
    d = d - hat * (d * hat).mean(1, keepdim=True)
    if kind == "layer":
        d = d - d.mean(1, keepdim=True)
    return d * rstd


def _plain(s):
    c = s["case"]
    dtype = DTYPES[c["dtype"]]
    out = {}
    if c["op"] == "experts":
        o = s["host_offsets"]
        d = c["dir"]
        if d in ("fwd", "all"):
            out["y"] = torch.zeros(c["rows"], c["N"], dtype=dtype, device="cuda")
        if d in ("dx", "grads", "all"):
            out["dx"] = torch.zeros(c["rows"], c["K"], dtype=dtype, device="cuda")
        if d in ("dw", "grads", "all"):
            out["dw"] = torch.zeros(c["experts"], c["N"], c["K"], dtype=dtype, device="cuda")
        for e in range(c["experts"]):
            lo, hi = o[e], o[e + 1]
            if lo == hi:
                continue
            if "y" in out:
                out["y"][lo:hi] = (s["x"][lo:hi].float() @ s["w"][e].float().t()).to(dtype)
            if "dx" in out:
                out["dx"][lo:hi] = (s["dy"][lo:hi].float() @ s["w"][e].float()).to(dtype)
            if "dw" in out:
                out["dw"][e] = (s["dy"][lo:hi].float().t() @ s["x"][lo:hi].float()).to(dtype)
    elif c["op"] == "norm":
        R = c["rows"]
        which = torch.arange(R, device="cuda") // s["per_gate"]
        gate, post, pre = s["gate"].float()[which], s["w_post"].float(), s["w_pre"].float()
        fhat, frstd = _normalise(s["f"].float(), c["kind"])
        if c["dir"] == "fwd":
            y = c["alpha"] * s["x"].float() + gate * _drop(fhat * post, c["p"], s["seed"], s["offset"])
            out["y"] = y.to(dtype)
            out["h"] = (_normalise(y, c["kind"])[0] * pre).to(dtype)
        else:
            dh = s["dh"].float()
            yhat, yrstd = _normalise(s["y"].float(), c["kind"])
            t = s["dy"].float() + _normalise_grad(dh * pre, yhat, yrstd, c["kind"])
            u = _drop(t * gate, c["p"], s["seed"], s["offset"])
            out["dx"] = (c["alpha"] * t).to(dtype)
            out["df"] = _normalise_grad(u * post, fhat, frstd, c["kind"]).to(dtype)
            z = t * _drop(fhat * post, c["p"], s["seed"], s["offset"])
            G = s["gate"].shape[0]
            spare = G * s["per_gate"] - R
            if spare:
                z = torch.cat([z, z.new_zeros(spare, z.shape[1])])
            out["dgate"] = z.view(G, s["per_gate"], -1).sum(1).to(dtype)
            out["dw_post"] = (u * fhat).sum(0)
            out["dw_pre"] = (dh * yhat).sum(0)
    elif c["op"] == "dropout":
        v = _drop(s["x"].float(), c["p"], s["seed"], s["offset"])
        if s["residual"] is not None:
            v = v + s["residual"].float()
        out["y"] = v.to(dtype)
    else:
        h = s["h"].float()
        g, u = h[:, :c["F"]], h[:, c["F"]:]
        if c["act"] == "silu":
            sig = 1.0 / (1.0 + torch.exp(-g))
            a, slope = g * sig, sig * (1.0 + g * (1.0 - sig))
        else:
            cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
            a, slope = g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
        if c["dir"] == "fwd":
            out["a"] = (a * u).to(dtype)
        else:
            da = s["da"].float()
            out["dh"] = torch.cat([da * u * slope, da * a], 1).to(dtype)
    return out


def _kernels(s):
    from paper_2101_07968_gb300 import layers as ly
    c = s["case"]
    if c["op"] == "experts":
        out, d = {}, c["dir"]
        if d in ("fwd", "all"):
            out["y"] = ly.expert_matmul(s["x"], s["w"], s["offsets"])
        if d in ("dx", "grads", "all"):
            out["dx"] = ly.expert_matmul_grad_input(s["dy"], s["w"], s["offsets"])
        if d in ("dw", "grads", "all"):
            out["dw"] = ly.expert_matmul_grad_weight(s["dy"], s["x"], s["offsets"])
        return out
    if c["op"] == "norm":
        how = dict(gate=s["gate"], rows_per_gate=s["per_gate"], w_post=s["w_post"],
                   w_pre=s["w_pre"], residual_scale=c["alpha"], kind=c["kind"], eps=EPS, p=c["p"],
                   seed=s["seed"], offset=s["offset"])
        if c["dir"] == "fwd":
            y, h = ly.block_norm(s["x"], s["f"], **how)
            return {"y": y, "h": h}
        r = ly.block_norm_grad(s["dy"], s["dh"], s["y"], s["f"], **how)
        return {k: r[k] for k in ("dx", "df", "dgate", "dw_post", "dw_pre")}
    if c["op"] == "dropout":
        return {"y": ly.dropout(s["x"], c["p"], s["seed"], offset=s["offset"], residual=s["residual"])}
    if c["dir"] == "fwd":
        return {"a": ly.gated_unit(s["h"], act=c["act"])}
    return {"dh": ly.gated_unit_grad(s["da"], s["h"], act=c["act"])}


def run(state):
    return _kernels(state) if own else _plain(state)


# ----------------------------------------------------------------- the least work
def work(case):
    b = SIZE[case["dtype"]]
    if case["op"] == "experts":
        R, N, K = case["rows"] - case["pad"], case["N"], case["K"]
        total = case["rows"]
        used, every = case["active"] * N * K, case["experts"] * N * K
        d = case["dir"]
        byte = {"fwd": R * K + total * N + used, "dx": R * N + total * K + used,
                "dw": R * (N + K) + every,
                "grads": R * (N + K) + total * K + used + every,
                "all": R * (N + K) + total * (N + K) + used + every}[d]
        n = {"grads": 2, "all": 3}.get(d, 1)
        return {"bytes": byte * b, "flops": 2.0 * n * R * N * K}
    if case["op"] == "norm":
        R, D = case["rows"], case["D"]
        gates = (R + case["per_gate"] - 1) // case["per_gate"]
        if case["dir"] == "fwd":
            return {"bytes": (4 * R + gates + 2) * D * b, "flops": 12.0 * R * D}
        return {"bytes": (6 * R + 2 * gates + 2) * D * b + 8 * D, "flops": 30.0 * R * D}
    if case["op"] == "dropout":
        n = case["rows"] * case["D"]
        return {"bytes": (3 if case["residual"] else 2) * n * b, "flops": 2.0 * n}
    n = case["rows"] * case["F"]
    return {"bytes": (3 if case["dir"] == "fwd" else 5) * n * b,
            "flops": (8.0 if case["dir"] == "fwd" else 20.0) * n}


# ------------------------------------------------- the definition, in 64 bits
def _mask64(R, C, p, seed, offset):
    """Kept elements by SplitMix64's definition in unsigned 64-bit numpy arithmetic."""
    words = (C + 3) // 4
    with np.errstate(over="ignore"):
        n = np.arange(R * words, dtype=np.uint64) + np.uint64(offset + 1)
        z = n * np.uint64(_GAMMA) + np.uint64(seed)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(_M1)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(_M2)
        z ^= z >> np.uint64(31)
    fields = np.ascontiguousarray(z.astype("<u8")).view("<u2").reshape(R, 4 * words)[:, :C]
    return torch.from_numpy(fields.astype(np.int32) >= int(math.floor(p * 65536 + 0.5))).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "experts":
        o, out, d = s["host_offsets"], {}, case["dir"]

        def zeros(*shape):
            return torch.zeros(shape, dtype=torch.float64, device="cuda")
        if d in ("fwd", "all"):
            out["y"] = zeros(case["rows"], case["N"])
            for e in range(case["experts"]):
                torch.matmul(s["x"][o[e]:o[e + 1]].double(), s["w"][e].double().t(),
                             out=out["y"][o[e]:o[e + 1]])
        if d in ("dx", "grads", "all"):
            out["dx"] = zeros(case["rows"], case["K"])
            for e in range(case["experts"]):
                torch.matmul(s["dy"][o[e]:o[e + 1]].double(), s["w"][e].double(),
                             out=out["dx"][o[e]:o[e + 1]])
        if d in ("dw", "grads", "all"):
            out["dw"] = zeros(case["experts"], case["N"], case["K"])
            for e in range(case["experts"]):
                if o[e] < o[e + 1]:
                    torch.matmul(s["dy"][o[e]:o[e + 1]].double().t(), s["x"][o[e]:o[e + 1]].double(),
                                 out=out["dw"][e])
        return out
    if case["op"] == "gated":
        g, u = s["h"].double().split(case["F"], 1)
        if case["act"] == "silu":
            sg = torch.sigmoid(g)
            a, slope = g * sg, sg + g * sg * (1 - sg)
        else:
            phi = torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
            cdf = torch.special.ndtr(g)
            a, slope = g * cdf, cdf + g * phi
        if case["dir"] == "fwd":
            return {"a": a * u}
        da = s["da"].double()
        dh = torch.empty(case["rows"], 2 * case["F"], dtype=torch.float64, device="cuda")
        dh[:, :case["F"]] = da * u * slope
        dh[:, case["F"]:] = da * a
        return {"dh": dh}
    if case["op"] == "dropout":
        keep = _mask64(case["rows"], case["D"], case["p"], s["seed"], s["offset"])
        kept = 1 - math.floor(case["p"] * 65536 + 0.5) / 65536
        y = s["x"].double() / kept * keep
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    # norms: variance and mean by their definitions, gradients by the chain rule
    R, D = case["rows"], case["D"]
    if case["p"] > 0:
        kept = 1 - math.floor(case["p"] * 65536 + 0.5) / 65536
        m = _mask64(R, D, case["p"], s["seed"], s["offset"]).double() / kept
    else:
        m = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    gate = s["gate"].double().repeat_interleave(s["per_gate"], 0)[:R]
    post, pre = s["w_post"].double(), s["w_pre"].double()
    layer = case["kind"] == "layer"

    def stats(v):
        mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
        var = ((v - mean) ** 2).sum(1, keepdim=True) / D
        return mean, (var + EPS) ** -0.5

    f = s["f"].double()
    fm, fr = stats(f)
    fhat = (f - fm) * fr
    if case["dir"] == "fwd":
        y = case["alpha"] * s["x"].double() + gate * m * post * fhat
        ym, yr = stats(y)
        return {"y": y, "h": (y - ym) * yr * pre}

    def back(d, hat, r):
        tot = (d * hat).sum(1, keepdim=True) / D
        return r * (d - (d.sum(1, keepdim=True) / D if layer else 0.0) - hat * tot)

    y, dh = s["y"].double(), s["dh"].double()
    ym, yr = stats(y)
    yhat = (y - ym) * yr
    t = s["dy"].double() + back(dh * pre, yhat, yr)
    G = s["gate"].shape[0]
    z = t * m * post * fhat
    dgate = torch.stack([z[i * s["per_gate"]:(i + 1) * s["per_gate"]].sum(0) for i in range(G)]) \
        if G <= 4096 else torch.zeros(G, D, dtype=torch.float64, device="cuda").index_add_(
            0, torch.arange(R, device="cuda") // s["per_gate"], z)
    return {"dx": case["alpha"] * t, "df": back(t * gate * m * post, fhat, fr), "dgate": dgate,
            "dw_post": (t * gate * m * fhat).sum(0), "dw_pre": (dh * yhat).sum(0)}
