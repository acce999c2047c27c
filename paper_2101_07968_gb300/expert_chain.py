"""A chain of mixture-of-experts blocks, measured on this GPU and scheduled.

The schedule of an iteration needs each layer's forward and backward compute time and the
size of what is pulled and pushed for it (Sec. IV-A). Here the layers are the blocks of a
language model's feed-forward chain, run by the layer operators: ``ExpertChain`` computes
forward and backward, ``measure`` takes their times on the GPU with CUDA events, and
``schedules`` solves the chain for many links at once.

    python -m paper_2101_07968_gb300.expert_chain [--layers 12] [--rows 8192] [--links 10000]

One block, for rows x (the residual stream) and h (its norm), with every row assigned to an
expert (rows are brought into expert order and back by index):

    f = down_e(act(gate_e(h)) * up_e(h)),  y = scale x + g drop(w_post n(f)),  h' = w_pre n(y)
"""
from __future__ import annotations

import argparse

import torch

from . import dynacomm as dc
from . import layers as ly


class ExpertChain:
    """Parameters of `layers` blocks (width D, `experts` experts of inner width F) and the
    forward and backward passes of one iteration. p is the dropout probability of the input
    and of every block's branch; each use takes its own range of the generator's draws."""

    def __init__(self, layers, D, F, experts, dtype=torch.bfloat16, device="cuda", p=0.0, seed=0,
                 residual_scale=1.0):
        self.D, self.F, self.E, self.p, self.seed = D, F, experts, p, seed
        self.residual_scale = residual_scale
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, scale, shift=0.0):
            return (torch.randn(shape, generator=g, device=device) * scale + shift).to(dtype)
        self.w_pre = [normal(D, scale=0.1, shift=1.0) for _ in range(layers + 1)]
        self.blocks = [dict(up=normal(experts, 2 * F, D, scale=D ** -0.5),
                            down=normal(experts, D, F, scale=F ** -0.5),
                            gate=normal(1, D, scale=0.1, shift=0.5),
                            w_post=normal(D, scale=0.1, shift=1.0)) for _ in range(layers)]

    def parameters(self):
        """Per block, how many parameters are pulled before it and pushed after it."""
        return [sum(t.numel() for t in b.values()) + self.D for b in self.blocks]

    def _norm(self, i, rows):
        b = self.blocks[i]
        return dict(gate=b["gate"], w_post=b["w_post"], w_pre=self.w_pre[i + 1],
                    residual_scale=self.residual_scale, p=self.p, seed=self.seed,
                    offset=(i + 1) * ly.dropout_draws(rows, self.D))

    @staticmethod
    def route(assigned, experts):
        """Rows in expert order, the way back, and each expert's first row."""
        order = torch.argsort(assigned, stable=True)
        back = torch.empty_like(order)
        back[order] = torch.arange(order.numel(), device=order.device)
        starts = torch.arange(experts + 1, device=assigned.device)
        return order, back, torch.searchsorted(assigned[order].contiguous(), starts)

    def forward_block(self, i, x, h, way, last):
        """(x, h) after block i and what its backward pass needs."""
        order, back, offsets = way
        b = self.blocks[i]
        hs = h[order]
        u = ly.expert_matmul(hs, b["up"], offsets)
        a = ly.gated_unit(u)
        f = ly.expert_matmul(a, b["down"], offsets)[back]
        y, h2 = ly.block_norm(x, f, want_h=not last, **self._norm(i, x.shape[0]))
        return y, h2, dict(hs=hs, u=u, a=a, f=f, y=y)

    def backward_block(self, i, dy, dh, saved, way):
        """Gradients of x and h before block i, and of its parameters."""
        order, back, offsets = way
        b = self.blocks[i]
        r = ly.block_norm_grad(dy, dh, saved["y"], saved["f"], **self._norm(i, saved["y"].shape[0]))
        df = r["df"][order]
        grads = dict(gate=r["dgate"], w_post=r["dw_post"], w_pre_next=r["dw_pre"],
                     down=ly.expert_matmul_grad_weight(df, saved["a"], offsets))
        da = ly.expert_matmul_grad_input(df, b["down"], offsets)
        du = ly.gated_unit_grad(da, saved["u"])
        grads["up"] = ly.expert_matmul_grad_weight(du, saved["hs"], offsets)
        dhs = ly.expert_matmul_grad_input(du, b["up"], offsets)
        return r["dx"], dhs[back], grads

    def step(self, x, assigned, dy, mark=lambda what, i: None):
        """One iteration: the output, the gradient of x and of every parameter. assigned: per
        block, the expert of each row; dy: the gradient of the output; mark(what, i) is called
        around every block ("forward" or "backward", before i and after it with i + 1)."""
        L = len(self.blocks)
        ways = [self.route(a, self.E) for a in assigned]
        x0 = ly.dropout(x, self.p, self.seed)
        y, h = ly.block_norm(x0, w_pre=self.w_pre[0])
        saved = []
        for i in range(L):
            mark("forward", i)
            y, h, s = self.forward_block(i, y, h, ways[i], last=i == L - 1)
            saved.append(s)
        mark("forward", L)
        out, dh, grads = y, None, [None] * L
        for i in reversed(range(L)):
            mark("backward", i + 1)
            dy, dh, grads[i] = self.backward_block(i, dy, dh, saved[i], ways[i])
        mark("backward", 0)
        first = ly.block_norm_grad(dy, dh, x0, w_pre=self.w_pre[0])
        return out, ly.dropout(first["dx"], self.p, self.seed), grads, first["dw_pre"]


def measure(chain, x, assigned, dy, steps=5, warmup=2):
    """Forward and backward time of every block on the GPU in whole microseconds, rounded up: the
    mean of `steps` iterations between CUDA events, after `warmup` (at least one). The iteration
    and its events are captured once as a CUDA graph and replayed, so that the times are the
    kernels' and not those of the host's calls, some 120 us for a block's forward."""
    L = len(chain.blocks)
    for _ in range(max(warmup, 1)):
        chain.step(x, assigned, dy)
    torch.cuda.synchronize()
    ev = {what: [torch.cuda.Event(enable_timing=True, external=True) for _ in range(L + 1)]
          for what in ("forward", "backward")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain.step(x, assigned, dy, lambda what, i: ev[what][i].record())
    total = {"forward": [0.0] * L, "backward": [0.0] * L}
    graph.replay()
    for _ in range(steps):
        graph.replay()
        torch.cuda.synchronize()
        for i in range(L):
            total["forward"][i] += ev["forward"][i].elapsed_time(ev["forward"][i + 1])
            total["backward"][i] += ev["backward"][i + 1].elapsed_time(ev["backward"][i])
    ly.check_status()
    return tuple([max(1, -int(-t * 1000 // steps)) for t in total[w]] for w in ("forward", "backward"))


def profiles(fc, bc, parameters, links, bits=16, seed=0, bw=(100_000_000, 10_000_000_000), dt=(5, 500)):
    """Cost rows of one measured chain over `links` links, by default those of a machine room:
    bandwidths (kbit/s) and latencies (us) log-uniform in their ranges; pt = gt = ceil(bits * 1000 * parameters / bandwidth)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def draw(lo, hi):
        u = torch.rand(links, generator=g, device="cuda", dtype=torch.float64)
        return (lo * (hi / lo) ** u).to(torch.int64)
    speed, wait = draw(*bw), draw(*dt)
    work = torch.tensor(parameters, dtype=torch.int64, device="cuda") * (bits * 1000)
    pt = (work[None, :] + speed[:, None] - 1) // speed[:, None]
    row = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda").expand(links, -1).contiguous()
    return {"fc": row(fc), "bc": row(bc), "pt": pt, "gt": pt, "dt": wait}


def schedules(prof):
    """The optimal forward and backward schedules and, for comparison, the makespans of one
    transmission for everything and of one a layer."""
    out = {}
    links, L = prof["fc"].shape
    words = max(dc.words(L), 1)
    for d, (c, x) in ((dc.FWD, ("fc", "pt")), (dc.BWD, ("bc", "gt"))):
        best = dc.schedule(d, prof[c], prof[x], prof["dt"])
        one = torch.zeros(links, words, dtype=torch.int32, device="cuda")
        each = torch.full((links, words), -1, dtype=torch.int32, device="cuda")
        if L % 32 != 1:  # only bits of breaks between layers
            each[:, -1] = (1 << ((L - 1) % 32)) - 1
        out[d] = dict(best, one=dc.eval_timeline(d, prof[c], prof[x], prof["dt"], one),
                      each=dc.eval_timeline(d, prof[c], prof[x], prof["dt"], each))
    return out


def main(argv=None):
    ap = argparse.ArgumentParser(description="measure a chain of expert blocks and schedule it")
    for name, value in (("layers", 12), ("rows", 8192), ("width", 2048), ("inner", 1024), ("experts", 8),
                        ("links", 10000)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    chain = ExpertChain(a.layers, a.width, a.inner, a.experts, p=0.1)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, dy = (torch.randn(a.rows, a.width, generator=g, device="cuda").bfloat16() for _ in range(2))
    assigned = [torch.randint(0, a.experts, (a.rows,), generator=g, device="cuda") for _ in range(a.layers)]
    fc, bc = measure(chain, x, assigned, dy)
    print("forward us ", fc)
    print("backward us", bc)
    res = schedules(profiles(fc, bc, chain.parameters(), a.links))
    for d, name in ((dc.FWD, "forward"), (dc.BWD, "backward")):
        r = res[d]
        gain = lambda k: float((1 - r["makespan"].double() / r[k].double()).mean()) * 100
        print(f"{name}: {float(r['nseg'].double().mean()):.1f} transmissions on average; "
              f"{gain('one'):.1f} % below one for everything, {gain('each'):.1f} % below one a layer")


if __name__ == "__main__":
    main()
