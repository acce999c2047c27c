"""The chain of expert blocks end to end: its outputs and gradients against automatic
differentiation of the same formulas in 64 bits, and the schedules of its measured times
against the oracle's."""
import numpy as np
import pytest
import torch

import layer_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ec():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import expert_chain
    return expert_chain


def plain(chain, x, assigned, p, seed, scale, eps=1e-6):
    """The chain in 64 bits on the CPU; parameters as leaves. Returns output, leaves."""
    leaf = lambda t: lo.d64(t).requires_grad_()
    leaves = dict(x=leaf(x), w_pre=[leaf(w) for w in chain.w_pre],
                  blocks=[{k: leaf(v) for k, v in b.items()} for b in chain.blocks])
    rows, D = x.shape
    rms = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * w
    draws = rows * ((D + 3) // 4)
    y = leaves["x"] * lo.keep_factor(rows, D, p, seed, 0)
    h = rms(y, leaves["w_pre"][0])
    for i, b in enumerate(leaves["blocks"]):
        up, down = b["up"][assigned[i].cpu()], b["down"][assigned[i].cpu()]
        u = torch.einsum("rfd,rd->rf", up, h)
        F = u.shape[1] // 2
        a = torch.nn.functional.silu(u[:, :F]) * u[:, F:]
        f = torch.einsum("rdf,rf->rd", down, a)
        keep = lo.keep_factor(rows, D, p, seed, (i + 1) * draws)
        y = scale * y + b["gate"] * keep * rms(f, b["w_post"])
        h = rms(y, leaves["w_pre"][i + 1])
    return y, leaves


def test_chain_against_automatic_differentiation(ec):
    """Floats: every quantity passes through some ten operators of at most 64 rounded
    operations each, whose inputs are of order one; 1e-4 of the largest element is 800 units of
    the last place, ten times what that adds up to."""
    p, seed, scale, rows = 0.2, 5, 0.9, 90
    chain = ec.ExpertChain(3, 64, 48, 4, dtype=torch.float32, p=p, seed=seed, residual_scale=scale)
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(rows, 64, generator=g).cuda() for _ in range(2))
    assigned = [torch.randint(0, 4, (rows,), generator=g).cuda() for _ in range(3)]
    assigned[1][:] = 2  # experts without a row
    out, dx, grads, dw_pre0 = chain.step(x, assigned, dy)
    want, leaves = plain(chain, x, assigned, p, seed, scale)
    want.backward(lo.d64(dy))

    def close(got, exact, what):
        err = float((lo.d64(got) - exact).abs().max())
        assert err <= 1e-4 * max(float(exact.abs().max()), 1e-3), (what, err)
    close(out, want.detach(), "output")
    close(dx, leaves["x"].grad, "x")
    close(dw_pre0, leaves["w_pre"][0].grad, "w_pre 0")
    for i, gr in enumerate(grads):
        for k in ("up", "down", "gate", "w_post"):
            close(gr[k], leaves["blocks"][i][k].grad, (i, k))
        if i < 2:
            close(gr["w_pre_next"], leaves["w_pre"][i + 1].grad, (i, "w_pre"))
    assert grads[2]["w_pre_next"] is None


def test_measured_chain_is_scheduled_as_the_oracle_does(ec, orc):
    from paper_2101_07968_gb300 import dynacomm as dc
    chain = ec.ExpertChain(5, 256, 128, 4, p=0.1)
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn(500, 256, generator=g).cuda().bfloat16() for _ in range(2))
    assigned = [torch.randint(0, 4, (500,), generator=g).cuda() for _ in range(5)]
    fc, bc = ec.measure(chain, x, assigned, dy, steps=2, warmup=1)
    assert len(fc) == len(bc) == 5 and min(fc + bc) >= 1
    prof = ec.profiles(fc, bc, chain.parameters(), 300)
    res = ec.schedules(prof)
    h = {k: v.cpu().numpy() for k, v in prof.items()}
    for d, (c, t) in ((dc.FWD, ("fc", "pt")), (dc.BWD, ("bc", "gt"))):
        exp = orc.schedule_batch(d, h[c], h[t], h["dt"])
        got = res[d]
        assert np.array_equal(got["makespan"].cpu().numpy(), exp["makespan"])
        assert np.array_equal(got["nseg"].cpu().numpy(), exp["nseg"])
        best = got["makespan"]
        assert bool((best <= got["one"]).all()) and bool((best <= got["each"]).all())
        if d == dc.FWD:  # one transmission: everything arrives, then everything is computed
            one = h["dt"] + h[t].sum(1) + h[c].sum(1)
            assert np.array_equal(got["one"].cpu().numpy(), one)
