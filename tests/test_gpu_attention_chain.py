"""The chain with attention before the experts: its outputs and gradients against automatic
differentiation of the same formulas in 64 bits, its measured times and schedules, its command."""
import math

import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ec():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import expert_chain
    yield expert_chain
    expert_chain.ly.check_status()


def plain(chain, x, assigned, lengths, p, seed, scale, eps=1e-6):
    """The chain in 64 bits on the CPU; parameters as leaves. Returns output, leaves."""
    leaf = lambda t: lo.d64(t).requires_grad_()
    leaves = dict(x=leaf(x), w_pre=[leaf(w) for w in chain.w_pre],
                  blocks=[{k: leaf(v) for k, v in b.items()} for b in chain.blocks])
    rows, D = x.shape
    H, G, W = chain.heads, chain.kv_heads, chain.head_dim
    rms = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * w
    keep = lambda use: lo.keep_factor(rows, D, p, seed, use * rows * ((D + 3) // 4))
    pos = torch.cat([torch.arange(n) for n in lengths])
    y = leaves["x"] * keep(0)
    h = rms(y, leaves["w_pre"][0])
    for i, b in enumerate(leaves["blocks"]):
        q, k, v = (h @ b["qkv"][0].t()).unflatten(1, (-1, W)).split((H, G, G), 1)
        q, k = (ao.rotary_forward(t, w, pos, W, 10000.0, False, True, eps) for t, w in ((q, b["w_q"]), (k, b["w_k"])))
        o, at = [], 0
        for n in lengths:
            kk, vv = (t[at:at + n].repeat_interleave(H // G, 1) for t in (k, v))
            s = torch.einsum("ihd,jhd->hij", q[at:at + n], kk) * W ** -0.5
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
            o.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), vv))
            at += n
        f = torch.cat(o).flatten(1) @ b["out"][0].t()
        y = scale * y + b["gate_a"] * keep(2 * i + 1) * rms(f, b["w_post_a"])
        h = rms(y, b["w_pre_a"])
        up, down = b["up"][assigned[i].cpu()], b["down"][assigned[i].cpu()]
        u = torch.einsum("rfd,rd->rf", up, h)
        F = u.shape[1] // 2
        a = torch.nn.functional.silu(u[:, :F]) * u[:, F:]
        f = torch.einsum("rdf,rf->rd", down, a)
        y = scale * y + b["gate"] * keep(2 * i + 2) * rms(f, b["w_post"])
        h = rms(y, leaves["w_pre"][i + 1])
    return y, leaves


def test_against_automatic_differentiation(ec):
    """Floats: every quantity passes through some twenty operators of at most 64 rounded operations
    each, whose inputs are of order one; 2e-4 of the largest element is 1,600 units of the last
    place, ten times what that adds up to."""
    p, seed, scale, lengths = 0.2, 5, 0.9, [40, 1, 49]
    rows = sum(lengths)
    chain = ec.ExpertChain(2, 64, 48, 4, dtype=torch.float32, p=p, seed=seed, residual_scale=scale, heads=4, kv_heads=2,
                           head_dim=24)
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(rows, 64, generator=g).cuda() for _ in range(2))
    assigned = [torch.randint(0, 4, (rows,), generator=g).cuda() for _ in range(2)]
    out, dx, grads, dw_pre0 = chain.step(x, assigned, dy, seq=chain.packed(lengths))
    want, leaves = plain(chain, x, assigned, lengths, p, seed, scale)
    want.backward(lo.d64(dy))

    def close(got, exact, what):
        err = float((lo.d64(got) - exact).abs().max())
        assert err <= 2e-4 * max(float(exact.abs().max()), 1e-3), (what, err)
    close(out, want.detach(), "output")
    close(dx, leaves["x"].grad, "x")
    close(dw_pre0, leaves["w_pre"][0].grad, "w_pre 0")
    for i, gr in enumerate(grads):
        for k in leaves["blocks"][i]:
            close(gr[k], leaves["blocks"][i][k].grad, (i, k))
    close(grads[0]["w_pre_next"], leaves["w_pre"][1].grad, "w_pre 1")


def test_parameters_without_attention_are_the_same(ec):
    a, b = ec.ExpertChain(2, 64, 32, 2), ec.ExpertChain(2, 64, 32, 2, heads=2, head_dim=32)
    for x, y in zip(a.blocks, b.blocks):
        assert all(torch.equal(x[k], y[k]) for k in x)
    more = sum(b.blocks[0][k].numel() for k in ("qkv", "out", "w_q", "w_k", "gate_a", "w_post_a", "w_pre_a"))
    assert [n + more for n in a.parameters()] == b.parameters()
    with pytest.raises(ValueError, match="seq"):
        x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
        b.step(x, [torch.zeros(4, dtype=torch.int64, device="cuda")] * 2, x)


def test_packed(ec):
    offsets, positions, whole = ec.ExpertChain.packed([3, 0, 2])
    assert offsets.tolist() == [0, 3, 3, 5] and positions.tolist() == [0, 1, 2, 0, 1] and whole.tolist() == [0, 5]


def test_measured_and_scheduled(ec):
    """Captured and replayed; attention's time is in the blocks' times."""
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn(2048, 256, generator=g).cuda().bfloat16() for _ in range(2))
    assigned = [torch.randint(0, 4, (2048,), generator=g).cuda() for _ in range(3)]
    chain = ec.ExpertChain(3, 256, 128, 4, p=0.1, heads=16, kv_heads=4, head_dim=128)
    seq = chain.packed([1500, 548])
    fc, bc = ec.measure(chain, x, assigned, dy, steps=2, warmup=1, seq=seq)
    chain.heads = 0
    fc0, bc0 = ec.measure(chain, x, assigned, dy, steps=2, warmup=1)
    assert all(a > b for a, b in zip(fc + bc, fc0 + bc0))
    res = ec.schedules(ec.profiles(fc, bc, chain.parameters(), 50))
    for r in res.values():
        assert bool((r["makespan"] <= r["one"]).all()) and bool((r["makespan"] <= r["each"]).all())


def test_command(ec, capsys):
    ec.main(["--layers", "2", "--rows", "300", "--width", "128", "--inner", "64", "--experts", "2", "--links", "20",
             "--heads", "4", "--kv-heads", "2", "--head-width", "64", "--sequences", "3"])
    out = capsys.readouterr().out
    assert "forward us" in out and "backward us" in out and "transmissions" in out
