"""Block norms, dropout and gated units on the GPU against their definitions in 64 bits,
within bounds derived in layer_oracle; their gradients also against differences of the
definition; refusals of wrong arguments."""
import math

import numpy as np
import pytest
import torch

import layer_oracle as lo

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    return layers


def normal(seed, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype).cuda()


# --------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2048), (3, 5), (257, 1001), (130, 1024), (7, 4)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(ly, dtype, rows, cols, p):
    x, res = normal(1, rows, cols, dtype=dtype), normal(2, rows, cols, dtype=dtype)
    seed, offset = 0x9E3779B97F4A7C15 - 5, 12345678901
    k = lo.keep_factor(rows, cols, p, seed, offset)
    lo.assert_within(ly.dropout(x, p, seed, offset), lo.d64(x) * k, 2 * lo.EPS * lo.d64(x).abs() * k, "y")
    got = ly.dropout(x, p, seed, offset, residual=res)
    mag = lo.d64(x).abs() * k + lo.d64(res).abs()
    lo.assert_within(got, lo.d64(x) * k + lo.d64(res), 3 * lo.EPS * mag, "y + residual")
    if p == 0.0:
        assert torch.equal(ly.dropout(x, p, seed, offset), x)


def test_dropout_rate_streams_and_slices(ly):
    """The kept share is 1 - q within five standard deviations; other seeds and offsets give
    other masks; rows of a longer call are the calls on its rows."""
    x = torch.ones(1000, 4096, device="cuda")
    y = ly.dropout(x, 0.1, 42)
    q = math.floor(0.1 * 65536 + 0.5) / 65536
    kept = float((y != 0).double().mean())
    assert abs(kept - (1 - q)) < 5 * math.sqrt(q * (1 - q) / x.numel())
    assert not torch.equal(y, ly.dropout(x, 0.1, 43))
    assert not torch.equal(y, ly.dropout(x, 0.1, 42, offset=1))
    part = ly.dropout(x[300:400], 0.1, 42, offset=ly.dropout_draws(300, 4096))
    assert torch.equal(part, y[300:400])
    strided = x[:, :1003]
    assert torch.equal(ly.dropout(strided, 0.3, 7), ly.dropout(strided.contiguous(), 0.3, 7))
    base = torch.randn(1 + 8 * 64, device="cuda")
    odd = base[1:].view(8, 64)  # rows that start off 16-byte boundaries
    assert torch.equal(ly.dropout(odd, 0.3, 7), ly.dropout(odd.clone(), 0.3, 7))


def test_dropout_dropped_elements_are_zero_whatever_they_hold(ly):
    x = torch.full((64, 64), float("nan"), device="cuda")
    k = lo.keep_factor(64, 64, 0.5, 3, 0)
    y = ly.dropout(x, 0.5, 3).cpu()
    assert bool((y[k == 0] == 0).all()) and bool(torch.isnan(y[k > 0]).all())
    x.fill_(float("inf"))
    assert bool((ly.dropout(x, 1.0, 3) == 0).all())


# ------------------------------------------------------------------------ gated unit
def act_bounds(h, act):
    """Relative cost of the activation in 32 bits: exp to 2 ulp of an argument that is itself
    rounded (|g| EPS in the exponent), the rest a handful of operations; the slope is bounded by
    its terms' magnitudes."""
    out, a, slope, g, u = lo.gated(h, act)
    rel = (16 + 2 * g.abs()) * lo.EPS if act == "silu" else (16 + g * g) * lo.EPS
    terms = a.abs() + 1.2 + (g * torch.exp(-g * g / 2)).abs() if act == "gelu" else \
        1.0 + a.abs()
    return out, a, slope, g, u, rel, terms * rel + 1e-37


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,F", [(1, 1), (1, 2048), (5, 7), (130, 513), (257, 1024), (600, 24), (20000, 64)])
def test_gated_unit(ly, act, dtype, rows, F):
    h = normal(3, rows, 2 * F, dtype=dtype, scale=2.5)
    da = normal(4, rows, F, dtype=dtype)
    out, a, slope, g, u, rel, bs = act_bounds(lo.d64(h), act)
    lo.assert_within(ly.gated_unit(h, act), out, out.abs() * rel + 1e-37, "a")
    d = lo.d64(da)
    dh = ly.gated_unit_grad(da, h, act)
    lo.assert_within(dh[:, :F], d * u * slope, (d * u).abs() * bs, "dg")
    lo.assert_within(dh[:, F:], d * a, (d * a).abs() * rel + 1e-37, "du")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_unit_strides_and_large_arguments(ly, act):
    wide = normal(5, 40, 200, dtype=torch.bfloat16)
    h = wide[:, 8:136]
    assert torch.equal(ly.gated_unit(h, act), ly.gated_unit(h.contiguous(), act))
    da = normal(6, 40, 100, dtype=torch.bfloat16)[:, :64]
    assert torch.equal(ly.gated_unit_grad(da, h, act), ly.gated_unit_grad(da.contiguous(), h.contiguous(), act))
    off = normal(7, 1 + 16 * 64)[1:].view(16, 64)
    assert torch.equal(ly.gated_unit(off, act), ly.gated_unit(off.clone(), act))
    big = torch.tensor([[-200.0, -90.0, -40.0, 40.0, 200.0, 3.0e38, 1, 1, 1, 1, 1, 1.0]], device="cuda")
    a = ly.gated_unit(big, act).cpu()[0]
    assert torch.equal(a[3:], torch.tensor([40.0, 200.0, 3.0e38])) and bool((a[:3].abs() < 1e-15).all())
    dh = ly.gated_unit_grad(torch.ones(1, 6, device="cuda"), big, act).cpu()[0]
    assert bool(torch.isfinite(dh).all()) and bool((dh[:3].abs() < 1e-15).all())
    assert torch.equal(dh[3:6], torch.ones(3))


# ----------------------------------------------------------------------- block norms
def norm_case(seed, rows, D, dtype, per_gate, kind, shift=0.3):
    n = lambda i, *s, **k: normal(seed + i, *s, dtype=dtype, **k)
    G = -(-rows // per_gate) if per_gate else 1
    return dict(x=n(0, rows, D, scale=2.0, shift=shift), f=n(1, rows, D, scale=0.7, shift=shift),
                gate=n(2, G, D, scale=0.3, shift=0.5), w_post=n(3, D, scale=0.1, shift=1.0),
                w_pre=n(4, D, scale=0.1, shift=1.0), dy=n(5, rows, D), dh=n(6, rows, D))


def per_row(gate, rows, per_gate):
    return gate.repeat_interleave(per_gate or rows, 0)[:rows]


SHAPES = [(1, 1, 1), (1, 2048, 1), (3, 5, 2), (37, 257, 5), (64, 512, 16), (50, 513, None),
          (401, 768, 7), (33, 4096, 8), (9, 4100, None), (6, 16384, 4), (700, 64, 100),
          (2000, 96, None), (5000, 40, 1)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,D,per_gate", SHAPES)
def test_block_norm_both_ways(ly, kind, dtype, rows, D, per_gate):
    c = norm_case(10, rows, D, dtype, per_gate, kind)
    alpha, eps, p, seed, offset = 0.75, 1e-5, 0.2, 99, 1 << 33
    how = dict(gate=c["gate"], w_post=c["w_post"], w_pre=c["w_pre"], residual_scale=alpha, kind=kind,
               eps=eps, p=p, seed=seed, offset=offset, rows_per_gate=per_gate)
    keep = lo.keep_factor(rows, D, p, seed, offset)
    e = {k: lo.d64(v) for k, v in c.items()}
    g = per_row(e["gate"], rows, per_gate)
    y, h = ly.block_norm(c["x"], c["f"], **how)
    args = (e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind, eps, keep)
    ey, eh = lo.norm_forward(*args)
    by, bh = lo.norm_forward_bounds(*args)
    lo.assert_within(y, ey, by, "y")
    lo.assert_within(h, eh, bh, "h")

    r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
    b = lo.norm_backward(e["dy"], e["dh"], e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind,
                         eps, keep)
    lo.assert_within(r["dx"], alpha * b["t"][0], alpha * b["t"][1], "dx")
    lo.assert_within(r["df"], *b["df"], "df")
    lo.assert_within(r["dgate"], *lo.add_rows(b["gate"], per_gate), "dgate")
    for k in ("w_post", "w_pre"):
        v, bd = lo.add_rows(b[k])
        lo.assert_within(r["d" + k], v[0], bd[0], "d" + k)
    again = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
    assert all(torch.equal(r[k], again[k]) for k in r)  # no sum's order depends on timing


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,D", [(5, 64), (40, 1001)])
def test_block_norm_forms(ly, kind, rows, D):
    """The first norm alone, the last residual alone, and operands left out."""
    dtype, eps = torch.bfloat16, 1e-6
    c = norm_case(20, rows, D, dtype, None, kind)
    e = {k: lo.d64(v) for k, v in c.items()}
    one = torch.ones(1, 1).double()
    y, h = ly.block_norm(c["x"], w_pre=c["w_pre"], kind=kind, residual_scale=3.0)
    assert y is c["x"]
    args = (e["x"], None, one, one, e["w_pre"], 1.0, kind, eps, one)
    lo.assert_within(h, lo.norm_forward(*args)[1], lo.norm_forward_bounds(*args)[1], "h")
    r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], w_pre=c["w_pre"], kind=kind, residual_scale=3.0)
    b = lo.norm_backward(e["dy"], e["dh"], e["x"], None, one, one, e["w_pre"], 1.0, kind, eps, one)
    lo.assert_within(r["dx"], *b["t"], "dx")
    assert r["df"] is None and r["dgate"] is None and r["dw_post"] is None
    r = ly.block_norm_grad(None, c["dh"], c["x"], kind=kind)  # dy zero, no weight
    b = lo.norm_backward(0 * e["dy"], e["dh"], e["x"], None, one, one, one, 1.0, kind, eps, one)
    lo.assert_within(r["dx"], *b["t"], "dx without dy")
    assert r["dw_pre"] is None

    y, h = ly.block_norm(c["x"], c["f"], kind=kind, want_h=False)
    assert h is None
    args = (e["x"], e["f"], one, one, one, 1.0, kind, eps, one)
    lo.assert_within(y, lo.norm_forward(*args)[0], lo.norm_forward_bounds(*args)[0], "y")
    r = ly.block_norm_grad(c["dy"], None, c["x"], c["f"], w_post=c["w_post"], kind=kind)
    b = lo.norm_backward(e["dy"], None, e["x"], e["f"], one, e["w_post"], one, 1.0, kind, eps, one)
    assert torch.equal(r["dx"], c["dy"])
    lo.assert_within(r["df"], *b["df"], "df")
    lo.assert_within(r["dw_post"], *(v[0] for v in lo.add_rows(b["w_post"])), "dw_post")


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_block_norm_rows_of_zeros_and_of_large_values(ly, kind):
    x = torch.zeros(4, 128, device="cuda")
    x[1] = 1e4
    x[2, ::2] = 3e4
    f = x.flip(0).contiguous()
    y, h = ly.block_norm(x, f, kind=kind, eps=1e-6)
    ey, eh = lo.norm_forward(lo.d64(x), lo.d64(f), 1.0, 1.0, torch.ones(1).double(), 1.0, kind, 1e-6, 1.0)
    args = (lo.d64(x), lo.d64(f), torch.ones(1).double(), torch.ones(1).double(), torch.ones(1).double(), 1.0,
            kind, 1e-6, torch.ones(1).double())
    by, bh = lo.norm_forward_bounds(*args)
    lo.assert_within(y, ey, by, "y")
    lo.assert_within(h, eh, bh, "h")
    nan = x.clone()
    nan[3] = float("nan")  # one row's fault stays in its row
    y, h = ly.block_norm(nan, f, kind=kind, eps=1e-6)
    assert bool(torch.isfinite(y[:3]).all()) and bool(torch.isfinite(h[:3]).all())


def test_block_norm_unaligned_rows(ly):
    """Rows that start off 16-byte boundaries give the same bits as copies that do not."""
    c = norm_case(30, 20, 256, torch.bfloat16, 4, "rms")
    off = {k: torch.cat([v.flatten()[:1], v.flatten()])[1:].view(v.shape) for k, v in c.items()}
    how = lambda d: dict(gate=d["gate"], w_post=d["w_post"], w_pre=d["w_pre"], rows_per_gate=4, p=0.3, seed=5)
    a, b = ly.block_norm(c["x"], c["f"], **how(c)), ly.block_norm(off["x"], off["f"], **how(off))
    e = {k: lo.d64(v) for k, v in c.items()}
    args = (e["x"], e["f"], per_row(e["gate"], 20, 4), e["w_post"], e["w_pre"], 1.0, "rms", 1e-6,
            lo.keep_factor(20, 256, 0.3, 5, 0))
    for (y, h) in (a, b):
        ey, eh = lo.norm_forward(*args)
        by, bh = lo.norm_forward_bounds(*args)
        lo.assert_within(y, ey, by, "y")
        lo.assert_within(h, eh, bh, "h")


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_against_differences(ly, kind):
    """<gradient, v> of every input against a central difference of the definition in 64 bits
    along v: step 1e-4 leaves a truncation of order 1e-8 of values near one, so what differs
    is the kernel's own error, bounded element by element."""
    rows, D, per = 6, 40, 2
    c = norm_case(40, rows, D, torch.float32, per, kind)
    e = {k: lo.d64(v) for k, v in c.items()}
    keep = lo.keep_factor(rows, D, 0.25, 8, 0)
    alpha, eps = 0.5, 1e-5

    def first_y(d):
        return lo.norm_forward(d["x"], d["f"], per_row(d["gate"], rows, per), d["w_post"], d["w_pre"],
                               alpha, kind, eps, keep)

    def loss(d):
        y, h = first_y(d)
        return float((y * e["dy"]).sum() + (h * e["dh"]).sum())

    y32 = first_y(e)[0].float().cuda()  # what the forward call would hand to the gradient
    r = ly.block_norm_grad(c["dy"], c["dh"], y32, c["f"], gate=c["gate"], w_post=c["w_post"],
                           w_pre=c["w_pre"], residual_scale=alpha, kind=kind, eps=eps, p=0.25, seed=8,
                           rows_per_gate=per)
    b = lo.norm_backward(e["dy"], e["dh"], lo.d64(y32), e["f"], per_row(e["gate"], rows, per), e["w_post"],
                         e["w_pre"], alpha, kind, eps, keep)
    bounds = {"x": alpha * b["t"][1], "f": b["df"][1], "gate": lo.add_rows(b["gate"], per)[1],
              "w_post": lo.add_rows(b["w_post"])[1][0], "w_pre": lo.add_rows(b["w_pre"])[1][0]}
    names = {"x": "dx", "f": "df", "gate": "dgate", "w_post": "dw_post", "w_pre": "dw_pre"}
    step = 1e-4
    for k, name in names.items():
        v = torch.randn(e[k].shape, generator=torch.Generator().manual_seed(77)).double()
        up, down = dict(e), dict(e)
        up[k], down[k] = e[k] + step * v, e[k] - step * v
        diff = (loss(up) - loss(down)) / (2 * step)
        got = float((lo.d64(r[name]) * v).sum())
        allowed = float((bounds[k] * v.abs()).sum() + (lo.d64(r[name]) * v).abs().sum() * 2.0 ** -23)
        assert abs(got - diff) <= allowed + 1e-6 * v.numel(), (k, got, diff, allowed)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_gradient_against_differences(ly, act):
    h, da = normal(50, 5, 14), normal(51, 5, 7)
    dh = ly.gated_unit_grad(da, h, act)
    v = lo.d64(normal(52, 5, 14))
    step = 1e-4
    f = lambda t: float((lo.gated(t, act)[0] * lo.d64(da)).sum())
    diff = (f(lo.d64(h) + step * v) - f(lo.d64(h) - step * v)) / (2 * step)
    got = float((lo.d64(dh) * v).sum())
    assert abs(got - diff) < 1e-6 * 70 + 64 * lo.EPS * float((lo.d64(dh) * v).abs().sum() + 70)


# -------------------------------------------------------------------- streams, refusals
def test_layers_on_another_stream_and_in_a_graph(ly):
    c = norm_case(60, 300, 512, torch.bfloat16, 100, "rms")
    how = dict(gate=c["gate"], w_post=c["w_post"], w_pre=c["w_pre"], rows_per_gate=100, p=0.1, seed=1)
    want = ly.block_norm(c["x"], c["f"], **how)
    grad = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ly.block_norm(c["x"], c["f"], stream=s, **how)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g1 = ly.block_norm(c["x"], c["f"], **how)
        g2 = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
        g3 = ly.gated_unit(ly.dropout(c["x"], 0.5, 3))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(g1, want))
    assert all(torch.equal(g2[k], grad[k]) for k in grad)
    assert torch.equal(g3, ly.gated_unit(ly.dropout(c["x"], 0.5, 3)))


def test_nothing_to_do(ly):
    z = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    assert ly.dropout(z, 0.5, 1).shape == (0, 64) and ly.gated_unit(z).shape == (0, 32)
    assert ly.gated_unit_grad(torch.empty(0, 32, device="cuda"), z).shape == (0, 64)
    y, h = ly.block_norm(z, z, w_post=w, w_pre=w)
    assert h.shape == (0, 64)
    r = ly.block_norm_grad(z, z, z, z, w_post=w, w_pre=w)
    assert torch.equal(r["dw_post"], 0 * w) and torch.equal(r["dw_pre"], 0 * w)


def test_refusals(ly):
    from paper_2101_07968_gb300.dynacomm import DynaCommError
    x = torch.zeros(4, 8, device="cuda")
    for bad in (-0.1, 1.1, float("nan")):
        with pytest.raises(DynaCommError):
            ly.dropout(x, bad, 1)
        with pytest.raises(DynaCommError):
            ly.block_norm(x, x, p=bad)
    with pytest.raises(DynaCommError):
        ly.dropout(x, 0.1, 1, offset=-1)
    with pytest.raises(DynaCommError):
        ly.block_norm(x, eps=-1.0)
    with pytest.raises(DynaCommError):
        ly.block_norm(torch.zeros(2, 16385, device="cuda"))
    with pytest.raises(ValueError):
        ly.dropout(x.cpu(), 0.1, 1)
    with pytest.raises(ValueError):
        ly.dropout(x.t(), 0.1, 1)
    with pytest.raises(ValueError):
        ly.dropout(x, 0.1, 1, residual=x.half())
    with pytest.raises(ValueError):
        ly.dropout(x.double(), 0.1, 1)
    with pytest.raises(ValueError):
        ly.gated_unit(x[:, :7])
    with pytest.raises(ValueError):
        ly.gated_unit(x, act="relu")
    with pytest.raises(ValueError):
        ly.gated_unit_grad(x, x)
    with pytest.raises(ValueError):
        ly.block_norm(x, x, kind="batch")
    with pytest.raises(ValueError):
        ly.block_norm(x, x, gate=x, rows_per_gate=2)
    with pytest.raises(ValueError):
        ly.block_norm(x, x, rows_per_gate=0)
    with pytest.raises(ValueError):
        ly.block_norm(x, want_h=False)
    with pytest.raises(ValueError):
        ly.block_norm(x[:, ::2], x[:, ::2])
    with pytest.raises(ValueError):
        ly.block_norm_grad(x, None, x)
