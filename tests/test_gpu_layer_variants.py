"""The layer operators' variants by size and alignment, at sizes that only one of them takes:
block norms of widths whose strides are constants or not, on and off 16-byte boundaries, with
gates of few and of many rows; float products of long sums; operands that are copied first, on
another stream."""
import pytest
import torch

import layer_oracle as lo
from test_gpu_experts import normal, offs, operands
from test_gpu_layers import DTYPES, norm_case, per_row

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    yield layers
    layers.check_status()


WIDTHS = [(40, 3001, 9), (21, 201, 4), (30, 1024, None), (70, 2048, 10), (19, 1536, 8), (300, 2560, 30),
          (12, 2050, 3), (500, 130, 60), (9, 512, 9), (1000, 256, 2), (333, 8, 333), (2500, 16, 1)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,D,per_gate", WIDTHS)
def test_block_norm_widths(ly, kind, dtype, rows, D, per_gate):
    c = norm_case(70, rows, D, dtype, per_gate, kind)
    alpha, eps, p, seed, offset = 1.25, 1e-6, 0.15, 1 << 40, 77
    how = dict(gate=c["gate"], w_post=c["w_post"], w_pre=c["w_pre"], residual_scale=alpha, kind=kind,
               eps=eps, p=p, seed=seed, offset=offset, rows_per_gate=per_gate)
    keep = lo.keep_factor(rows, D, p, seed, offset)
    e = {k: lo.d64(v) for k, v in c.items()}
    g = per_row(e["gate"], rows, per_gate)
    args = (e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind, eps, keep)
    y, h = ly.block_norm(c["x"], c["f"], **how)
    for got, exact, bound, what in zip((y, h), lo.norm_forward(*args), lo.norm_forward_bounds(*args), "yh"):
        lo.assert_within(got, exact, bound, what)
    r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
    b = lo.norm_backward(e["dy"], e["dh"], e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind, eps, keep)
    lo.assert_within(r["dx"], alpha * b["t"][0], alpha * b["t"][1], "dx")
    lo.assert_within(r["df"], *b["df"], "df")
    lo.assert_within(r["dgate"], *lo.add_rows(b["gate"], per_gate), "dgate")
    for k in ("w_post", "w_pre"):
        v, bd = lo.add_rows(b[k])
        lo.assert_within(r["d" + k], v[0], bd[0], "d" + k)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,D,per_gate", [(7, 5120, 3), (400, 8192, None), (5, 8200, 2), (6, 4104, 1)])
def test_block_norm_wide_rows(ly, kind, dtype, rows, D, per_gate):
    test_block_norm_widths(ly, kind, dtype, rows, D, per_gate)


@pytest.mark.parametrize("dtype", DTYPES)
def test_layer_norm_far_from_zero(ly, dtype):
    """Rows whose mean is many deviations from zero, and rows whose first element is far from
    the rest: the sums about the first element are then taken again."""
    rows, D = 24, 640
    c = norm_case(80, rows, D, dtype, None, "layer", shift=5.0)
    c["x"][::2, 0] = 60.0
    c["f"][1::2, 0] = -40.0
    e = {k: lo.d64(v) for k, v in c.items()}
    one = torch.ones(1, 1).double()
    b = lo.norm_backward(e["dy"], e["dh"], e["x"], e["f"], one, e["w_post"], e["w_pre"], 1.0, "layer", 1e-6, one)
    r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], w_post=c["w_post"], w_pre=c["w_pre"], kind="layer")
    lo.assert_within(r["dx"], *b["t"], "dx")
    lo.assert_within(r["df"], *b["df"], "df")
    args = (e["x"], e["f"], one, e["w_post"], e["w_pre"], 1.0, "layer", 1e-6, one)
    y, h = ly.block_norm(c["x"], c["f"], w_post=c["w_post"], w_pre=c["w_pre"], kind="layer")
    by, bh = lo.norm_forward_bounds(*args)
    lo.assert_within(y, lo.norm_forward(*args)[0], by, "y")
    lo.assert_within(h, lo.norm_forward(*args)[1], bh, "h")


@pytest.mark.parametrize("rows,E,N,K", [(6000, 1, 136, 72), (300, 2, 96, 4096), (5000, 3, 1000, 136)])
def test_float_products_of_long_sums(ly, rows, E, N, K):
    """Floats lose no more than sums in floats do. In the root mean square of standard normal
    operands: the parts leave out at most 3 2^-22 of a product, at random; a sum's 16 steps cut
    off below 2^-23 of it each, in one direction; adding up the rounds rounds by 2^-24 each, at
    random. Together below 2^-20 of the result."""
    x, w, dy = operands(90, rows, E, N, K, torch.float32)
    o = offs(*[rows * i // E for i in range(E + 1)])
    y, dx, dw = (ly.expert_matmul(x, w, o), ly.expert_matmul_grad_input(dy, w, o),
                 ly.expert_matmul_grad_weight(dy, x, o))
    for e in range(E):
        a, b = int(o[e]), int(o[e + 1])
        X, W, D = x[a:b].double(), w[e].double(), dy[a:b].double()
        for got, exact in ((y[a:b], X @ W.t()), (dx[a:b], D @ W), (dw[e], D.t() @ X)):
            rms = float((got.double() - exact).norm() / exact.norm())
            assert rms < 2.0 ** -20, rms


@pytest.mark.parametrize("dtype", DTYPES)
def test_floats_and_copied_operands_on_another_stream(ly, dtype):
    """Products that need a workspace, many in a row on a stream of their own while the current
    one allocates: a workspace is not handed out again before its product is done."""
    x, w, dy = operands(95, 400, 3, 501, 333, dtype)
    o = offs(0, 100, 250, 400)
    f = lambda **k: (ly.expert_matmul(x, w, o, **k), ly.expert_matmul_grad_input(dy, w, o, **k),
                     ly.expert_matmul_grad_weight(dy, x, o, **k))
    want = f()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, junk = [], []
    for _ in range(8):
        got.append(f(stream=s))
        junk.append(torch.full((1 << 20,), float("nan"), device="cuda"))
        junk.pop()
    s.synchronize()
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 16, 17, 64, 65])
def test_around_the_few_rows_limits(ly, dtype, rows):
    """The streaming kernel and the tiles agree with the definition on either side of the limits."""
    x, w, dy = operands(97, rows, 3, 200, 264, dtype)
    o = offs(0, rows // 3, rows // 3, rows)
    ref = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), o.tolist(), rows)
    lo.assert_within(ly.expert_matmul(x, w, o), *ref["y"], "y")
    lo.assert_within(ly.expert_matmul_grad_input(dy, w, o), *ref["dx"], "dx")
    lo.assert_within(ly.expert_matmul_grad_weight(dy, x, o), *ref["dw"], "dw")
