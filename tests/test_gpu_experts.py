"""Products grouped by expert on the GPU against their definition in 64 bits, within bounds
derived in layer_oracle, at the sizes, offsets, layouts and values where they can go wrong."""
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
    yield layers
    layers.check_status()


def normal(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def operands(seed, rows, E, N, K, dtype):
    return (normal(seed, rows, K, dtype=dtype), normal(seed + 1, E, N, K, dtype=dtype, scale=K ** -0.5),
            normal(seed + 2, rows, N, dtype=dtype))


def offs(*v):
    return torch.tensor(v, dtype=torch.int64, device="cuda")


def check(ly, x, w, dy, offsets):
    ref = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), offsets.tolist(), x.shape[0])
    lo.assert_within(ly.expert_matmul(x, w, offsets), *ref["y"], "y")
    lo.assert_within(ly.expert_matmul_grad_input(dy, w, offsets), *ref["dx"], "dx")
    lo.assert_within(ly.expert_matmul_grad_weight(dy, x, offsets), *ref["dw"], "dw")


# one row to several tiles; experts without rows; rows before the first and after the last;
# sizes around a tile's; sizes that are multiples of nothing
CASES = [
    (1, 1, 1, (0, 1)), (1, 8, 8, (0, 1)), (1, 64, 128, (0, 0, 1, 1)), (2, 4096, 256, (0, 0, 1, 1, 2)),
    (3, 5, 7, (0, 2, 3)), (40, 128, 64, (0, 0, 17, 17, 40)), (100, 136, 72, (3, 40, 40, 90)),
    (255, 256, 192, (0, 255)), (256, 128, 128, (0, 256)), (257, 120, 200, (0, 1, 257)),
    (300, 1000, 264, (0, 16, 31, 63, 128, 300)), (513, 384, 520, (100, 100, 400)),
    (700, 129, 65, (0, 350, 690)), (64, 8, 2048, (0, 63)), (1300, 272, 136, (0, 1100, 1101, 1299)),
    (129, 2048, 24, (0, 64, 129)), (50, 77, 96, (50, 50)), (16, 96, 77, (0, 0)),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K,o", CASES)
def test_products(ly, dtype, rows, N, K, o):
    x, w, dy = operands(1, rows, len(o) - 1, N, K, dtype)
    check(ly, x, w, dy, offs(*o))


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_experts(ly, dtype):
    g = torch.Generator().manual_seed(5)
    E, rows = 1024, 1500
    cuts = torch.sort(torch.randint(0, rows + 1, (E - 1,), generator=g)).values.tolist()
    x, w, dy = operands(6, rows, E, 40, 64, dtype)
    check(ly, x, w, dy, offs(0, *cuts, rows))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("o", [(-5, 10, 30), (0, 90, 30), (0, 10, 500), (60, 20, 70), (500, 600, 700),
                               (-(2 ** 40), 2 ** 40, 3), (2 ** 62, -(2 ** 62), 0)])
def test_offsets_out_of_order_or_range_count_as_the_nearest_valid(ly, dtype, o):
    x, w, dy = operands(9, 70, 2, 48, 32, dtype)
    check(ly, x, w, dy, offs(*o))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", [(70, 64, 128), (300, 264, 72), (5, 100, 60)])
def test_layouts(ly, dtype, rows, N, K):
    """Rows with a stride, weights with N contiguous, weights inside a larger array, rows off
    16-byte boundaries."""
    o = offs(0, 3, rows)
    x, w, dy = operands(12, rows, 2, N, K, dtype)
    want = [ly.expert_matmul(x, w, o), ly.expert_matmul_grad_input(dy, w, o),
            ly.expert_matmul_grad_weight(dy, x, o)]
    ref = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), o.tolist(), rows)

    def wide(t):
        big = torch.full((t.shape[0], t.shape[1] + 40), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 8:8 + t.shape[1]] = t
        return big[:, 8:8 + t.shape[1]]

    def shifted(t):
        return torch.cat([t.flatten()[:1], t.flatten()])[1:].view(t.shape)

    kn = w.transpose(1, 2).contiguous().transpose(1, 2)
    part = torch.full((2, N + 3, K + 8), float("nan"), dtype=dtype, device="cuda")
    part[:, :N, :K] = w
    for xs, ws, ds in ((wide(x), w, wide(dy)), (x, kn, dy), (x, part[:, :N, :K], dy),
                       (shifted(x), w, dy), (x, shifted(w), shifted(dy)), (shifted(x), shifted(kn), dy)):
        lo.assert_within(ly.expert_matmul(xs, ws, o), *ref["y"], "y")
        lo.assert_within(ly.expert_matmul_grad_input(ds, ws, o), *ref["dx"], "dx")
        lo.assert_within(ly.expert_matmul_grad_weight(ds, xs, o), *ref["dw"], "dw")
    again = [ly.expert_matmul(x, w, o), ly.expert_matmul_grad_input(dy, w, o),
             ly.expert_matmul_grad_weight(dy, x, o)]
    assert all(torch.equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lo_row,hi_row", [(37, 120), (64, 65), (16, 47)])
def test_rows_of_other_experts_do_not_leak(ly, dtype, bad, lo_row, hi_row):
    """Rows of a neighbour, of no expert, and a neighbour's weights hold NaN or infinities:
    nothing of them reaches an expert's outputs."""
    rows, N, K = 160, 136, 72
    o = offs(lo_row, hi_row, hi_row + 9, 150)
    x, w, dy = operands(20, rows, 3, N, K, dtype)
    ref = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), o.tolist(), rows)
    xb, wb, db = x.clone(), w.clone(), dy.clone()
    out = torch.ones(rows, dtype=torch.bool)
    out[lo_row:hi_row] = False
    xb[out.cuda()] = bad
    db[out.cuda()] = bad
    wb[1:] = bad
    y, dx, dw = (ly.expert_matmul(xb, wb, o), ly.expert_matmul_grad_input(db, wb, o),
                 ly.expert_matmul_grad_weight(db, xb, o))
    own = slice(lo_row, hi_row)
    lo.assert_within(y[own], ref["y"][0][own], ref["y"][1][own], "y")
    lo.assert_within(dx[own], ref["dx"][0][own], ref["dx"][1][own], "dx")
    lo.assert_within(dw[0], ref["dw"][0][0], ref["dw"][1][0], "dw")
    for t in (y, dx):
        assert bool((t[:lo_row] == 0).all()) and bool((t[150:] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_far_apart(ly, dtype):
    """Element offsets past 32 bits."""
    rows, ld, N, K = 270_000, 8192, 64, 64
    big = torch.empty(rows, ld, dtype=dtype, device="cuda")
    x, w, dy = operands(30, 600, 2, N, K, dtype)
    o = offs(rows - 600, rows - 250, rows)
    big[:, :64].zero_()
    big[-600:, :64] = x
    ref = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), (0, 350, 600), 600)
    y = ly.expert_matmul(big[:, :64], w, o)
    lo.assert_within(y[-600:], *ref["y"], "y")
    assert bool((y[:-600] == 0).all())
    big[-600:, :64] = dy
    dx = ly.expert_matmul_grad_input(big[:, :64], w, o)
    lo.assert_within(dx[-600:], *ref["dx"], "dx")
    xs = torch.zeros(rows, K, dtype=dtype, device="cuda")
    xs[-600:] = x
    lo.assert_within(ly.expert_matmul_grad_weight(big[:, :64], xs, o), *ref["dw"], "dw")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_batches(ly, dtype):
    """Many tiles per SM and ragged experts, against 64-bit products on the GPU at sampled
    experts, with the bound of layer_oracle."""
    rows, N, K = 20_001, 1032, 520
    o = offs(0, 1, 4000, 4000, 4257, 12_000, 19_990)
    x, w, dy = operands(33, rows, 6, N, K, dtype)
    y, dx, dw = (ly.expert_matmul(x, w, o), ly.expert_matmul_grad_input(dy, w, o),
                 ly.expert_matmul_grad_weight(dy, x, o))
    for e in range(6):
        a, b = int(o[e]), int(o[e + 1])
        X, W, D = x[a:b].double(), w[e].double(), dy[a:b].double()
        for got, p, q, n in ((y[a:b], X, W.t(), K), (dx[a:b], D, W, N), (dw[e], D.t(), X, b - a)):
            lo.assert_within(got, (p @ q).cpu(), (n + 2) * lo.EPS * (p.abs() @ q.abs()).cpu(), "product")
    assert bool((y[19_990:] == 0).all()) and bool((dx[19_990:] == 0).all())


def test_gradients_against_differences(ly):
    """The products are linear in each operand: the change of <dy, y> along a direction is the
    gradient's product with it, exactly but for rounding."""
    x, w, dy = operands(40, 60, 3, 56, 48, torch.float32)
    o = offs(0, 20, 25, 58)
    dx, dw = ly.expert_matmul_grad_input(dy, w, o), ly.expert_matmul_grad_weight(dy, x, o)
    vx, vw, _ = operands(43, 60, 3, 56, 48, torch.float32)
    f = lambda a, b: float((lo.expert_products(lo.d64(a), b, None, o.tolist(), 60)["y"][0] * lo.d64(dy)).sum())
    for got, diff, v in ((dx, f(x + vx, lo.d64(w)) - f(x, lo.d64(w)), vx),
                         (dw, f(x, lo.d64(w) + lo.d64(vw)) - f(x, lo.d64(w)), vw)):
        terms = lo.d64(got) * lo.d64(v)
        # x + vx is rounded to 32 bits, as are the gradients: 64 products of 56 or 48 terms each
        allowed = 64 * lo.EPS * float(lo.d64(got).abs().sum() * lo.d64(v).abs().max())
        assert abs(float(terms.sum()) - diff) <= allowed


def test_streams_and_graphs(ly):
    x, w, dy = operands(50, 300, 4, 256, 128, torch.bfloat16)
    o = offs(0, 100, 100, 250, 300)
    f = lambda **k: (ly.expert_matmul(x, w, o, **k), ly.expert_matmul_grad_input(dy, w, o, **k),
                     ly.expert_matmul_grad_weight(dy, x, o, **k))
    want = f()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = f(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = f()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(caught, want))


def test_nothing_to_do(ly):
    x, w, dy = (torch.empty(0, 16, device="cuda"), torch.ones(2, 8, 16, device="cuda"),
                torch.empty(0, 8, device="cuda"))
    o = offs(0, 0, 0)
    assert ly.expert_matmul(x, w, o).shape == (0, 8)
    assert ly.expert_matmul_grad_input(dy, w, o).shape == (0, 16)
    assert torch.equal(ly.expert_matmul_grad_weight(dy, x, o), 0 * w)


def test_refusals(ly):
    from paper_2101_07968_gb300.dynacomm import DynaCommError
    x, w, dy = operands(60, 10, 2, 8, 16, torch.float32)
    o = offs(0, 5, 10)
    for bad in (lambda: ly.expert_matmul(x.cpu(), w, o), lambda: ly.expert_matmul(x, w.half(), o),
                lambda: ly.expert_matmul(x[:, :8], w, o), lambda: ly.expert_matmul(x, w, o[:2]),
                lambda: ly.expert_matmul(x, w, o.int()), lambda: ly.expert_matmul(x, w, o.cpu()),
                lambda: ly.expert_matmul(x.double(), w.double(), o), lambda: ly.expert_matmul(x, w[0], o),
                lambda: ly.expert_matmul(x.t().contiguous().t(), w, o),
                lambda: ly.expert_matmul(x[:, ::2], w[:, :, ::2], o),
                lambda: ly.expert_matmul(x[:1].expand(10, 16), w, o),
                lambda: ly.expert_matmul_grad_input(x, w, o),
                lambda: ly.expert_matmul_grad_weight(dy[:5], x, o)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(DynaCommError):  # experts that share memory
        ly.expert_matmul(x, w[:1].expand(2, 8, 16), o)
    with pytest.raises(DynaCommError):
        ly.expert_matmul_grad_weight(dy, x, torch.zeros(1026, dtype=torch.int64, device="cuda"))
