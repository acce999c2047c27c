"""Sums of the expert products: long ones, whose error must not grow with their length, sums of
floats against plain 32-bit ones, and sums with infinities among their terms."""
import math

import pytest
import torch

import layer_oracle as lo
from test_gpu_experts import check, normal, offs, operands

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    yield layers
    layers.check_status()


def positive(seed, lines, length, dtype, along):
    """[lines, length] (along 1) or [length, lines] (along 0): terms of one sign, the lines' sums
    spread over a factor of two, so that their roundings are spread, too."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.rand(lines, length, generator=g, device="cuda") * 0.125
    t = t * (1 + torch.rand(lines, 1, generator=g, device="cuda"))
    return (t if along else t.t()).contiguous().to(dtype)


# A round of 512 steps of the tensor cores loses at most two units of the last place of the sum so
# far (its terms are cut off when they are aligned, and the sum is) a step, 2 x 2^-23, while that sum
# grows evenly: 256 x 2^-22. Adding up 33 rounds, rounded, loses 33 x 2^-24 more.
LOST = 2.0 ** -14 + 33 * 2.0 ** -24


def assert_not_cut_off(got, exact):
    """Elementwise within LOST and one rounding; on average within LOST and five deviations of the
    mean of independent roundings, each of at most the type's unit."""
    u = lo.UNIT[got.dtype]
    off = (got.double() - exact) / exact
    assert float(off.abs().max()) <= (1 + u) * (u + LOST)
    assert abs(float(off.mean())) <= LOST + 5 * u / math.sqrt(3 * off.numel())


@pytest.mark.parametrize("dtype", HALVES)
def test_long_sums_of_one_sign(ly, dtype):
    """2^18 summed elements: in one go the tensor cores would cut off some 1.7e-3."""
    n, o = 1 << 18, offs(0, 30, 40)
    x, w = positive(1, 40, n, dtype, 1), positive(2, 144, n, dtype, 1).view(2, 72, n)
    y = ly.expert_matmul(x, w, o)
    dx = ly.expert_matmul_grad_input(x, w.transpose(1, 2), o)  # the same sums, features contiguous or not
    dx2 = ly.expert_matmul_grad_input(x, w.transpose(1, 2).contiguous(), o)
    exact = torch.cat([x[:30].double() @ w[0].double().t(), x[30:].double() @ w[1].double().t()])
    for t in (y, dx, dx2):
        assert_not_cut_off(t, exact)
    x, dy = positive(3, 72, n + 5000, dtype, 0), positive(4, 136, n + 5000, dtype, 0)
    dw = ly.expert_matmul_grad_weight(dy, x, offs(0, 4999, n + 4999))
    assert_not_cut_off(dw[1], dy[4999:-1].double().t() @ x[4999:-1].double())
    assert_not_cut_off(dw[0], dy[:4999].double().t() @ x[:4999].double())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("length", [8192, 8193, 16_384, 24_600])
def test_sums_around_a_round(ly, dtype, length):
    """One round, one element more, and several, of all three products."""
    for rows, N, K, o in ((70, 136, length, (0, 3, 70)), (70, length, 72, (0, 3, 70)),
                          (2 * length + 9, 136, 72, (5, length + 5, length + 6, 2 * length + 6))):
        x, w, dy = operands(7, rows, len(o) - 1, N, K, dtype)
        check(ly, x, w, dy, offs(*o))


def test_long_sums_repeat_and_do_not_mix(ly):
    """More tiles than pairs of SMs, each of several rounds: equal calls give equal bits, and each
    tile's sums are its own."""
    rows, N, K = 18_000, 2600, 2300
    x, w, dy = operands(11, rows, 1, N, K, torch.bfloat16)
    o = offs(0, rows)
    dw = ly.expert_matmul_grad_weight(dy, x, o)
    assert torch.equal(dw, ly.expert_matmul_grad_weight(dy, x, o))
    exact = dy.double().t() @ x.double()
    bound = (rows + 2) * lo.EPS * (dy.double().abs().t() @ x.double().abs())
    lo.assert_within(dw[0], exact.cpu(), bound.cpu(), "dw")
    x, w = normal(13, 3000, 18_000, dtype=torch.bfloat16), normal(14, 1, 3000, 18_000, dtype=torch.bfloat16)
    o = offs(0, 3000)
    y = ly.expert_matmul(x, w, o)
    assert torch.equal(y, ly.expert_matmul(x, w, o))
    exact = x.double() @ w[0].double().t()
    bound = 18_002 * lo.EPS * (x.double().abs() @ w[0].double().abs().t())
    lo.assert_within(y, exact.cpu(), bound.cpu(), "y")


@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("rows", [4, 5, 64, 65, 300])
@pytest.mark.parametrize("depth", [32, 63, 64, 256])
def test_own_infinities(ly, dtype, rows, depth):
    """Infinities and NaN among an expert's own operands give the infinities and NaN of the
    definition, whichever kernel the sizes choose; the other outputs are as without them. Factors
    of 1, whose low part is zero, and of 0 among them."""
    x, w, dy = operands(17, rows, 2, depth, depth, dtype)
    o, edge = offs(0, rows - 1, rows), float("inf")
    for t in (x, w[0], dy):
        t[0, :4] = torch.tensor([1.0, 0.0, -1.0, 0.5])
        t[:, 2] = 1.0
    plain = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), o.tolist(), rows)
    x[1, 3], x[2, 5], x[2, 7] = edge, -edge, float("nan")
    dy[1, 4], dy[2, 6] = -edge, edge
    w[0, 1, 2], w[0, 9, 11] = edge, -edge
    exact = lo.expert_products(lo.d64(x), lo.d64(w), lo.d64(dy), o.tolist(), rows)
    got = {"y": ly.expert_matmul(x, w, o), "dx": ly.expert_matmul_grad_input(dy, w, o),
           "dw": ly.expert_matmul_grad_weight(dy, x, o)}
    for k, t in got.items():
        want = exact[k][0]
        assert torch.equal(torch.isnan(lo.d64(t)), torch.isnan(want)), k
        far = torch.isinf(want)
        assert torch.equal(lo.d64(t)[far], want[far]), k
        near = torch.isfinite(want)
        lo.assert_within(t.cpu()[near], plain[k][0][near], plain[k][1][near], k)


def test_floats_whose_products_pass_the_largest(ly):
    """3e19 x 3e19 is past the largest float: an infinity of its sign, not a NaN."""
    rows, depth = 300, 256
    x, w, dy = operands(19, rows, 1, depth, depth, torch.float32)
    big = 3.1415926e19
    x[5, 3], w[0, 7, 3], dy[5, 7] = -big, big, big
    o = offs(0, rows)
    assert float(ly.expert_matmul(x, w, o)[5, 7]) == -float("inf")
    assert float(ly.expert_matmul_grad_input(dy, w, o)[5, 3]) == float("inf")
    assert float(ly.expert_matmul_grad_weight(dy, x, o)[0, 7, 3]) == -float("inf")


@pytest.mark.parametrize("depth,sign", [(64, "both"), *[(d, s) for d in (96, 128, 200, 512, 2048) for s in ("both", "one")]])
def test_floats_lose_no_more_than_a_sum_in_floats(ly, depth, sign):
    """The root mean square error of float products in parts is below that of a 32-bit sum of one
    product after another, on the same operands; of one sign, from 96 summed elements on."""
    g = torch.Generator(device="cuda").manual_seed(depth)
    draw = torch.randn if sign == "both" else torch.rand
    a, b = (draw(512, depth, generator=g, device="cuda") for _ in range(2))
    exact = a.double() @ b.double().t()
    plain = torch.zeros(512, 512, device="cuda")
    for k in range(depth):
        plain = torch.addcmul(plain, a[:, k:k + 1], b[:, k][None])
    off = lambda t: float((t.double() - exact).norm() / exact.norm())
    o = offs(0, 512)
    for got in (ly.expert_matmul(a, b[None], o), ly.expert_matmul_grad_input(a, b.t()[None].contiguous(), o),
                ly.expert_matmul_grad_weight(a.t().contiguous(), b.t().contiguous(), offs(0, depth))[0]):
        assert off(got) <= off(plain), (off(got), off(plain))


def test_a_product_of_seconds(ly):
    """One expert of 640 million rows, whose one tile takes longer than a wait may: the waits of
    every warp go on as long as the tile's copies do. Terms of one sign: some 78,000 rounds are added
    up, each within 2^-24."""
    rows, n = 640_000_003, 8
    x, dy = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(23)
    x.uniform_(0.25, 1, generator=g)
    dy.uniform_(0.25, 1, generator=g)
    dw = ly.expert_matmul_grad_weight(dy, x, offs(0, rows))
    ly.check_status()
    exact = torch.zeros(n, n, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 1 << 24):
        exact += dy[i:i + (1 << 24)].double().t() @ x[i:i + (1 << 24)].double()
    off = (dw[0].double() - exact) / exact
    assert float(off.abs().max()) <= lo.UNIT[torch.bfloat16] + 2.0 ** -14 + 78_200 * 2.0 ** -24
