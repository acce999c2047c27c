"""Causal attention of packed sequences on the GPU against its definition in 64 bits, within bounds
derived in attention_oracle: types, head sizes and sharing, lengths, strides, offsets of any kind,
values that a mask hides, streams, graphs, far addresses; refusals."""
import math

import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
DTYPES = [BF, HF, FL]


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    yield layers
    layers.check_status()


def normal(seed, *shape, dtype=FL, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(dtype)


def offs(*v):
    return torch.tensor(v, dtype=torch.int64, device="cuda")


def packed(*lengths):
    o = [0]
    for n in lengths:
        o.append(o[-1] + n)
    return o


def operands(seed, T, H, G, D, dtype, scale=1.2):
    return (normal(seed, T, H, D, dtype=dtype, scale=scale), normal(seed + 1, T, G, D, dtype=dtype, scale=scale),
            normal(seed + 2, T, G, D, dtype=dtype), normal(seed + 3, T, H, D, dtype=dtype))


def both(ly, q, k, v, dy, o, scale=None, **how):
    y, lse = ly.attention(q, k, v, o, scale=scale, **how)
    return dict(zip(("y", "lse", "dq", "dk", "dv"),
                    (y, lse) + ly.attention_grad(dy, q, k, v, y, lse, o, scale=scale, **how)))


def check(got, q, k, v, dy, offsets, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want = ao.attention(q.double(), k.double(), v.double(), offsets, scale, dy.double(), got["y"].double(), q.dtype)
    for n, (value, bound) in want.items():
        lo.assert_within(got[n], value, bound, n)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G,D", [(1, 1, 128), (2, 1, 64), (4, 2, 128), (3, 3, 64), (3, 1, 80), (6, 2, 16), (2, 2, 120),
                                   (8, 1, 128)])
@pytest.mark.parametrize("lengths", [(1,), (130, 1, 257), (5, 64, 63, 128, 65)])
def test_sizes(ly, dtype, H, G, D, lengths):
    o = packed(*lengths)
    q, k, v, dy = operands(10 * H + D, o[-1], H, G, D, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [1, 2, 7, 33, 65, 99, 127])
def test_odd_heads(ly, dtype, D):
    o = packed(3, 129, 70)
    q, k, v, dy = operands(D, o[-1], 4, 2, D, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("n", list(range(1, 9)) + [31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511,
                                                    512, 513, 640])
def test_lengths(ly, n):
    for dtype, H, G, D in ((BF, 2, 1, 128), (HF, 1, 1, 64), (HF, 3, 1, 128)):
        q, k, v, dy = operands(n, n, H, G, D, dtype)
        check(both(ly, q, k, v, dy, offs(0, n)), q, k, v, dy, [0, n])


@pytest.mark.parametrize("dtype,H,G,D", [(BF, 4, 1, 128), (HF, 2, 2, 64), (HF, 3, 1, 128), (FL, 2, 1, 64)])
def test_long(ly, dtype, H, G, D):
    o = packed(2200, 1111, 1793)
    q, k, v, dy = operands(77, o[-1], H, G, D, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("dtype,H,G,D", [(BF, 12, 4, 128), (HF, 9, 3, 64), (HF, 16, 8, 128), (BF, 8, 2, 64), (FL, 8, 2, 48),
                                          (HF, 10, 2, 72)])
def test_many_items(ly, dtype, H, G, D):
    """Several times as many tiles as SMs: each block takes one after another, of long and short sequences."""
    g = torch.Generator().manual_seed(8)
    o = packed(*torch.randint(1, 600, (50,), generator=g).tolist(), 1300)
    q, k, v, dy = operands(9, o[-1], H, G, D, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G", [(7, 1), (16, 1), (5, 5), (64, 2)])
def test_few_key_heads(ly, dtype, H, G):
    """A group's heads dealt to several blocks, evenly and unevenly."""
    o = packed(140, 300, 3)
    q, k, v, dy = operands(H, o[-1] + 9, H, G, 64, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_sequences(ly, dtype):
    """More sequences than a block of the plan takes at a time, empty ones among them."""
    g = torch.Generator().manual_seed(3)
    o = packed(*torch.randint(0, 5, (2500,), generator=g).tolist())
    q, k, v, dy = operands(5, o[-1], 2, 1, 64, dtype)
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offsets", [[0], [7], [0, 0, 0], [40, 200, 200, 300], [-5, 100, 90, 260, 1000], [300, 300],
                                     [2**62, 5, 2**63 - 1], [-2**63, 150], [150, -2**63, 299]])
def test_offsets_of_any_kind(ly, dtype, offsets):
    """Rows of no sequence get zeros; offsets out of range or out of order count as the nearest valid."""
    q, k, v, dy = operands(21, 300, 4, 2, 64, dtype)
    got = both(ly, q, k, v, dy, offs(*offsets))
    check(got, q, k, v, dy, offsets)
    o = lo.clean_offsets(offsets, 300)
    for n, t in got.items():
        t = t.t() if n == "lse" else t
        assert not t[:o[0]].any() and not t[o[-1]:].any()


def test_no_tokens(ly):
    for dtype in DTYPES:
        q, k, v, dy = operands(1, 0, 4, 2, 64, dtype)
        got = both(ly, q, k, v, dy, offs(0, 0))
        assert [tuple(t.shape) for t in got.values()] == [(0, 4, 64), (4, 0), (0, 4, 64), (0, 2, 64), (0, 2, 64)]


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(ly, dtype):
    """Slices of one projection's output, heads before tokens, rows off 16-byte boundaries: the
    same bits as of contiguous copies."""
    T, H, G, D = 333, 4, 2, 64
    o = offs(0, 100, 333)
    fused = normal(1, T, H + 2 * G, D, dtype=dtype)
    dy = normal(2, T, H, D, dtype=dtype)
    odd = normal(3, T, (H + 2 * G) * D + 3, dtype=dtype)[:, 1:1 + (H + 2 * G) * D].unflatten(1, (H + 2 * G, D))
    across = normal(4, H + 2 * G, T, D, dtype=dtype).transpose(0, 1)
    for x in (fused, odd, across):
        q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
        a = both(ly, q, k, v, dy, o)
        b = both(ly, q.contiguous(), k.contiguous(), v.contiguous(), dy, o)
        assert all(torch.equal(a[n], b[n]) for n in a)
    # heads of 75 elements 80 apart: aligned as they are; the same bits as of copies
    wide = normal(6, T, H + 2 * G, 80, dtype=dtype)[..., :75]
    q, k, v, d75 = wide[:, :H], wide[:, H:H + G], wide[:, H + G:], normal(7, T, H, 75, dtype=dtype)
    a = both(ly, q, k, v, d75, o)
    b = both(ly, q.contiguous(), k.contiguous(), v.contiguous(), d75, o)
    assert all(torch.equal(a[n], b[n]) for n in a)
    q, k, v = across[:, :H], across[:, H:H + G], across[:, H + G:]
    # a gradient that is contiguous but starts off 16-byte boundaries
    shifted = torch.empty(dy.numel() + 1, dtype=dtype, device="cuda")[1:].view(dy.shape).copy_(dy)
    assert all(torch.equal(x, y) for x, y in zip(both(ly, q, k, v, shifted, o).values(), both(ly, q, k, v, dy, o).values()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.0, 0.5, -0.3, 4.0])
def test_scale(ly, dtype, scale):
    o = packed(150, 133)
    q, k, v, dy = operands(31, o[-1], 2, 1, 64, dtype, scale=0.7)
    check(both(ly, q, k, v, dy, offs(*o), scale=scale), q, k, v, dy, o, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rising_scores(ly, dtype):
    """Each block of keys raises the rows' largest score by far (or lowers it)."""
    n = 700
    for up in (1.0, -1.0):
        q, k, v, dy = operands(41, n, 2, 1, 64, dtype, scale=0.3)
        k[:, :, 0] = (up * torch.arange(n, device="cuda") / 16).to(dtype)[:, None]
        q[:, :, 0] = 4.0
        check(both(ly, q, k, v, dy, offs(0, n)), q, k, v, dy, [0, n])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_rows_of_others_do_not_matter(ly, dtype, what):
    """Infinities and NaN in rows of no sequence, and in another sequence, change no bit elsewhere."""
    q, k, v, dy = operands(51, 500, 4, 2, 64, dtype)
    o = offs(3, 200, 330, 460)
    want = both(ly, q, k, v, dy, o)
    for rows in (slice(0, 3), slice(460, 500), slice(200, 330)):
        for t in (q, k, v, dy):
            t[rows] = what
    got = both(ly, q, k, v, dy, o)
    for n in want:
        a, b = (t.t() if n == "lse" else t for t in (want[n], got[n]))
        for rows in (slice(0, 200), slice(330, 500)):
            assert torch.equal(a[rows], b[rows]), n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [(0,), (1,), (60, 61), (127, 128), (255,), (299,)])
def test_masked_values_do_not_matter(ly, dtype, D, at):
    """NaN in a key's or a row's own data stays where the mask lets it: y and dq of earlier rows, dk and
    dv of later keys are what they are without it, and finite."""
    n, scale = 300, D ** -0.5
    q, k, v, dy = operands(61, n, 2, 1, D, dtype)
    o = offs(0, n)
    first, last = min(at), max(at) + 1
    good_y, good_lse = ly.attention(q, k, v, o)
    want = ao.attention(q.double(), k.double(), v.double(), [0, n], scale, dy.double(), good_y.double(), dtype)
    for what in (math.nan, math.inf):
        k2, v2 = k.clone(), v.clone()
        k2[list(at)] = what
        v2[list(at)] = what
        y, lse = ly.attention(q, k2, v2, o)
        for got, name in ((y, "y"), (lse.t(), "lse")):
            value, bound = (t.t() if name == "lse" else t for t in want[name])
            lo.assert_within(got[:first], value[:first], bound[:first], name)
        assert not torch.isfinite(y[first:].float()).any()
        # of the gradient, y's rows before them: dq reads keys and values
        dq = ly.attention_grad(dy, q, k2, v2, good_y, good_lse, o)[0]
        lo.assert_within(dq[:first], want["dq"][0][:first], want["dq"][1][:first], "dq")
        # the rows of `at` have bad queries and gradients
        q2, dy2 = q.clone(), dy.clone()
        q2[list(at)] = what
        dy2[list(at)] = what
        dq, dk, dv = ly.attention_grad(dy2, q2, k, v, good_y, good_lse, o)
        for got, name in ((dk, "dk"), (dv, "dv")):
            lo.assert_within(got[last:], want[name][0][last:], want[name][1][last:], name)
        keep = torch.ones(n, dtype=torch.bool)
        keep[list(at)] = False
        lo.assert_within(dq[keep.cuda()], want["dq"][0][keep], want["dq"][1][keep], "dq")


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_scores(ly, dtype):
    """A key of -inf score counts as none; a row of nothing else has no value (NaN)."""
    n = 200
    q, k, v, dy = operands(71, n, 1, 1, 64, dtype, scale=0.5)
    q[:, :, 0] = 1.0
    k[:130, :, 0] = -math.inf
    y, lse = ly.attention(q, k, v, offs(0, n))
    assert torch.isnan(y[:130].float()).all() and (lse[:, :130] == -math.inf).all()
    # the rows after it see the keys from 130 on
    want = ao.attention(*(t[130:].double() for t in (q, k, v)), [0, n - 130], 64 ** -0.5, dtype=dtype)
    lo.assert_within(y[130:], *want["y"], "y")
    lo.assert_within(lse[:, 130:], *want["lse"], "lse")


def test_equal_calls_equal_bits(ly):
    for dtype in DTYPES:
        o = packed(700, 33, 400)
        q, k, v, dy = operands(81, o[-1], 8, 2, 64, dtype)
        a, b = (both(ly, q, k, v, dy, offs(*o)) for _ in range(2))
        assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", [BF, FL])
def test_small_gradients_keep_their_digits(ly, dtype):
    o = packed(513)
    q, k, v, dy = operands(91, 513, 2, 1, 64, dtype)
    dy = dy * 2.0 ** -12
    check(both(ly, q, k, v, dy, offs(*o)), q, k, v, dy, o)


def test_small_gradients_of_halves(ly):
    """dS of halves is held in a scale of its own: gradients of 2^-10 lose no digits but their rounding."""
    q, k, v, dy = operands(92, 513, 2, 1, 64, HF)
    dy = dy * 2.0 ** -10
    check(both(ly, q, k, v, dy, offs(0, 513)), q, k, v, dy, [0, 513])
    big = (dy * 2.0 ** 20).clamp(-6e4, 6e4)
    v = v * 8
    y, lse = ly.attention(q, k, v, offs(0, 513))
    want = ao.attention(q.double(), k.double(), v.double(), [0, 513], 64 ** -0.5, big.double(), y.double(), HF)
    got = dict(zip(("dq", "dk", "dv"), ly.attention_grad(big, q, k, v, y, lse, offs(0, 513))))
    for n in got:
        value, bound = want[n]
        ok = value.abs() + bound < 6e4  # what halves can hold
        g = got[n].cpu().double()
        assert float(((g - value).abs() - (lo.UNIT[HF] * (value.abs() + bound) + bound))[ok].max()) <= 0, n


@pytest.mark.parametrize("dtype", [BF, HF])
def test_gradient_does_not_feel_how_y_was_rounded(ly, dtype):
    """Short rows, whose y is large: y off by four roundings gives the gradients of the exact one."""
    o = packed(*[7] * 30, 60)
    q, k, v, dy = operands(93, o[-1], 4, 2, 64, dtype)
    y, lse = ly.attention(q, k, v, offs(*o))
    worse = (y.float() * (1 + 4 * lo.UNIT[dtype])).to(dtype)
    got = dict(zip(("dq", "dk", "dv"), ly.attention_grad(dy, q, k, v, worse, lse, offs(*o))))
    want = ao.attention(q.double(), k.double(), v.double(), o, 64 ** -0.5, dy.double(), worse.double(), dtype)
    for n in got:
        lo.assert_within(got[n], *want[n], n)


@pytest.mark.parametrize("dtype", DTYPES)
def test_against_differences(ly, dtype):
    """The definition's own gradients (which the kernels are tested against) against differences."""
    o = [0, 5, 12]
    q, k, v, dy = (t.double().cpu() for t in operands(95, 12, 4, 2, 8, dtype))
    f = lambda q, k, v: float((ao.attention(q, k, v, o, 0.4)["y"][0] * dy).sum())
    want = ao.attention(q, k, v, o, 0.4, dy)
    for i, n in enumerate(("dq", "dk", "dv")):
        for at in ((0, 0, 0), (4, 1, 3), (7, 1, 7), (11, 0, 2)):
            args = [q, k, v]
            d = []
            for step in (1e-5, -1e-5):
                t = args[i].clone()
                t[at] += step
                d.append(f(*args[:i], t, *args[i + 1:]))
            assert abs((d[0] - d[1]) / 2e-5 - float(want[n][0][at])) < 1e-7


def test_streams_and_graphs(ly):
    o = offs(0, 300, 777)
    q, k, v, dy = operands(101, 777, 4, 2, 128, BF)
    want = both(ly, q, k, v, dy, o)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(ly, q, k, v, dy, o, stream=side)
    with torch.cuda.stream(side):
        also = both(ly, q, k, v, dy, o)
    side.synchronize()
    assert all(torch.equal(want[n], got[n]) and torch.equal(want[n], also[n]) for n in want)
    # captured; replayed with other values and lengths
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(ly, q, k, v, dy, o)
    second = torch.cuda.CUDAGraph()
    with torch.cuda.graph(second, pool=graph.pool()):
        out2 = both(ly, q, k, v, dy, o)
    for lengths in ((300, 477), (1, 700)):
        o.copy_(offs(0, lengths[0], sum(lengths)))
        q.mul_(0.5)
        ref = both(ly, q, k, v, dy, o)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(ref[n], out[n]) for n in ref)
        second.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(ref[n], out2[n]) for n in ref)


def test_far_addresses(ly):
    """More than 2^31 elements: the last rows are those of a short call on them."""
    T, H, D = 150_000, 120, 128
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory")
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.empty(s, dtype=BF, device="cuda").normal_(generator=g)
    q, dy, k, v = make(T, H, D), make(T, H, D), make(T, H, D), make(T, H, D)
    o = torch.arange(0, T + 1, 125, device="cuda")
    got = both(ly, q, k, v, dy, o)
    last = slice(T - 250, T)
    small = both(ly, *(t[last].contiguous() for t in (q, k, v, dy)), offs(0, 125, 250))
    for n in got:
        if n == "lse":
            assert torch.equal(got[n][:, last], small[n])
        else:
            assert torch.equal(got[n][last], small[n]), n


def test_chain_with_head_norms(ly):
    """Norms, rotation and attention as they are used together: y and the gradients of the projection's
    output through both, against 64 bits."""
    T, H, G, D = 190, 4, 2, 64
    o = packed(60, 130)
    pos = torch.cat([torch.arange(60), torch.arange(130)]).cuda()
    x = normal(1, T, H + 2 * G, D, dtype=FL)
    wq, wk = normal(2, D, scale=0.1, shift=1.0), normal(3, D, scale=0.1, shift=1.0)
    dy = normal(4, T, H, D)
    q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    qr, kr = ly.head_norm_rotary(q, k, pos, wq, wk)
    y, lse = ly.attention(qr, kr, v, offs(*o))
    dqr, dkr, dv = ly.attention_grad(dy, qr, kr, v, y, lse, offs(*o))
    r = ly.head_norm_rotary_grad(dqr, dkr, q, k, pos, wq, wk)
    d = [t.double().cpu() for t in (q, k, v, wq, wk, dy)]
    for t in d[:5]:
        t.requires_grad_()
    p = pos.cpu()
    qe = ao.rotary_forward(d[0], d[3], p, D, 10000.0, False, True, 1e-6)
    ke = ao.rotary_forward(d[1], d[4], p, D, 10000.0, False, True, 1e-6)
    outs = []
    for a, b in zip(o[:-1], o[1:]):
        kk, vv = (t[a:b].repeat_interleave(H // G, 1) for t in (ke, d[2]))
        s = torch.einsum("ihd,jhd->hij", qe[a:b], kk) * D ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -math.inf)
        outs.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), vv))
    ye = torch.cat(outs)
    (ye * d[5]).sum().backward()
    # floats: some hundred operations on the way, sums of up to 130 terms
    for got, want in ((y, ye.detach()), (r["dq"], d[0].grad), (r["dk"], d[1].grad), (dv, d[2].grad),
                      (r["dw_q"], d[3].grad), (r["dw_k"], d[4].grad)):
        assert float((got.cpu().double() - want).abs().max()) < 1000 * lo.EPS * float(want.abs().max())


def test_refusals(ly):
    q, k, v, dy = operands(1, 20, 4, 2, 32, BF)
    o = offs(0, 20)
    y, lse = ly.attention(q, k, v, o)
    bad = [dict(q=q.float()), dict(k=k[:19]), dict(v=v[:, :, :16]), dict(k=k[:, :1]), dict(q=q[:, :3]), dict(q=q.cpu()),
           dict(q=q.transpose(1, 2)), dict(offsets=o.int()), dict(offsets=o.cpu()), dict(offsets=o[None]),
           dict(q=q[0]), dict(q=q.double(), k=k.double(), v=v.double()), dict(k=k[:, :0], v=v[:, :0])]
    args = dict(q=q, k=k, v=v, offsets=o)
    for b in bad:
        with pytest.raises(ValueError):
            ly.attention(**{**args, **b})
        with pytest.raises(ValueError):
            ly.attention_grad(dy, **{**args, **b}, y=y, lse=lse)
    for b in (dict(dy=dy[:, :2]), dict(dy=dy.float()), dict(y=y[:10]), dict(lse=lse.half()), dict(lse=lse.t().contiguous()),
              dict(dy=dy.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            ly.attention_grad(**{**dict(dy=dy, y=y, lse=lse), **b}, **args)
    from paper_2101_07968_gb300 import dynacomm as dc
    wide = operands(2, 20, 2, 1, 129, BF)
    with pytest.raises(dc.DynaCommError):
        ly.attention(*wide[:3], o)
    with pytest.raises(dc.DynaCommError):
        ly.attention(q, k, v, o, scale=math.nan)
    with pytest.raises(dc.DynaCommError):  # every head the same elements
        ly.attention(q[:, :1].expand(20, 4, 32), k, v, o)
    for name, t in (("q", q), ("k", k), ("v", v)):
        with pytest.raises(ValueError, match="gradient"):
            ly.attention(**{**args, name: t.clone().requires_grad_()})
        with pytest.raises(ValueError, match="gradient"):
            ly.attention_grad(dy, **{**args, name: t.clone().requires_grad_()}, y=y, lse=lse)
