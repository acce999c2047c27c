"""Attention of halves on the GPU, whose exponents are few: flat tails of long rows, and gradients beside others that
are larger by orders of magnitude, in other sequences, heads, later keys and earlier rows.

Bounds. P is held 2^7 times larger forward (2^14 in the gradient): what lies below 2^-14 of that is rounded in steps
of 2^-24 of it, so a term is off by 2^-32 (2^-39) of the row's largest at most, besides half's rounding u = 2^-11.
dS is held in a power of two that follows from what an output may see and nothing else: whatever it may not see leaves
its bits as they are."""
import math

import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo
from test_gpu_attention import BF, HF, both, ly, normal, offs, operands, packed  # noqa: F401

pytestmark = pytest.mark.gpu
U = lo.UNIT[HF]


def peaked(n, ahead, at, dtype, D=64, heads=1):
    """Queries and keys of score 0, but for the key `at`, `ahead` in front of the rest; its value is zero, the others' one."""
    q, k, v = (torch.zeros(n, h, D, dtype=dtype, device="cuda") for h in (heads, 1, 1))
    q[:, :, 0] = 4.0
    k[at, 0, 0] = ahead * D ** 0.5 / 4.0
    v[:] = 1.0
    v[at] = 0.0
    return q, k, v, float(k[at, 0, 0]) * 4.0 * D ** -0.5


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,ahead", [(16384, 12.0), (16384, 15.0), (16384, 17.0), (16384, 17.4), (40000, 18.0), (262144, 17.4)])
def test_flat_tails(ly, dtype, heads, D, n, ahead):  # noqa: F811
    for at in (0, 5000):
        q, k, v, ahead_held = peaked(n, ahead, at, dtype, D, heads)
        y, lse = ly.attention(q, k, v, offs(0, n))
        rows = torch.arange(n - 200, n, dtype=torch.float64)
        tail = rows * math.exp(-ahead_held)
        want = (tail / (1 + tail))[:, None, None].expand(200, heads, D)
        # the scores are exact or off by 20 steps of 2^-23; sums of 16 terms a step lose 2^-24 each at most
        rel = 2.0 ** -22 * 20 + n / 16 * 2.0 ** -24
        bound = want * (rel + lo.UNIT[dtype]) + (n * 2.0 ** -32 if dtype is HF else 0.0)
        lo.assert_within(y[-200:], want, bound, "y")
        exact = ahead_held + torch.log1p(tail)
        lo.assert_within(lse[:, -200:].t(), exact[:, None].expand(200, heads), exact[:, None] * 2.0 ** -21 + rel, "lse")


def test_values_of_faint_keys(ly):  # noqa: F811
    """A key that every row all but overlooks: P = e^-20, of which halves would hold no digit."""
    n, D = 3000, 64
    q, k, v, _ = peaked(n, -20.0, 0, HF)
    dy = torch.full((n, 1, D), 1000.0, dtype=HF, device="cuda")
    y, lse = ly.attention(q, k, v, offs(0, n))
    dv = ly.attention_grad(dy, q, k, v, y, lse, offs(0, n))[2]
    rows = torch.arange(1, n, dtype=torch.float64)
    far = float(k[0, 0, 0]) * 4.0 / 8.0
    p = math.exp(far) / (rows + math.exp(far))
    want = (1000.0 * (1.0 + p.sum())).expand(D)  # the first row sees nothing else
    lo.assert_within(dv[0, 0], want, want * (U + n * 2.0 ** -24), "dv of the first row's key")
    # two keys, the first of which has weight one in its own row: leave that row's gradient out
    dy[0] = 0.0
    dv = ly.attention_grad(dy, q, k, v, y, lse, offs(0, n))[2]
    want = (1000.0 * p.sum()).expand(D)
    lo.assert_within(dv[0, 0], want, want * (U + n * 2.0 ** -22) + 1000.0 * n * 2.0 ** -39, "dv")


def gradients(ly, q, k, v, dy, o):  # noqa: F811
    y, lse = ly.attention(q, k, v, offs(*o))
    return y, dict(zip(("dq", "dk", "dv"), ly.attention_grad(dy, q, k, v, y, lse, offs(*o))))


def small(D=64, H=4, G=2):
    o = packed(300, 500, 224)
    q, k, v, dy = operands(17, o[-1], H, G, D, HF)
    return o, q, k, v, dy * 1e-3


@pytest.mark.parametrize("D", [64, 128, 75])
@pytest.mark.parametrize("big_dy,big_v", [(100.0, 20.0), (1000.0, 60.0), (60000.0, 1.0), (60000.0, 60000.0)])
def test_large_values_of_another_sequence(ly, D, big_dy, big_v):  # noqa: F811
    """Finite ones, of the magnitudes that halves hold: no bit of the others' gradients changes, and each
    sequence's are within the bounds of a call of its own."""
    o, q, k, v, dy = small(D)
    _, want = gradients(ly, q, k, v, dy, o)
    for a, b in ((300, 800), (800, 1024)):
        v2, dy2 = v.clone(), dy.clone()
        v2[a:b] = (normal(3, b - a, v.shape[1], D) * big_v).clamp(-6e4, 6e4).half()
        dy2[a:b] = (normal(4, b - a, q.shape[1], D) * big_dy).clamp(-6e4, 6e4).half()
        y, got = gradients(ly, q, k, v2, dy2, o)
        for s, e in zip(o[:-1], o[1:]):
            if s == a:
                continue
            for n in got:
                assert torch.equal(got[n][s:e], want[n][s:e]), (n, s)
            own = ao.attention(*(t[s:e].double() for t in (q, k, v)), [0, e - s], D ** -0.5, dy[s:e].double(),
                               y[s:e].double(), HF)
            for n in got:
                lo.assert_within(got[n][s:e], *own[n], n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("big", [100.0, 6e4])
def test_large_values_of_another_head(ly, D, big):  # noqa: F811
    """Key head 1 and the query heads that read it: those of key head 0 keep their bits."""
    o, q, k, v, dy = small(D)
    _, want = gradients(ly, q, k, v, dy, o)
    v[:, 1] = big
    dy[:, 2:] = big
    _, got = gradients(ly, q, k, v, dy, o)
    assert torch.equal(got["dq"][:, :2], want["dq"][:, :2])
    assert torch.equal(got["dk"][:, 0], want["dk"][:, 0]) and torch.equal(got["dv"][:, 0], want["dv"][:, 0])
    # a query head alone: the other's dq, which shares its keys
    dy2 = dy.clone()
    dy2[:, 0] = big
    _, one = gradients(ly, q, k, v, dy2, o)
    assert torch.equal(one["dq"][:, 1], want["dq"][:, 1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [1, 127, 128, 200, 499])
@pytest.mark.parametrize("big", [100.0, 6e4])
def test_large_values_behind_the_mask(ly, D, at, big):  # noqa: F811
    """Of a later key: earlier rows' dq; of an earlier row: later keys' dk and dv."""
    o = [0, 500]
    q, k, v, dy = operands(19, 500, 4, 2, D, HF)
    dy = dy * 1e-3
    _, want = gradients(ly, q, k, v, dy, o)
    v2 = v.clone()
    v2[at] = big
    _, got = gradients(ly, q, k, v2, dy, o)
    assert torch.equal(got["dq"][:at], want["dq"][:at])
    dy2 = dy.clone()
    dy2[at] = big
    _, got = gradients(ly, q, k, v, dy2, o)
    assert torch.equal(got["dk"][at + 1:], want["dk"][at + 1:]) and torch.equal(got["dv"][at + 1:], want["dv"][at + 1:])
    # rows apart from it: dq is a row's own
    other = torch.arange(500, device="cuda") != at
    assert torch.equal(got["dq"][other], want["dq"][other])


@pytest.mark.parametrize("power", [-22, -12, 0, 10])
@pytest.mark.parametrize("D", [64, 128])
def test_gradients_of_any_size(ly, D, power):  # noqa: F811
    """Every row, head and sequence in a magnitude of its own."""
    o = packed(200, 1, 431)
    q, k, v, dy = operands(23, o[-1], 4, 2, D, HF, scale=0.8)
    dy = (dy.float() * torch.exp2(torch.randint(-2, 3, (o[-1], 4, 1), device="cuda") + float(power))).half()
    y, got = gradients(ly, q, k, v, dy, o)
    want = ao.attention(*(t.double() for t in (q, k, v)), o, D ** -0.5, dy.double(), y.double(), HF)
    for n in got:
        lo.assert_within(got[n], *want[n], n)


@pytest.mark.parametrize("zero", ["dy", "v", "both"])
def test_gradients_of_zeros(ly, zero):  # noqa: F811
    o, q, k, v, dy = small()
    if zero != "v":
        dy.zero_()
    if zero != "dy":
        v.zero_()
    y, got = gradients(ly, q, k, v, dy, o)
    assert not got["dq"].any() and not got["dk"].any()
    assert zero == "v" or not got["dv"].any()


def test_captured(ly):  # noqa: F811
    """The gradient's powers of two follow the values of a replay, and the lengths."""
    o, q, k, v, dy = small()
    o = offs(*o)
    y, lse = ly.attention(q, k, v, o)
    ly.attention_grad(dy, q, k, v, y, lse, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, lse = ly.attention(q, k, v, o)
        out = ly.attention_grad(dy, q, k, v, y, lse, o)
    for lengths, by in ((None, 1.0), ((500, 300, 200), 3e4), ((1, 2, 1000), 1e-7)):
        if lengths:
            o.copy_(offs(*packed(*lengths)))
        dy.copy_((dy.float() * by).clamp(-6e4, 6e4))
        graph.replay()
        want_y, want_lse = ly.attention(q, k, v, o)
        want = ly.attention_grad(dy, q, k, v, want_y, want_lse, o)
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("H,G", [(16, 1), (7, 1)])
def test_large_values_of_another_sequence_in_parts(ly, H, G):  # noqa: F811
    """The same where a group's heads are dealt to several blocks."""
    o, D = packed(200, 130), 64
    q, k, v, dy = operands(29, o[-1], H, G, D, HF)
    dy = dy * 1e-3
    _, want = gradients(ly, q, k, v, dy, o)
    v[200:], dy[200:] = 6e4, 6e4
    _, got = gradients(ly, q, k, v, dy, o)
    assert all(torch.equal(got[n][:200], want[n][:200]) for n in got)


def test_two_streams_at_once(ly):  # noqa: F811
    """Two gradients on two streams, their kernels mixed."""
    o, q, k, v, dy = small(128)
    y, want = gradients(ly, q, k, v, dy, o)
    lse = ly.attention(q, k, v, offs(*o))[1]
    other = (dy.float() * 1e4).half()
    want2 = ly.attention_grad(other, q, k, v, y, lse, offs(*o))
    at = offs(*o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, d in enumerate((dy, other)):
            got[i].append(ly.attention_grad(d, q, k, v, y, lse, at, stream=streams[i]))
    torch.cuda.synchronize()
    for r in got[0]:
        assert all(torch.equal(a, want[n]) for a, n in zip(r, ("dq", "dk", "dv")))
    for r in got[1]:
        assert all(torch.equal(a, b) for a, b in zip(r, want2))
