"""Attention of halves on the GPU, whose exponents are few: flat tails of long rows, keys of little weight.

Bounds. P is held 2^7 times larger forward (2^14 in the gradient): what lies below 2^-14 of that is rounded in steps
of 2^-24 of it, so a term is off by 2^-32 (2^-39) of the row's largest at most, besides half's rounding u = 2^-11."""
import math

import pytest
import torch

import layer_oracle as lo
from test_gpu_attention import BF, HF, ly, offs  # noqa: F401

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
