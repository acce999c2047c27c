"""The rotation of far positions on the GPU, up to the ends of 64 bits, against angles from 80 decimal digits."""
from decimal import Decimal, getcontext, localcontext

import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo
from test_gpu_head_norm import DTYPES, ly, operands  # noqa: F401

pytestmark = pytest.mark.gpu
FAR = [2**31, 2**40 + 12345, 2**45 - 1, -2**45, 2**50 + 1, 2**53 + 1, -2**58 + 77, 2**62 - 5, 2**63 - 1, -2**63]


def pi():
    """Machin's sum of arc tangents, in the context's digits."""
    def arctan(n):
        x = Decimal(1) / n
        total, term, k = x, x, 1
        while abs(term) > Decimal(10) ** -(getcontext().prec + 2):
            term = -term / (n * n)
            k += 2
            total += term / k
        return total
    return 4 * (4 * arctan(5) - arctan(239))


def angles(positions, rotary, base):
    """[positions, rotary / 2] in doubles: what is left of a turn, in radians, nearest to zero."""
    with localcontext() as c:
        c.prec = 80
        turn = 2 * pi()
        rows = []
        for p in positions:
            row = []
            for i in range(rotary // 2):
                t = Decimal(p) * Decimal(base) ** (Decimal(-2 * i) / Decimal(rotary)) / turn
                t -= t.to_integral_value()
                row.append(float(t * turn))
            rows.append(row)
    return torch.tensor(rows, dtype=torch.float64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,rotary,interleaved", [(64, 64, False), (128, 128, True), (65, 62, False), (256, 256, False)])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1e-3, 0.7, 1e30])
def test_far_positions(ly, dtype, D, rotary, interleaved, base):  # noqa: F811
    """An angle is off by what 32 bits of a turn and the sines' floats cost, 4 steps of 2^-23, wherever it is."""
    T = len(FAR)
    q, k, _, _, dq, dk = operands(3, T, 2, 1, D, dtype)
    pos = torch.tensor(FAR, device="cuda")
    a = angles(FAR, rotary, base)
    how = dict(rotary=rotary, base=base, interleaved=interleaved, norm=False)
    got = ly.head_norm_rotary(q, k, pos, **how)[0]
    back = ly.head_norm_rotary_grad(dq, dk, q, k, pos, **how)["dq"]
    e, f = ao._pairs(rotary, interleaved)
    for x, y, sign in ((lo.d64(q), got, 1.0), (lo.d64(dq), back, -1.0)):
        c, s = torch.cos(a)[:, None], sign * torch.sin(a)[:, None]
        want, size = x.clone(), x.abs()
        want[..., e] = x[..., e] * c - x[..., f] * s
        want[..., f] = x[..., f] * c + x[..., e] * s
        size[..., e] = size[..., f] = x[..., e].abs() + x[..., f].abs()
        lo.assert_within(y, want, 8 * lo.EPS * size, "turned")
