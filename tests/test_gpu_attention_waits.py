"""Attention's gradient on the GPU where one item takes longer than a wait without progress may: 1,024 heads that read
one key head, 260,000 tokens, so that the first keys' tile takes some two and a half seconds."""
import pytest
import torch

import layer_oracle as lo
from test_gpu_attention import BF, ly, offs  # noqa: F401

pytestmark = pytest.mark.gpu


def test_items_of_seconds(ly):  # noqa: F811
    """No wait gives up while the work goes on. Queries and values of zero: P = 1 / (i + 1), and with gradients in the
    last 100 rows alone dv_j = sum of 1 / (i + 1) over those of them from j on and all heads, a sum of 102,400 terms (cut
    off by 2^-24 every 16 of them) of P rounded to bfloat16."""
    n, H, D, rows = 260_000, 1024, 8, 100
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    q = torch.zeros(n, H, D, dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.empty(n, 1, D, dtype=BF, device="cuda").normal_(generator=g)
    v, y, dy = torch.zeros_like(k), torch.zeros_like(q), torch.zeros_like(q)
    dy[-rows:] = 1.0
    lse = torch.log(torch.arange(1, n + 1, device="cuda", dtype=torch.float64)).float().expand(H, n).contiguous()
    dq, dk, dv = ly.attention_grad(dy, q, k, v, y, lse, offs(0, n))
    ly.check_status()
    assert not dq.any() and not dk.any()
    p = torch.zeros(n, dtype=torch.float64)
    p[-rows:] = 1.0 / torch.arange(n - rows + 1, n + 1, dtype=torch.float64)
    want = (H * p.flip(0).cumsum(0).flip(0))[:, None, None].expand(n, 1, D)
    # exponentials of lse near 12: 16 steps of 2^-23 of it
    lo.assert_within(dv, want, want * (lo.UNIT[BF] + H * rows / 16 * 2.0 ** -24 + 12 * 2.0 ** -19), "dv")
