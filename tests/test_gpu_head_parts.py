"""Head norms of few tokens, whose heads are dealt to several groups of lanes, on the GPU: head counts that no
power of two divides, of which the last group gets fewer, at the end of their buffers."""
import pytest
import torch

from test_gpu_head_norm import BF, DTYPES, FL, check, ly, operands  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G", [(3, 1), (5, 3), (6, 6), (12, 4), (24, 5), (40, 10), (63, 7), (513, 27)])
@pytest.mark.parametrize("T", [1, 2, 3, 33])
def test_few_tokens(ly, dtype, T, H, G):  # noqa: F811
    q, k, wq, wk, dq, dk = operands(H, T, H, G, 128, dtype)
    check(ly, q, k, torch.arange(T, device="cuda") + 7, wq, wk, dq, dk)


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("D", [40, 64, 256])
def test_same_bits_as_many_tokens(ly, dtype, D):  # noqa: F811
    """A token's result does not depend on how its heads are dealt."""
    T, H, G = 6000, 6, 5
    q, k, wq, wk, dq, dk = operands(3, T, H, G, D, dtype)
    pos = torch.arange(T, device="cuda")
    many, grads = ly.head_norm_rotary(q, k, pos, wq, wk), ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk)
    last = slice(T - 3, T)
    few = ly.head_norm_rotary(q[last], k[last], pos[last], wq, wk)
    some = ly.head_norm_rotary_grad(dq[last], dk[last], q[last], k[last], pos[last], wq, wk)
    assert all(torch.equal(a[last], b) for a, b in zip(many, few))
    assert all(torch.equal(grads[n][last], some[n]) for n in ("dq", "dk"))
