"""Head norms with rotation on the GPU: elements that do not turn keep to themselves, whatever stands in them, in
heads of any size and alignment."""
import math

import pytest
import torch

from test_gpu_head_norm import DTYPES, ly, normal, operands  # noqa: F401

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,rotary,aligned", [(64, 32, True), (64, 20, True), (64, 32, False), (65, 64, True), (50, 20, True),
                                              (130, 8, True), (255, 0, True)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_elements_past_the_rotation(ly, dtype, D, rotary, aligned, interleaved, what):  # noqa: F811
    """Without a norm an element past `rotary` is its weight times itself, and its neighbours are what they are
    without it; the same of its gradient."""
    T, H = 5, 3
    q, k, wq, wk, dq, dk = operands(D, T, H, 1, D, dtype)
    if not aligned:
        q = normal(1, T, H * D + 1, dtype=dtype)[:, 1:].unflatten(1, (H, D))
    pos = torch.arange(T, device="cuda") + 3
    how = dict(rotary=rotary, interleaved=interleaved, norm=False)
    at = [e for e in (rotary, rotary + 1, D - 1) if rotary <= e < D]
    q2, dq2 = q.clone(), dq.clone()
    if not aligned:
        q2 = torch.cat([q.flatten(1)[:, :1], q.flatten(1)], 1)[:, 1:].unflatten(1, (H, D))
    want, grad = ly.head_norm_rotary(q, k, pos, wq, wk, **how), ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk, **how)
    for e in at:
        for t in (q2, dq2):
            keep = t[2, 1, e].item()
            t[2, 1, e] = what
            got = ly.head_norm_rotary(q2, k, pos, wq, wk, **how)
            back = ly.head_norm_rotary_grad(dq2, dk, q, k, pos, wq, wk, **how)
            t[2, 1, e] = keep
            for name, a, b in (("q", got[0], want[0]), ("dq", back["dq"], grad["dq"])):
                hit = t is (q2 if name == "q" else dq2)
                assert torch.isfinite(a[2, 1, e].float()).item() != hit, name
                other = torch.ones(T, H, D, dtype=torch.bool, device="cuda")
                other[2, 1, e] = False
                assert torch.equal(bits(a)[other], bits(b)[other]), name
            others = torch.arange(D, device="cuda") != e
            assert torch.equal(back["dw_q"][others], grad["dw_q"][others])
            assert torch.equal(got[1], want[1]) and torch.equal(back["dk"], grad["dk"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,rotary", [(64, 32), (65, 20)])
def test_elements_that_turn(ly, dtype, D, rotary):  # noqa: F811
    """One that turns reaches its partner and no other."""
    q, k, wq, wk, _, _ = operands(D, 4, 2, 1, D, dtype)
    pos = torch.arange(4, device="cuda") + 1
    for interleaved in (False, True):
        how = dict(rotary=rotary, interleaved=interleaved, norm=False)
        want = ly.head_norm_rotary(q, k, pos, wq, wk, **how)[0]
        q2 = q.clone()
        q2[1, 0, 2] = math.inf
        got = ly.head_norm_rotary(q2, k, pos, wq, wk, **how)[0]
        other = torch.ones_like(q, dtype=torch.bool)
        other[1, 0, 2] = other[1, 0, 3 if interleaved else 2 + rotary // 2] = False
        assert torch.equal(bits(got)[other], bits(want)[other])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,rotary", [(64, 64), (64, 32), (128, 128), (65, 20), (50, 50)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_gradient_without_a_norm_does_not_read_its_input(ly, dtype, D, rotary, what):  # noqa: F811
    """Without a norm, dq and dk are the weights times what comes back, whatever stands in q and k; of the
    weights' gradients only that element's feels it."""
    q, k, wq, wk, dq, dk = operands(D, 6, 3, 2, D, dtype)
    pos = torch.arange(6, device="cuda")
    want = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk, rotary=rotary, norm=False)
    q[3, 2, 5] = what
    got = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk, rotary=rotary, norm=False)
    assert torch.equal(got["dq"], want["dq"]) and torch.equal(got["dk"], want["dk"])
    others = torch.arange(D, device="cuda") != 5
    assert torch.equal(got["dw_q"][others], want["dw_q"][others]) and not torch.isfinite(got["dw_q"][5])
    assert torch.equal(got["dw_k"], want["dw_k"])
