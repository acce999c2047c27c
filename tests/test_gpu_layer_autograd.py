"""The layer operators build no autograd graph: a tensor that requires a gradient is refused, and
not answered with an output that has lost it."""
import pytest
import torch

from test_gpu_experts import normal, offs, operands

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


def calls(ly):
    """Each function and the tensors that it takes."""
    x, w, dy = operands(1, 12, 2, 16, 24, torch.float32)
    o = offs(0, 5, 12)
    n = normal
    norm = dict(x=n(2, 6, 32), f=n(3, 6, 32), gate=n(4, 1, 32), w_post=n(5, 32), w_pre=n(6, 32))
    grad = dict(norm, dy=n(7, 6, 32), dh=n(8, 6, 32))
    grad["y"] = grad.pop("x")
    return {"expert_matmul": (lambda x, w: ly.expert_matmul(x, w, o), dict(x=x, w=w)),
            "expert_matmul_grad_input": (lambda dy, w: ly.expert_matmul_grad_input(dy, w, o), dict(dy=dy, w=w)),
            "expert_matmul_grad_weight": (lambda dy, x: ly.expert_matmul_grad_weight(dy, x, o), dict(dy=dy, x=x)),
            "gated_unit": (ly.gated_unit, dict(h=n(9, 4, 16))),
            "gated_unit_grad": (ly.gated_unit_grad, dict(da=n(10, 4, 8), h=n(9, 4, 16))),
            "dropout": (lambda x, residual: ly.dropout(x, 0.5, 1, residual=residual), dict(x=n(11, 4, 8), residual=n(12, 4, 8))),
            "block_norm": (ly.block_norm, norm), "block_norm_grad": (ly.block_norm_grad, grad)}


NAMES = ["expert_matmul", "expert_matmul_grad_input", "expert_matmul_grad_weight", "gated_unit", "gated_unit_grad",
         "dropout", "block_norm", "block_norm_grad"]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_require_a_gradient(ly, name):
    f, tensors = calls(ly)[name]
    flat = lambda r: [t for t in (r.values() if isinstance(r, dict) else r if isinstance(r, tuple) else [r]) if t is not None]
    want = flat(f(**tensors))
    for k in tensors:
        leaf = {**tensors, k: tensors[k].clone().requires_grad_()}
        with pytest.raises(ValueError, match="gradient"):
            f(**leaf)
        with torch.no_grad():
            got = flat(f(**leaf))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        got = flat(f(**{q: t.detach() for q, t in leaf.items()}))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
