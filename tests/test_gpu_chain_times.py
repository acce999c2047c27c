"""The measured times of a chain's blocks are the GPU's, whatever the host needs to launch them."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ec():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import expert_chain
    return expert_chain


def small(ec, rows=200):
    chain = ec.ExpertChain(3, 128, 64, 4, p=0.1)
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn(rows, 128, generator=g).cuda().bfloat16() for _ in range(2))
    return chain, x, [torch.randint(0, 4, (rows,), generator=g).cuda() for _ in range(3)], dy


def test_a_slow_host_is_not_in_the_times(ec, monkeypatch):
    """A host that takes 5 ms for one call of each pass: the kernels of a block take some 50 us."""
    args = small(ec)
    for name in ("gated_unit", "gated_unit_grad"):
        def slow(*a, f=getattr(ec.ly, name), **k):
            time.sleep(0.005)
            return f(*a, **k)
        monkeypatch.setattr(ec.ly, name, slow)
    fc, bc = ec.measure(*args, steps=2, warmup=1)
    assert len(fc) == len(bc) == 3 and 1 <= min(fc + bc) and max(fc + bc) < 5000


def test_measuring_again_and_without_warm_up(ec):
    """Every call captures its own iteration and leaves nothing behind that the next one sees."""
    args = small(ec)
    a = ec.measure(*args, steps=3, warmup=0)
    before = args[0].step(*args[1:])
    ec.measure(*args, steps=1)
    after = args[0].step(*args[1:])
    assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])
    assert all(1 <= t < 5000 for times in a for t in times)
