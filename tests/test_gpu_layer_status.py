"""The word that the expert products' kernels report to: made once, outside of graphs, and read
after every stream is done; and a wait that runs out."""
import os
import subprocess
import sys
import threading
import time

import pytest
import torch

from test_gpu_experts import offs, operands

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    yield layers
    layers.check_status()


FIRST_IN_A_CAPTURE = """
import torch
from paper_2101_07968_gb300 import dynacomm as dc, layers as ly
x, w = torch.ones(100, 64, device="cuda").half(), torch.ones(2, 64, 64, device="cuda").half()
o = torch.tensor([0, 50, 100], device="cuda")
{warm}
graph = torch.cuda.CUDAGraph()
try:
    with torch.cuda.graph(graph):
        y = ly.expert_matmul(x, w, o)
except RuntimeError as e:
    print("refused", e)
    raise SystemExit
ly._status[0][0].fill_(dc.DC_ERR_INTERNAL)  # what a kernel of another call would report
graph.replay()
try:
    ly.check_status()
    print("lost")
except dc.DynaCommError:
    print("kept")
ly.check_status()
graph.replay()
ly.check_status()
print("right" if bool((y == 64).all()) else "wrong")
"""


@pytest.mark.parametrize("warm,want", [("", ["refused"]), ("ly.check_status()", ["kept", "right"]),
                                       ("ly.expert_matmul(x, w, o)", ["kept", "right"])])
def test_first_product_in_a_capture(ly, warm, want):
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE.format(warm=warm)], cwd=ROOT, capture_output=True,
                       text=True, timeout=120)
    assert [line.split()[0] for line in r.stdout.splitlines()] == want, r.stdout + r.stderr


def test_check_waits_for_other_streams(ly):
    """A report that comes late, on a stream that is not the current one."""
    from paper_2101_07968_gb300.dynacomm import DynaCommError
    x, w, _ = operands(1, 10, 1, 8, 8, torch.float32)
    ly.expert_matmul(x, w, offs(0, 10))
    word = ly._status[torch.cuda.current_device()][0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = torch.ones(8192, 8192, device="cuda")
        for _ in range(20):
            a = a @ a * 1e-4
        word.fill_(8)
    with pytest.raises(DynaCommError):
        ly.check_status()
    ly.check_status()


def test_one_word_for_threads_that_come_together(ly, monkeypatch):
    zeros = torch.zeros

    def slow(*a, **k):
        time.sleep(0.05)
        return zeros(*a, **k)
    ly.check_status()
    monkeypatch.setattr(ly, "_status", {})
    monkeypatch.setattr(torch, "zeros", slow)
    got = []
    device = torch.cuda.current_device()
    threads = [threading.Thread(target=lambda: got.append(ly._status_of(device))) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(got) == 4 and len(set(got)) == 1 and got[0] == ly._status[device][0].data_ptr()


def test_a_wait_that_runs_out_ends_and_reports(ly):
    """Two threads wait for copies that nothing has started: the kernel ends within some two
    seconds, reports, and the device goes on."""
    from paper_2101_07968_gb300.dynacomm import DC_ERR_INTERNAL, DC_ERR_NULL, DynaCommError
    x, w, _ = operands(1, 100, 2, 64, 64, torch.float16)
    o = offs(0, 50, 100)
    want = ly.expert_matmul(x, w, o)
    ly.check_status()
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    ly._run("dc_wait_probe", x, None, ly._status_of(x.get_device()))
    stop.record()
    with pytest.raises(DynaCommError) as e:
        ly.check_status()
    assert e.value.status == DC_ERR_INTERNAL
    assert start.elapsed_time(stop) < 4000
    assert ly._function("dc_wait_probe")(None, None) == DC_ERR_NULL
    ly.check_status()
    assert torch.equal(ly.expert_matmul(x, w, o), want)
