"""Block norms with many rows a block: the ring's slots are filled again and again, gate rows begin
and end inside a block's run of rows or span several, and gates outnumber the runs. Every output
against its definition in 64 bits on the GPU, within the bounds of layer_oracle, and again for
equal bits."""
import functools

import pytest
import torch

import layer_oracle as lo
from test_gpu_layers import norm_case

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    return layers


@functools.lru_cache(maxsize=1)
def keep_of(rows, D, p, seed, offset):
    return lo.keep_factor(rows, D, p, seed, offset).cuda()


def assert_within(got, exact, bound, what):
    """lo.assert_within on the GPU."""
    g, u = got.double(), lo.UNIT[got.dtype]
    assert g.shape == exact.shape, (what, g.shape, exact.shape)
    allowed = u * (exact.abs() + bound) + bound + lo.TINY[got.dtype] + 1e-300
    over = float(((g - exact).abs() / allowed).max())
    assert bool(torch.isfinite(g).all()) and over <= 1, (what, over)


def add_gates(pair, per_gate):
    """Sums of the gates' rows and their bounds, as lo.add_rows."""
    v, b = pair
    at = torch.arange(v.shape[0], device=v.device) // per_gate
    G = int(at[-1]) + 1
    add = lambda t: torch.zeros(G, v.shape[1], dtype=torch.float64, device=v.device).index_add_(0, at, t)
    return add(v), add(b) + (per_gate + 2) * lo.EPS * add(v.abs())


# rows, columns, rows a gate: aligned rows of one warp, of several, of a power of two and not, with 512
# threads; off 16-byte boundaries; gates longer than a run, shorter, of eight rows and fewer, more than runs
CASES = [(60_000, 96, 7, BF16), (60_000, 96, 2048, FP32), (20_000, 40, 2, BF16), (20_000, 40, 3, FP16),
         (30_000, 200, None, BF16), (30_001, 512, 9, BF16), (30_000, 512, 2048, FP16), (9_000, 1536, 100, BF16),
         (5_000, 4096, 7, BF16), (5_000, 4096, 9, FP16), (5_000, 4096, None, BF16), (5_003, 2048, 33, FP32),
         (5_000, 3001, 9, BF16), (5_000, 3001, 700, FP16), (6_000, 1001, 3, BF16), (30_000, 130, 9, FP32),
         (3_000, 5120, 9, BF16), (3_000, 5120, 3, BF16), (3_000, 8192, None, FP16), (1_500, 8200, 20, BF16)]


@pytest.mark.parametrize("rows,D,per_gate,dtype", CASES)
def test_many_rows_a_block(ly, rows, D, per_gate, dtype):
    p, seed, offset, alpha, eps = 0.2, 1 << 50, 11, 0.75, 1e-6
    keep = keep_of(rows, D, p, seed, offset)
    for kind in ("rms", "layer"):
        c = norm_case(100, rows, D, dtype, per_gate, kind)
        how = dict(gate=c["gate"], w_post=c["w_post"], w_pre=c["w_pre"], residual_scale=alpha, kind=kind,
                   eps=eps, p=p, seed=seed, offset=offset, rows_per_gate=per_gate)
        e = {k: v.double() for k, v in c.items()}
        g = e["gate"].repeat_interleave(per_gate or rows, 0)[:rows]
        args = (e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind, eps, keep)
        got = ly.block_norm(c["x"], c["f"], **how)
        for t, exact, bound, what in zip(got, lo.norm_forward(*args), lo.norm_forward_bounds(*args), "yh"):
            assert_within(t, exact, bound, what)
        again = ly.block_norm(c["x"], c["f"], **how)
        assert all(torch.equal(a, b) for a, b in zip(got, again))

        r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
        b = lo.norm_backward(e["dy"], e["dh"], e["x"], e["f"], g, e["w_post"], e["w_pre"], alpha, kind, eps, keep)
        assert_within(r["dx"], alpha * b["t"][0], alpha * b["t"][1], "dx")
        assert_within(r["df"], *b["df"], "df")
        assert_within(r["dgate"], *add_gates(b["gate"], per_gate or rows), "dgate")
        for k in ("w_post", "w_pre"):
            v, bd = add_gates(b[k], rows)
            assert_within(r["d" + k], v[0], bd[0], "d" + k)
        again = ly.block_norm_grad(c["dy"], c["dh"], c["x"], c["f"], **how)
        assert all(torch.equal(r[k], again[k]) for k in r)


@pytest.mark.parametrize("rows,D,dtype", [(20_000, 96, BF16), (5_000, 4096, BF16), (5_000, 3001, FP16)])
def test_many_rows_a_block_of_each_form(ly, rows, D, dtype):
    """The first norm alone and the last residual alone."""
    one = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    for kind in ("rms", "layer"):
        c = norm_case(110, rows, D, dtype, None, kind)
        e = {k: v.double() for k, v in c.items()}
        args = (e["x"], None, one, one, e["w_pre"], 1.0, kind, 1e-6, one)
        assert_within(ly.block_norm(c["x"], w_pre=c["w_pre"], kind=kind)[1], lo.norm_forward(*args)[1],
                      lo.norm_forward_bounds(*args)[1], "h")
        r = ly.block_norm_grad(c["dy"], c["dh"], c["x"], w_pre=c["w_pre"], kind=kind)
        b = lo.norm_backward(e["dy"], e["dh"], e["x"], None, one, one, e["w_pre"], 1.0, kind, 1e-6, one)
        assert_within(r["dx"], *b["t"], "dx")
        assert_within(r["dw_pre"], *(t[0] for t in add_gates(b["w_pre"], rows)), "dw_pre")
        args = (e["x"], e["f"], one, e["w_post"], one, 1.0, kind, 1e-6, one)
        assert_within(ly.block_norm(c["x"], c["f"], w_post=c["w_post"], kind=kind, want_h=False)[0],
                      lo.norm_forward(*args)[0], lo.norm_forward_bounds(*args)[0], "y")
        r = ly.block_norm_grad(c["dy"], None, c["x"], c["f"], w_post=c["w_post"], kind=kind)
        b = lo.norm_backward(e["dy"], None, e["x"], e["f"], one, e["w_post"], one, 1.0, kind, 1e-6, one)
        assert torch.equal(r["dx"], c["dy"])
        assert_within(r["df"], *b["df"], "df")
        assert_within(r["dw_post"], *(t[0] for t in add_gates(b["w_post"], rows)), "dw_post")
