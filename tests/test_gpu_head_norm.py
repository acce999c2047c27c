"""Norms of queries and keys with the rotation by position on the GPU against their definition in 64
bits, within bounds derived in attention_oracle; their gradients; refusals."""
import math

import pytest
import torch

import attention_oracle as ao
import layer_oracle as lo

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
DTYPES = [BF, HF, FL]


@pytest.fixture(scope="module")
def ly():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_07968_gb300 import build
    build.build()
    from paper_2101_07968_gb300 import layers
    return layers


def normal(seed, *shape, dtype=FL, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype).cuda()


def check(ly, q, k, pos, wq, wk, dq, dk, rotary=None, base=10000.0, interleaved=False, norm=True, eps=1e-6):
    how = dict(rotary=rotary, base=base, interleaved=interleaved, norm=norm, eps=eps)
    got = dict(zip("qk", ly.head_norm_rotary(q, k, pos, wq, wk, **how)))
    grad = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk, **how)
    D = q.shape[2]
    rotary = D // 2 * 2 if rotary is None else rotary
    p = pos.cpu()
    for name, x, w, dy in (("q", q, wq, dq), ("k", k, wk, dk)):
        X, Y = lo.d64(x), lo.d64(dy)
        W = torch.ones(D).double() if w is None else lo.d64(w)
        a = (p, rotary, base, interleaved, norm, eps)
        by, bdx, bdw = ao.rotary_bounds(X, W, Y, p, rotary, interleaved, norm, eps, base)
        lo.assert_within(got[name], ao.rotary_forward(X, W, *a), by, name)
        dx, dw = ao.rotary_grad(Y, X, W, *a)
        lo.assert_within(grad["d" + name], dx, bdx, "d" + name)
        if w is None:
            assert grad["dw_" + name] is None
        else:
            lo.assert_within(grad["dw_" + name], dw, bdw, "dw_" + name)
    return got, grad


def operands(seed, T, H, G, D, dtype):
    return (normal(seed, T, H, D, dtype=dtype), normal(seed + 1, T, G, D, dtype=dtype, scale=2.0),
            normal(seed + 2, D, dtype=dtype, scale=0.2, shift=1.0), normal(seed + 3, D, dtype=dtype, scale=0.2, shift=1.0),
            normal(seed + 4, T, H, D, dtype=dtype), normal(seed + 5, T, G, D, dtype=dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [1, 2, 8, 40, 63, 64, 65, 80, 128, 130, 200, 255, 256])
@pytest.mark.parametrize("T,H,G", [(1, 1, 1), (1, 16, 4), (37, 5, 1), (300, 2, 2)])
def test_sizes(ly, dtype, D, T, H, G):
    q, k, wq, wk, dq, dk = operands(D, T, H, G, D, dtype)
    pos = torch.arange(T, device="cuda") * 3
    check(ly, q, k, pos, wq, wk, dq, dk)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,rotary", [(64, 0), (64, 2), (64, 16), (64, 24), (80, 32), (128, 64), (128, 126), (65, 64), (96, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_and_order(ly, dtype, D, rotary, interleaved):
    q, k, wq, wk, dq, dk = operands(rotary, 41, 3, 2, D, dtype)
    pos = torch.arange(41, device="cuda") + 100
    check(ly, q, k, pos, wq, wk, dq, dk, rotary=rotary, interleaved=interleaved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("weights", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("D", [64, 50])
def test_weights_and_norm(ly, dtype, weights, norm, D):
    q, k, wq, wk, dq, dk = operands(7, 50, 4, 2, D, dtype)
    pos = torch.arange(50, device="cuda")
    check(ly, q, k, pos, wq if weights[0] else None, wk if weights[1] else None, dq, dk, norm=norm, eps=1e-3)


@pytest.mark.parametrize("base", [10000.0, 500000.0, 0.5, 1.0])
def test_positions(ly, base):
    """Far and negative ones: whole turns are dropped exactly."""
    v = [0, 1, -1, 1000003, -77777, 2**31 - 1, 2**31 + 5, -2**33]
    pos = torch.tensor(v, device="cuda")
    for dtype in DTYPES:
        q, k, wq, wk, dq, dk = operands(9, len(v), 2, 1, 64, dtype)
        check(ly, q, k, pos, wq, wk, dq, dk, base=base)
    check(ly, q, k, torch.zeros_like(pos), wq, wk, dq, dk, base=base)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(ly, dtype):
    """Slices of a projection's output, heads before tokens, and heads off aligned addresses: the bits
    of contiguous copies."""
    T, H, G, D = 70, 4, 2, 64
    wq, wk = normal(1, D, dtype=dtype), normal(2, D, dtype=dtype)
    dq, dk = normal(3, T, H, D, dtype=dtype), normal(4, T, G, D, dtype=dtype)
    pos = torch.arange(T, device="cuda")
    for x in (normal(5, T, H + 2 * G, D, dtype=dtype), normal(6, H + 2 * G, T, D, dtype=dtype).transpose(0, 1)):
        q, k = x[:, :H], x[:, H:H + G]
        a = ly.head_norm_rotary(q, k, pos, wq, wk)
        b = ly.head_norm_rotary(q.contiguous(), k.contiguous(), pos, wq, wk)
        assert all(torch.equal(s, t) for s, t in zip(a, b))
        a = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk)
        b = ly.head_norm_rotary_grad(dq, dk, q.contiguous(), k.contiguous(), pos, wq, wk)
        assert all(torch.equal(a[n], b[n]) for n in a)
    odd = normal(7, T, (H + G) * D + 5, dtype=dtype)[:, 1:1 + (H + G) * D].unflatten(1, (H + G, D))
    check(ly, odd[:, :H], odd[:, H:], pos, wq, wk, dq, dk)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [128, 100])
def test_many_tokens(ly, dtype, D):
    """More tokens than warps: the weights' gradients are summed over many rounds."""
    T = 30011
    q, k, wq, wk, dq, dk = operands(13, T, 2, 1, D, dtype)
    pos = torch.arange(T, device="cuda") % 4096
    got, grad = check(ly, q, k, pos, wq, wk, dq, dk)
    again = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk)
    assert all(torch.equal(grad[n], again[n]) for n in grad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_keep_to_themselves(ly, dtype):
    """NaN and infinity in a head stay in it; a head of zeros is zero."""
    q, k, wq, wk, dq, dk = operands(17, 9, 3, 2, 64, dtype)
    pos = torch.arange(9, device="cuda")
    want = ly.head_norm_rotary(q, k, pos, wq, wk)
    q2 = q.clone()
    q2[4, 1], q2[5, 2], q2[6, 0] = math.nan, math.inf, 0.0
    got = ly.head_norm_rotary(q2, k, pos, wq, wk)
    assert torch.equal(got[1], want[1]) and torch.isnan(got[0][4, 1].float()).all() and not got[0][6, 0].any()
    keep = torch.ones(9, 3, dtype=torch.bool, device="cuda")
    keep[4, 1] = keep[5, 2] = keep[6, 0] = False
    assert torch.equal(got[0][keep], want[0][keep])


def test_no_tokens(ly):
    q, k, wq, wk, dq, dk = operands(1, 0, 4, 2, 64, BF)
    pos = torch.arange(0, device="cuda")
    assert [t.shape for t in ly.head_norm_rotary(q, k, pos, wq, wk)] == [q.shape, k.shape]
    r = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk)
    assert not r["dw_q"].any() and not r["dw_k"].any() and r["dq"].shape == q.shape


def test_streams_and_graphs(ly):
    q, k, wq, wk, dq, dk = operands(19, 500, 4, 2, 128, BF)
    pos = torch.arange(500, device="cuda")

    def call(**how):
        r = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk, **how)
        return list(ly.head_norm_rotary(q, k, pos, wq, wk, **how)) + list(r.values())
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    pos.add_(5)
    q.mul_(0.5)
    want = call()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_far_addresses(ly):
    T, H, D = 140_000, 120, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.empty(s, dtype=BF, device="cuda").normal_(generator=g)
    q, k, dq, dk = make(T, H, D), make(T, 1, D), make(T, H, D), make(T, 1, D)
    pos = torch.arange(T, device="cuda")
    last = slice(T - 100, T)
    a = ly.head_norm_rotary(q, k, pos)
    b = ly.head_norm_rotary(q[last], k[last], pos[last])
    assert all(torch.equal(s[last], t) for s, t in zip(a, b))
    a = ly.head_norm_rotary_grad(dq, dk, q, k, pos)
    b = ly.head_norm_rotary_grad(dq[last], dk[last], q[last], k[last], pos[last])
    assert torch.equal(a["dq"][last], b["dq"]) and torch.equal(a["dk"][last], b["dk"])


@pytest.mark.parametrize("D,H,G", [(64, 5, 2), (128, 3, 1), (50, 4, 3)])
def test_in_place(ly, D, H, G):
    """The C functions may write over their inputs."""
    import ctypes

    from paper_2101_07968_gb300 import dynacomm as dc
    T = 700
    q, k, wq, wk, dq, dk = operands(29, T, H, G, D, BF)
    pos = torch.arange(T, device="cuda")
    want = ly.head_norm_rotary(q, k, pos, wq, wk)
    grad = ly.head_norm_rotary_grad(dq, dk, q, k, pos, wq, wk)
    cfg = ctypes.byref(dc.dc_head_norm_cfg(dc.DC_BF16, H, G, D, D, 0, 1, T, H * D, D, G * D, D, 1e4, 1e-6))
    s, p = torch.cuda.current_stream().cuda_stream, lambda t: t.data_ptr()
    need = dc.lib().dc_head_norm_rotary_grad_workspace_bytes(cfg)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dw = torch.empty(2, D, device="cuda")
    assert dc.lib().dc_head_norm_rotary_grad(cfg, p(dq), p(dk), p(q), p(k), p(pos), p(wq), p(wk), p(dq), p(dk), p(dw[0]),
                                             p(dw[1]), p(ws), need, s) == 0
    assert torch.equal(dq, grad["dq"]) and torch.equal(dk, grad["dk"]) and torch.equal(dw[0], grad["dw_q"])
    assert dc.lib().dc_head_norm_rotary(cfg, p(q), p(k), p(pos), p(wq), p(wk), p(q), p(k), s) == 0
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_against_differences(ly):
    q, k, wq, wk, dq, dk = (lo.d64(t) for t in operands(23, 3, 2, 1, 10, FL))
    pos = torch.tensor([0, 4, 9])
    for interleaved in (False, True):
        a = (pos, 8, 100.0, interleaved, True, 1e-3)
        dx, dw = ao.rotary_grad(dq, q, wq, *a)
        for at in ((0, 0, 0), (1, 1, 5), (2, 0, 9), (2, 1, 3)):
            d = []
            for step in (1e-6, -1e-6):
                t = q.clone()
                t[at] += step
                d.append(float((ao.rotary_forward(t, wq, *a) * dq).sum()))
            assert abs((d[0] - d[1]) / 2e-6 - float(dx[at])) < 1e-7
            d = []
            for step in (1e-6, -1e-6):
                t = wq.clone()
                t[at[2]] += step
                d.append(float((ao.rotary_forward(q, t, *a) * dq).sum()))
            assert abs((d[0] - d[1]) / 2e-6 - float(dw[at[2]])) < 1e-7


def test_refusals(ly):
    from paper_2101_07968_gb300 import dynacomm as dc
    q, k, wq, wk, dq, dk = operands(1, 10, 4, 2, 32, BF)
    pos = torch.arange(10, device="cuda")
    args = dict(q=q, k=k, positions=pos, w_q=wq, w_k=wk)
    for b in (dict(q=q.float()), dict(k=k[:9]), dict(k=k[..., :16]), dict(q=q.cpu()), dict(q=q[0]), dict(q=q.transpose(1, 2)),
              dict(positions=pos.int()), dict(positions=pos[:9]), dict(positions=pos.cpu()), dict(w_q=wq.float()),
              dict(w_k=wk[:31]), dict(q=q.double(), k=k.double())):
        with pytest.raises(ValueError):
            ly.head_norm_rotary(**{**args, **b})
        with pytest.raises(ValueError):
            ly.head_norm_rotary_grad(dq, dk, **{**args, **b})
    for b in (dict(dq=dq.float()), dict(dk=dk[:, :1]), dict(dq=dq.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            ly.head_norm_rotary_grad(**{**dict(dq=dq, dk=dk), **b}, **args)
    for b in (dict(rotary=33), dict(rotary=3), dict(rotary=-2), dict(rotary=64), dict(base=0.0), dict(base=math.nan),
              dict(base=math.inf), dict(eps=-1.0), dict(eps=math.nan), dict(q=q[:, :1].expand(10, 4, 32)),
              dict(q=q[:1].expand(10, 4, 32))):
        with pytest.raises(dc.DynaCommError):
            ly.head_norm_rotary(**{**args, **b})
    wide = operands(2, 3, 1, 1, 257, BF)
    with pytest.raises(dc.DynaCommError):
        ly.head_norm_rotary(wide[0], wide[1], pos[:3])
    for name in ("q", "k", "w_q", "w_k"):
        with pytest.raises(ValueError, match="gradient"):
            ly.head_norm_rotary(**{**args, name: args[name].clone().requires_grad_()})
