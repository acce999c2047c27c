"""Layer operators on torch tensors: the training block of a mixture of experts.

The cost rows of a schedule are a model's measured layer times; these are layers of large
language models, forward and backward, whose times can be measured on this GPU
(``expert_chain`` does that and schedules the result). Every function allocates its outputs
with torch, checks its arguments (ValueError) and launches the library's kernels on torch's
current CUDA stream or ``stream``; nothing synchronises. A caller that uses tensors on
another stream than their own orders the streams and keeps the tensors alive, as with any
kernel launch. No function builds an autograd graph: a tensor that requires a gradient is
refused unless gradients are off (torch.no_grad()).

* ``expert_matmul``, ``expert_matmul_grad_input``, ``expert_matmul_grad_weight``
* ``gated_unit``, ``gated_unit_grad``
* ``dropout`` (its gradient is the same call on the gradient)
* ``block_norm``, ``block_norm_grad``

The operations are defined in include/dynacomm.h.
"""
from __future__ import annotations

import ctypes
import threading

import torch

from . import dynacomm as dc

_DTYPES = {torch.bfloat16: dc.DC_BF16, torch.float16: dc.DC_FP16, torch.float32: dc.DC_FP32}
_empty = torch.empty
_ACTS = {"silu": dc.DC_ACT_SILU, "gelu": dc.DC_ACT_GELU}
_KINDS = {"rms": dc.DC_NORM_RMS, "layer": dc.DC_NORM_LAYER}


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"bfloat16, float16 or float32 expected, not {t.dtype}")
    return code


def _like(name, t, ref, shape):
    """t has ref's type and device and the given shape (ref is on a device)."""
    if t.dtype is not ref.dtype or t.shape != shape or t.get_device() != ref.get_device():
        raise ValueError(f"{name}: {tuple(shape)} {ref.dtype} on {ref.device} expected, not "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")


def _no_graph(*tensors):
    """Outputs carry no autograd graph, so a gradient that is asked for would be lost."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("a tensor requires a gradient, and the layer operators build no autograd graph: "
                                 "call them under torch.no_grad() or on detached tensors, and their gradients "
                                 "by the ..._grad functions")


def _rows(name, t) -> int:
    """The stride of a [rows, columns] tensor whose rows are contiguous and apart."""
    if not t.is_cuda:
        raise ValueError("device tensor expected (the library takes device pointers)")
    if t.dim() != 2:
        raise ValueError(f"{name}: two dimensions expected")
    rows, cols = t.shape
    ld, one = t.stride()
    if cols > 1 and one != 1:
        raise ValueError(f"{name}: contiguous rows expected")
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError(f"{name}: rows that do not overlap expected")
    return ld


_current_device = torch._C._cuda_getDevice
_library = None  # the one that _functions come from
_functions = {}


def _function(name):
    """The library's function, looked up once: a call costs the host some ten microseconds."""
    global _library
    lib = dc._lib or dc.lib()
    if lib is not _library:
        _library = lib
        _functions.clear()
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(lib, name)
    return fn


def _run(name, t, stream, *args):
    """One call of the library on t's device."""
    fn = _function(name)
    if t.get_device() == _current_device():
        st = fn(*args, dc._stream(stream))
    else:
        with torch.cuda.device(t.device):
            st = fn(*args, dc._stream(stream))
    if st:
        raise dc.DynaCommError(st, name)


def _used_on(ws, stream):
    """A workspace goes back to the allocator when the call returns; tell it of a stream other
    than the current one that still uses it."""
    if ws is not None and stream is not None:
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=ws.device)
        ws.record_stream(stream)


# ------------------------------------------------------------------- expert products
_status = {}  # per device: the word that kernels report to, and its address
_status_lock = threading.Lock()


def _status_of(device):
    at = _status.get(device)
    if at is None:
        with _status_lock, torch.cuda.device(device):
            at = _status.get(device)
            if at is None:
                # its fill must be done before a kernel of any stream, and be part of no graph,
                # whose replays would clear what other calls reported
                if torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("the first expert product on a device cannot be captured: "
                                       "call one of them, or check_status(), before the capture")
                t = torch.zeros(1, dtype=torch.int32, device=f"cuda:{device}")
                torch.cuda.current_stream().synchronize()
                at = _status[device] = (t, t.data_ptr())
    return at[1]


def check_status() -> None:
    """Waits for everything on the devices that expert products have run on (and the current
    one) and raises DynaCommError if a kernel of this module has given up a wait (a bug of the
    library or a fault of the machine; the call's outputs are incomplete)."""
    if torch.cuda.is_available():
        _status_of(torch.cuda.current_device())
    for device, (t, _) in list(_status.items()):
        torch.cuda.synchronize(device)
        s = int(t.item())
        if s:
            t.zero_()
            torch.cuda.synchronize(device)
            raise dc.DynaCommError(s, f"layer operators on cuda:{device}")


def _weights(name, w):
    if not w.is_cuda:
        raise ValueError("device tensor expected (the library takes device pointers)")
    if w.dim() != 3:
        raise ValueError(f"{name}: [experts, N, K] expected")
    E, N, K = w.shape
    se, sn, sk = w.stride()
    # a dimension of one element has no stride of its own
    if K == 1:
        sk = 1 if sn != 1 or N == 1 else N
    if N == 1:
        sn = K if sk == 1 else 1
    if not (sk == 1 and sn >= K) and not (sn == 1 and sk >= N):
        raise ValueError(f"{name}: N or K contiguous expected")
    return E, N, K, (se if E > 1 else 0), sn, sk


def _offsets(offsets, experts, ref):
    if offsets.dtype is not torch.int64 or offsets.shape != (experts + 1,) \
            or offsets.get_device() != ref.get_device() or not offsets.is_contiguous():
        raise ValueError(f"offsets: {experts + 1} contiguous int64 on {ref.device} expected")


def _shape(code, E, rows, N, K, ldx, ldy, se, sn, sk):
    return ctypes.byref(dc.dc_expert_shape(code, E, rows, N, K, ldx, ldy, se, sn, sk))


_PRODUCTS = ("dc_expert_matmul", "dc_expert_matmul_grad_input", "dc_expert_matmul_grad_weight")


def _product(which, shape, a, b, offsets, c, stream):
    _no_graph(a, b)
    ap, bp = a.data_ptr(), b.data_ptr()
    # few rows need none in any case
    few = which < 2 and a.shape[0] <= dc.DC_FEW_ROWS
    need = 0 if few else _function("dc_expert_workspace_bytes")(shape, which, ap, bp)
    ws = _empty(need, dtype=torch.uint8, device=a.device) if need else None
    _run(_PRODUCTS[which], a, stream, shape, ap, bp, offsets.data_ptr(), c.data_ptr(),
         _status_of(a.get_device()), ws.data_ptr() if need else None, need)
    _used_on(ws, stream)
    return c


def expert_matmul(x, w, offsets, stream=None):
    """y [rows, N]: y[r] = w[e] @ x[r] for the expert e whose rows hold r (offsets[e] <= r <
    offsets[e + 1], int64 [experts + 1]); zeros for rows of no expert. x [rows, K] with any row
    stride, w [experts, N, K] with N or K contiguous and each expert's matrix apart from the others'."""
    ldx = _rows("x", x)
    E, N, K, se, sn, sk = _weights("w", w)
    R = x.shape[0]
    _like("x", x, w, (R, K))
    _offsets(offsets, E, x)
    return _product(0, _shape(_dtype(x), E, R, N, K, ldx, N, se, sn, sk), x, w, offsets,
                    _empty((R, N), dtype=x.dtype, device=x.device), stream)


def expert_matmul_grad_input(dy, w, offsets, stream=None):
    """dx [rows, K] of expert_matmul from dy [rows, N]."""
    ldy = _rows("dy", dy)
    E, N, K, se, sn, sk = _weights("w", w)
    R = dy.shape[0]
    _like("dy", dy, w, (R, N))
    _offsets(offsets, E, dy)
    return _product(1, _shape(_dtype(dy), E, R, N, K, K, ldy, se, sn, sk), dy, w, offsets,
                    _empty((R, K), dtype=dy.dtype, device=dy.device), stream)


def expert_matmul_grad_weight(dy, x, offsets, stream=None):
    """dw [experts, N, K] of expert_matmul from dy [rows, N] and x [rows, K]; the number of
    experts is that of offsets."""
    ldy, ldx = _rows("dy", dy), _rows("x", x)
    R, N = dy.shape
    K = x.shape[1]
    _like("x", x, dy, (R, K))
    E = offsets.numel() - 1
    _offsets(offsets, E, dy)
    return _product(2, _shape(_dtype(dy), E, R, N, K, ldx, ldy, N * K, K, 1), dy, x, offsets,
                    _empty((E, N, K), dtype=dy.dtype, device=dy.device), stream)


# ------------------------------------------------------------------------ gated unit
def _act(act) -> int:
    if act not in _ACTS:
        raise ValueError(f"act: one of {sorted(_ACTS)} expected")
    return _ACTS[act]


def gated_unit(h, act="silu", stream=None):
    """[rows, F]: act(h[:, :F]) * h[:, F:] for h [rows, 2F]."""
    ldh = _rows("h", h)
    R, F2 = h.shape
    if F2 % 2:
        raise ValueError("h: an even number of columns expected")
    _no_graph(h)
    a = _empty((R, F2 // 2), dtype=h.dtype, device=h.device)
    _run("dc_gated_unit", h, stream, _dtype(h), _act(act), R, F2 // 2, h.data_ptr(), ldh,
         a.data_ptr(), F2 // 2)
    return a


def gated_unit_grad(da, h, act="silu", stream=None):
    """dh [rows, 2F] of gated_unit from da [rows, F] and h."""
    ldh, ldda = _rows("h", h), _rows("da", da)
    R, F2 = h.shape
    if F2 % 2:
        raise ValueError("h: an even number of columns expected")
    _like("da", da, h, (R, F2 // 2))
    _no_graph(da, h)
    dh = _empty((R, F2), dtype=h.dtype, device=h.device)
    _run("dc_gated_unit_grad", h, stream, _dtype(h), _act(act), R, F2 // 2, da.data_ptr(), ldda,
         h.data_ptr(), ldh, dh.data_ptr(), F2)
    return dh


# --------------------------------------------------------------------------- dropout
def dropout_draws(rows, cols) -> int:
    """How far one call on [rows, cols] moves the generator: add it to the next offset."""
    return rows * ((cols + 3) // 4)


def dropout(x, p, seed, offset=0, residual=None, stream=None):
    """x / (1 - p) where kept, else 0, plus residual if given; the mask is a function of
    (seed, offset, row, column) and is never stored. The gradient is the same call on dy."""
    ldx = _rows("x", x)
    R, C = x.shape
    ldr, res = 0, None
    if residual is not None:
        ldr, res = _rows("residual", residual), residual.data_ptr()
        _like("residual", residual, x, (R, C))
    _no_graph(x, residual)
    y = _empty((R, C), dtype=x.dtype, device=x.device)
    _run("dc_dropout", x, stream, _dtype(x), R, C, x.data_ptr(), ldx, res, ldr, y.data_ptr(), C,
         p, int(seed), int(offset))
    return y


# ----------------------------------------------------------------------- block norms
def _norm_cfg(x, kind, rows_per_gate, residual_scale, eps, p, seed, offset):
    if kind not in _KINDS:
        raise ValueError(f"kind: one of {sorted(_KINDS)} expected")
    R, D = x.shape
    return dc.dc_block_norm_cfg(_dtype(x), _KINDS[kind], R, D, rows_per_gate or max(R, 1),
                                residual_scale, eps, p, int(seed), int(offset))


def _contiguous(name, t, ref, shape):
    """t's address: contiguous, of ref's type and device and the given shape; None for None."""
    if t is None:
        return None
    _like(name, t, ref, shape)
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensor expected")
    return t.data_ptr()


def _norm_operands(x, f, gate, w_post, w_pre, rows_per_gate):
    """Checks; the pointers of x, f, gate, w_post, w_pre."""
    if not x.is_cuda:
        raise ValueError("device tensor expected (the library takes device pointers)")
    if x.dim() != 2:
        raise ValueError("x or y: two dimensions expected")
    _no_graph(x, f, gate, w_post, w_pre)
    R, D = shape = x.shape
    if rows_per_gate is not None and rows_per_gate < 1:
        raise ValueError("rows_per_gate: at least one expected")
    gates = -(-R // rows_per_gate) if rows_per_gate else (1 if R else 0)
    return (_contiguous("x or y", x, x, shape), _contiguous("f", f, x, shape),
            _contiguous("gate", gate, x, (gates, D)), _contiguous("w_post", w_post, x, (D,)),
            _contiguous("w_pre", w_pre, x, (D,)))


def block_norm(x, f=None, gate=None, w_post=None, w_pre=None, residual_scale=1.0, kind="rms",
               eps=1e-6, p=0.0, seed=0, offset=0, rows_per_gate=None, want_h=True, stream=None):
    """(y, h): y = residual_scale * x + gate * drop(w_post * n(f)) and h = w_pre * n(y), in one
    pass. x, f [rows, D] contiguous; gate [ceil(rows / rows_per_gate), D] (rows_per_gate None:
    one gate for all rows); w_post, w_pre [D]; any of the three None for ones. f None: the
    first norm alone, y is x. want_h False: the last residual alone, h is None."""
    xp, fp, gp, pp, ep = _norm_operands(x, f, gate, w_post, w_pre, rows_per_gate)
    if f is None and not want_h:
        raise ValueError("f or want_h expected: there is nothing to compute")
    cfg = _norm_cfg(x, kind, rows_per_gate, residual_scale, eps, p, seed, offset)
    y = torch.empty_like(x) if f is not None else None
    h = torch.empty_like(x) if want_h else None
    _run("dc_block_norm", x, stream, ctypes.byref(cfg), xp, fp, gp, pp, ep,
         None if y is None else y.data_ptr(), None if h is None else h.data_ptr())
    return (x if y is None else y), h


def block_norm_grad(dy, dh, y, f=None, gate=None, w_post=None, w_pre=None, residual_scale=1.0,
                    kind="rms", eps=1e-6, p=0.0, seed=0, offset=0, rows_per_gate=None,
                    stream=None):
    """Gradients of block_norm as a dict: dx, df, dgate (gate's shape and type), dw_post and
    dw_pre (float32 [D]); None for what the call did not have. dy, dh: the gradients of y and h
    (either may be None: dy zero, dh for a call without h); y: the call's output (x where f was
    None)."""
    yp, fp, gp, pp, ep = _norm_operands(y, f, gate, w_post, w_pre, rows_per_gate)
    _no_graph(dy, dh)
    dyp, dhp = _contiguous("dy", dy, y, y.shape), _contiguous("dh", dh, y, y.shape)
    if dh is None and (dy is None or f is None):
        raise ValueError("dh expected, or dy and f")
    cfg = _norm_cfg(y, kind, rows_per_gate, residual_scale, eps, p, seed, offset)
    D = y.shape[1]
    out = {"dx": torch.empty_like(y), "df": None, "dgate": None, "dw_post": None, "dw_pre": None}
    if f is not None:
        out["df"] = torch.empty_like(f)
        if gate is not None:
            out["dgate"] = torch.empty_like(gate)
        if w_post is not None:
            out["dw_post"] = _empty(D, dtype=torch.float32, device=y.device)
    if dh is not None and w_pre is not None:
        out["dw_pre"] = _empty(D, dtype=torch.float32, device=y.device)
    need = _function("dc_block_norm_grad_workspace_bytes")(ctypes.byref(cfg))
    ws = _empty(max(need, 1), dtype=torch.uint8, device=y.device)
    _run("dc_block_norm_grad", y, stream, ctypes.byref(cfg), dyp, dhp, yp, fp, gp, pp, ep,
         *[None if t is None else t.data_ptr() for t in out.values()], ws.data_ptr(), need)
    _used_on(ws, stream)
    return out
