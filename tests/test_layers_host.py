"""Host-side checks of the layer operators' C ABI (no GPU): bad arguments are refused before
anything is launched, workspace queries, and the oracle's own generator against the published
SplitMix64 test vector."""
import ctypes

import numpy as np
import pytest

from conftest import read_golden
from paper_2101_07968_gb300 import build as libbuild
from paper_2101_07968_gb300 import dynacomm as dc

FAKE = 0x1000  # never dereferenced: every case below fails its host check first
PRODUCTS = ["dc_expert_matmul", "dc_expert_matmul_grad_input", "dc_expert_matmul_grad_weight"]


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dc.lib()


def shape(**kw):
    d = dict(dtype=dc.DC_BF16, experts=2, rows=100, N=64, K=32, ldx=32, ldy=64, w_expert=64 * 32, w_n=32, w_k=1)
    d.update(kw)
    return ctypes.byref(dc.dc_expert_shape(*d.values()))


@pytest.mark.parametrize("fn", PRODUCTS)
def test_expert_checks(lib, fn):
    f = getattr(lib, fn)
    go = lambda s, a=FAKE, b=FAKE, o=FAKE, c=FAKE, ws=None, n=0: f(s, a, b, o, c, None, ws, n, None)
    for bad in (dict(dtype=3), dict(dtype=-1), dict(experts=0), dict(experts=1025), dict(rows=-1), dict(rows=2**31),
                dict(N=0), dict(K=0), dict(N=2**20 + 1, ldy=2**20 + 1, w_expert=2**40), dict(ldx=31), dict(ldy=63),
                dict(w_n=31), dict(w_k=2), dict(w_k=63, w_n=1), dict(w_expert=64 * 32 - 1), dict(w_expert=0),
                dict(ldx=2**40 + 1)):
        assert go(shape(**bad)) == dc.DC_ERR_BAD_LAYER, bad
    assert f(None, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == dc.DC_ERR_NULL
    for null in ("a", "b", "o", "c"):
        assert go(shape(), **{null: None}) == dc.DC_ERR_NULL, null
    if fn != "dc_expert_matmul_grad_weight":
        assert f(shape(rows=0), None, None, None, None, None, None, 0, None) == dc.DC_OK
    # operands off 16-byte boundaries need room for their aligned copies
    which = PRODUCTS.index(fn)
    odd = shape(K=33, ldx=33, w_n=33, w_expert=64 * 33)
    need = lib.dc_expert_workspace_bytes(odd, which, FAKE, FAKE)
    assert need > 0
    assert go(odd) == dc.DC_ERR_WORKSPACE
    assert go(odd, ws=FAKE, n=need - 1) == dc.DC_ERR_WORKSPACE


def test_expert_workspace(lib):
    q = lib.dc_expert_workspace_bytes
    for which in range(3):
        assert q(shape(), which, FAKE, FAKE) == 0
        assert q(shape(), which, FAKE + 2, FAKE) > 0      # rows start off the boundary
    assert q(shape(rows=dc.DC_FEW_ROWS, K=33, ldx=33, w_n=33, w_expert=64 * 33), 0, FAKE, FAKE) == 0  # few rows
    assert q(shape(dtype=3), 0, FAKE, FAKE) == 0 and q(shape(), 3, FAKE, FAKE) == 0
    assert q(shape(rows=0), 0, FAKE, FAKE) == 0 and q(None, 0, FAKE, FAKE) == 0
    # floats: two parts of both operands
    f = dict(dtype=dc.DC_FP32, rows=1000, K=256, ldx=256, w_n=256, w_expert=64 * 256)
    assert q(shape(**f), 0, FAKE, FAKE) >= 2 * 4 * 256 * (1000 + 2 * 64)
    assert q(shape(**f), 2, FAKE, FAKE) >= 2 * 4 * 1000 * (64 + 256)


def test_gated_checks(lib):
    g = lambda dt=0, act=0, rows=5, F=8, h=FAKE, ldh=16, a=FAKE, lda=8: lib.dc_gated_unit(dt, act, rows, F, h, ldh,
                                                                                          a, lda, None)
    for bad in (dict(dt=3), dict(act=2), dict(act=-1), dict(rows=-1), dict(F=0), dict(ldh=15), dict(lda=7)):
        assert g(**bad) == dc.DC_ERR_BAD_LAYER, bad
    assert g(h=None) == dc.DC_ERR_NULL and g(a=None) == dc.DC_ERR_NULL
    assert g(rows=0, h=None, a=None) == dc.DC_OK
    b = lambda rows=5, ldda=8, ldh=16, lddh=16, da=FAKE: lib.dc_gated_unit_grad(0, 0, rows, 8, da, ldda, FAKE, ldh,
                                                                               FAKE, lddh, None)
    assert b(ldda=7) == b(ldh=15) == b(lddh=15) == dc.DC_ERR_BAD_LAYER
    assert b(da=None) == dc.DC_ERR_NULL and b(rows=0) == dc.DC_OK


def test_dropout_checks(lib):
    d = lambda dt=0, rows=5, cols=8, x=FAKE, ldx=8, r=None, ldr=0, y=FAKE, ldy=8, p=0.1, off=0: lib.dc_dropout(
        dt, rows, cols, x, ldx, r, ldr, y, ldy, p, 1, off, None)
    for bad in (dict(dt=5), dict(rows=-1), dict(cols=0), dict(ldx=7), dict(ldy=7), dict(r=FAKE, ldr=7), dict(p=-0.01),
                dict(p=1.01), dict(p=float("nan")), dict(off=-1)):
        assert d(**bad) == dc.DC_ERR_BAD_LAYER, bad
    assert d(x=None) == dc.DC_ERR_NULL and d(y=None) == dc.DC_ERR_NULL
    assert d(rows=0, x=None, y=None) == dc.DC_OK


def test_norm_checks(lib):
    def cfg(**kw):
        d = dict(dtype=0, kind=0, rows=10, D=64, rows_per_gate=5, residual_scale=1.0, eps=1e-6, p=0.0, seed=0, offset=0)
        d.update(kw)
        return ctypes.byref(dc.dc_block_norm_cfg(*d.values()))
    fwd = lambda c, x=FAKE, f=FAKE, y=FAKE, h=FAKE: lib.dc_block_norm(c, x, f, None, None, None, y, h, None)
    bwd = lambda c, dy=FAKE, dh=FAKE, y=FAKE, f=FAKE, dx=FAKE, df=FAKE, ws=FAKE, n=1 << 30: lib.dc_block_norm_grad(
        c, dy, dh, y, f, None, None, None, dx, df, None, None, None, ws, n, None)
    for bad in (dict(dtype=3), dict(kind=2), dict(rows=-1), dict(rows=2**31), dict(D=0), dict(D=16385),
                dict(rows_per_gate=0), dict(eps=-1.0), dict(eps=float("nan")), dict(p=2.0), dict(offset=-1)):
        assert fwd(cfg(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert bwd(cfg(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert lib.dc_block_norm_grad_workspace_bytes(cfg(**bad)) == 0
    assert lib.dc_block_norm(None, FAKE, FAKE, None, None, None, FAKE, FAKE, None) == dc.DC_ERR_NULL
    for null in (dict(x=None), dict(y=None), dict(f=None, h=None)):
        assert fwd(cfg(), **null) == dc.DC_ERR_NULL, null
    for null in (dict(y=None), dict(dx=None), dict(df=None), dict(dy=None, dh=None), dict(f=None, dh=None)):
        assert bwd(cfg(), **null) == dc.DC_ERR_NULL, null
    need = lib.dc_block_norm_grad_workspace_bytes(cfg())
    assert need >= 10 * 2 * 64 * 4
    assert bwd(cfg(), ws=None) == dc.DC_ERR_WORKSPACE and bwd(cfg(), n=need - 1) == dc.DC_ERR_WORKSPACE
    assert fwd(cfg(rows=0), x=None) == dc.DC_OK and bwd(cfg(rows=0)) == dc.DC_OK


def test_oracle_generator_is_splitmix64():
    """The dropout oracle's draws against the published outputs for seed 1234567."""
    import layer_oracle as lo
    want = [int(r[-1], 0) for r in read_golden("splitmix64_seed1234567.txt")]
    got = lo.splitmix(1234567, np.arange(1, len(want) + 1))
    assert [int(v) for v in got] == want
