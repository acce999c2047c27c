"""Host-side checks of the C ABI of head norms and attention (no GPU): bad arguments are refused
before anything is launched; workspace queries; the list of tiles' room; the frequencies' fractions."""
import ctypes

import pytest

from paper_2101_07968_gb300 import build as libbuild
from paper_2101_07968_gb300 import dynacomm as dc

FAKE = 0x1000  # never dereferenced: every case below fails its host check first


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dc.lib()


def norm_cfg(**kw):
    d = dict(dtype=0, heads=4, kv_heads=2, D=64, rotary=64, interleaved=0, norm=1, tokens=10, q_token=256, q_head=64,
             k_token=128, k_head=64, base=1e4, eps=1e-6)
    d.update(kw)
    return ctypes.byref(dc.dc_head_norm_cfg(*d.values()))


def shape(**kw):
    d = dict(dtype=0, heads=4, kv_heads=2, D=64, sequences=3, tokens=100, q_token=256, q_head=64, k_token=128, k_head=64,
             v_token=128, v_head=64, scale=0.125)
    d.update(kw)
    return ctypes.byref(dc.dc_attention_shape(*d.values()))


STRIDES = [dict(q_head=63), dict(q_token=255), dict(k_token=127), dict(q_token=0), dict(q_token=2**37 + 1), dict(q_head=-64)]


def test_head_norm_checks(lib):
    fwd = lambda c, q=FAKE, k=FAKE, p=FAKE, qo=FAKE, ko=FAKE: lib.dc_head_norm_rotary(c, q, k, p, None, None, qo, ko, None)
    bwd = lambda c, ws=FAKE, n=1 << 30, dwq=FAKE, **null: lib.dc_head_norm_rotary_grad(
        c, *[null.get(a, FAKE) for a in ("dqo", "dko", "q", "k", "p")], None, None, null.get("dq", FAKE),
        null.get("dk", FAKE), dwq, None, ws, n, None)
    for bad in STRIDES + [dict(dtype=3), dict(heads=0), dict(kv_heads=0), dict(heads=1025, q_token=1025 * 64), dict(D=0),
                          dict(D=257, q_head=257, k_head=257, q_token=2000, k_token=1000), dict(rotary=63), dict(rotary=-2),
                          dict(rotary=66), dict(tokens=-1), dict(tokens=2**31), dict(base=0.0), dict(base=-1.0), dict(base=9e-4),
                          dict(base=1.1e30), dict(eps=1e39),
                          dict(base=float("inf")), dict(base=float("nan")), dict(eps=-1e-9), dict(eps=float("nan"))]:
        assert fwd(norm_cfg(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert bwd(norm_cfg(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert lib.dc_head_norm_rotary_grad_workspace_bytes(norm_cfg(**bad)) == 0
    assert fwd(None) == dc.DC_ERR_NULL and bwd(None) == dc.DC_ERR_NULL
    for null in ("q", "k", "p", "qo", "ko"):
        assert fwd(norm_cfg(), **{null: None}) == dc.DC_ERR_NULL, null
    for null in ("dqo", "dko", "q", "k", "p", "dq", "dk"):
        assert bwd(norm_cfg(), **{null: None}) == dc.DC_ERR_NULL, null
    need = lib.dc_head_norm_rotary_grad_workspace_bytes(norm_cfg())
    assert need > 0 and bwd(norm_cfg(), ws=None) == dc.DC_ERR_WORKSPACE and bwd(norm_cfg(), n=need - 1) == dc.DC_ERR_WORKSPACE
    assert fwd(norm_cfg(tokens=0), q=None) == dc.DC_OK
    # heads before tokens do not overlap either
    assert fwd(norm_cfg(q_token=64, q_head=640, k_token=64, k_head=640), q=None) == dc.DC_ERR_NULL
    assert fwd(norm_cfg(q_token=64, q_head=639)) == dc.DC_ERR_BAD_LAYER


def test_attention_checks(lib):
    names = ("q", "k", "v", "o", "y", "lse")
    fwd = lambda s, ws=FAKE, n=1 << 40, **null: lib.dc_attention(s, *[null.get(a, FAKE) for a in names], None, ws, n, None)
    gnames = ("dy", "q", "k", "v", "y", "lse", "o", "dq", "dk", "dv")
    bwd = lambda s, ws=FAKE, n=1 << 40, **null: lib.dc_attention_grad(s, *[null.get(a, FAKE) for a in gnames], None, ws, n,
                                                                     None)
    for bad in STRIDES + [dict(dtype=3), dict(dtype=-1), dict(heads=3), dict(heads=0), dict(kv_heads=0), dict(kv_heads=8), dict(D=0),
                          dict(D=129, q_head=129, k_head=129, v_head=129, q_token=999, k_token=999, v_token=999),
                          dict(sequences=-1), dict(sequences=2**20 + 1), dict(tokens=-1), dict(tokens=2**31 - 1023), dict(scale=3e38),
                          dict(scale=float("nan")), dict(scale=float("inf")), dict(v_head=63), dict(v_token=127)]:
        assert fwd(shape(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert bwd(shape(**bad)) == dc.DC_ERR_BAD_LAYER, bad
        assert lib.dc_attention_workspace_bytes(shape(**bad), 0, FAKE, FAKE, FAKE, FAKE) == 0
    assert fwd(None) == dc.DC_ERR_NULL and bwd(None) == dc.DC_ERR_NULL
    for null in names:
        assert fwd(shape(), **{null: None}) == dc.DC_ERR_NULL, null
    for null in gnames:
        assert bwd(shape(), **{null: None}) == dc.DC_ERR_NULL, null
    for grad, call in ((0, fwd), (1, bwd)):
        need = lib.dc_attention_workspace_bytes(shape(), grad, FAKE, FAKE, FAKE, FAKE)
        assert need > 0
        assert call(shape(), ws=None) == dc.DC_ERR_WORKSPACE and call(shape(), n=need - 1) == dc.DC_ERR_WORKSPACE
    assert fwd(shape(tokens=0), q=None) == dc.DC_OK and bwd(shape(tokens=0), q=None) == dc.DC_OK


def test_attention_workspace(lib):
    q = lambda s, grad=0, **p: lib.dc_attention_workspace_bytes(s, grad, *[p.get(a, FAKE) for a in ("q", "k", "v", "dy")])
    base = q(shape())
    assert q(shape(), 2) == 0 and q(shape(), -1) == 0 and q(None) == 0 and q(shape(tokens=0)) == 0
    # operands off 16-byte boundaries are copied: heads of 64 elements of 2 bytes
    assert q(shape(), q=FAKE + 2) >= base + 100 * 4 * 64 * 2
    assert q(shape(), v=FAKE + 2) >= base + 100 * 2 * 64 * 2
    assert q(shape(), 0, dy=FAKE + 2) == base and q(shape(), 1, dy=FAKE + 2) > q(shape(), 1)
    assert q(shape(scale=-1.0)) >= base + 100 * 4 * 64 * 2  # the copy negates q
    assert q(shape(dtype=2), q=FAKE + 4) == q(shape(dtype=2))  # floats are read as they lie
    # room for a short tile of every sequence
    assert q(shape(sequences=50000)) >= base + 49000 * (16 + 8)
    # few key heads: floats of the parts
    one, many = dict(heads=8, kv_heads=8, q_token=512, k_token=512, v_token=512), dict(heads=8, kv_heads=1, q_token=512)
    assert q(shape(**many), 1) >= 2 * 8 * 100 * 64 * 4
    assert q(shape(**one), 1) < 100 * 8 * 4 * 4 + 8192
