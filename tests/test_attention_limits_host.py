"""Calls of attention whose loops would not fit their counters are refused on the host (no GPU)."""
import ctypes

import pytest

from paper_2101_07968_gb300 import build as libbuild
from paper_2101_07968_gb300 import dynacomm as dc

FAKE = 0x1000  # never dereferenced: the calls fail or are not made
MOST = dc.DC_ATTENTION_TOKENS_MAX


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dc.lib()


def shape(tokens, heads, kv_heads, dtype=0):
    return ctypes.byref(dc.dc_attention_shape(dtype, heads, kv_heads, 8, 1, tokens, heads * 8, 8, kv_heads * 8, 8,
                                              kv_heads * 8, 8, 1.0))


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_steps_of_an_item(lib, dtype):
    """A tile of keys is taken with every 64 rows of every head that reads it: at most 2^31 - 1 steps."""
    need = lambda *s: lib.dc_attention_workspace_bytes(shape(*s, dtype), 1, FAKE, FAKE, FAKE, FAKE)
    for tokens, heads, kv_heads in ((MOST, 64, 1), (MOST, 1024, 16), (2**27, 1024, 1), (MOST, 1, 1)):
        fits = (tokens // 64 + 1) * (heads // kv_heads) < 2**31
        assert (need(tokens, heads, kv_heads) > 0) == fits, (tokens, heads, kv_heads)
    for tokens, heads, kv_heads in ((MOST, 65, 1), (MOST, 1024, 1), (2**27 + 64, 1024, 1)):
        assert need(tokens, heads, kv_heads) == 0
        args = [FAKE] * 6
        assert lib.dc_attention(shape(tokens, heads, kv_heads, dtype), *args, None, FAKE, 1 << 60, None) == dc.DC_ERR_BAD_LAYER
        assert lib.dc_attention_grad(shape(tokens, heads, kv_heads, dtype), *[FAKE] * 10, None, FAKE, 1 << 60,
                                     None) == dc.DC_ERR_BAD_LAYER
