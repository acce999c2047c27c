"""How the head norms deal a token's heads to groups of lanes (no GPU): every part has a head, and the
parts hold each head once, whatever the number of heads and tokens."""
import ctypes

import pytest

from paper_2101_07968_gb300 import build as libbuild
from paper_2101_07968_gb300 import dynacomm as dc


@pytest.fixture(scope="module")
def parts_of():
    libbuild.build()
    probe = dc.lib().dc_head_parts_probe
    parts, per = ctypes.c_int32(), ctypes.c_int32()

    def call(tokens, heads, wanted, least):
        probe(tokens, heads, wanted, least, ctypes.byref(parts), ctypes.byref(per))
        return parts.value, per.value
    return call


@pytest.mark.parametrize("least", [1, 2])
@pytest.mark.parametrize("units", [8, 16, 32])
def test_every_part_has_heads(parts_of, least, units):
    """units: heads that a block takes at a time, of one warp or several groups of lanes each."""
    for heads in range(1, 1025):
        for tokens in (1, 2, 3, 37, 600, 5000):
            parts, per = parts_of(tokens, heads, 152 * units, least)
            assert parts >= 1 and per >= 1
            assert (parts - 1) * per < heads <= parts * per, (heads, tokens, parts, per)


def test_parts_fill_the_gpu(parts_of):
    """As fine as needed and no finer: one part with many tokens, a head or two a part with one."""
    assert parts_of(5000, 40, 152 * 16, 2) == (1, 40)
    assert parts_of(1, 16, 152 * 16, 2) == (8, 2)
    for heads in (5, 6, 12, 40, 513):
        assert parts_of(1, heads, 152 * 16, 2)[1] <= 2
