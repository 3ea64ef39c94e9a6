"""Sizes and numbers at the edge of what the operators of the inner step take (CPU only: a refused call touches no address)."""
import pytest

import paper_2501_18512_amd as sdl

INVALID, UNSUPPORTED, ALIGNMENT, OK = -1, -2, -3, 0


def view(data, batch=1 << 20, token=1 << 10, head=128):
    return sdl._View(data, batch, token, head)


def rotary(batch, tokens, heads, width=64, rot=64, out=0x40000):
    return sdl._lib.sdl_rotary(view(0x10000), batch, tokens, heads, width, sdl.DTYPE_BF16, rot, sdl.ROTARY_HALF, None, 0, 0x30000, 1.0, 0, view(out), None)


@pytest.mark.parametrize("shape", [
    (1 << 31, 1 << 31, 4), (1 << 31, 1 << 31, 1), (1 << 31, 1 << 31, 1 << 31), (1 << 16, 1 << 16, 1 << 30), (0xffffffff, 0xffffffff, 0xffffffff),
    (0xffffffff, 1, 0xffffffff), (1, 1, 0xffffffff), (1 << 29, 1, 1), (1 << 14, 1 << 14, 2)])
def test_rotary_of_too_many_groups_is_refused(shape):
    """Also where the number of tokens, or of groups of pairs, is a multiple of 2^64."""
    assert rotary(*shape) == UNSUPPORTED
    assert rotary(*shape, out=0x10000) == UNSUPPORTED
