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


def attention(scale=0.1, batch=2, queries=3, keys=5, heads=4, kv_heads=2, width=64):
    return sdl._lib.sdl_attention(view(0x10000), view(0x20000), view(0x30000), batch, queries, keys, heads, kv_heads, width, sdl.DTYPE_BF16, scale, 1, None, None,
                                  view(0x40000), 0x50000, 0x60000, 1 << 30, None)


def attention_backward(scale=0.1, batch=2, queries=3, keys=5, heads=4, kv_heads=2, width=64):
    return sdl._lib.sdl_attention_backward(*[view(0x10000 * i) for i in range(1, 6)], 0x60000, batch, queries, keys, heads, kv_heads, width, sdl.DTYPE_BF16, scale, 1,
                                           None, None, view(0x70000), view(0x80000), view(0x90000), 0xa0000, 1 << 30, None)


@pytest.mark.parametrize("call", [attention, attention_backward])
@pytest.mark.parametrize("scale", [2.4e38, 3.4028234e38])
def test_attention_refuses_a_scale_that_is_not_finite_times_log2_e(call, scale):
    """The kernels work in powers of two: with an infinite factor a score of 0 would be no number."""
    assert call(scale=scale) == INVALID
