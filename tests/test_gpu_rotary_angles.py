"""Rotary positions whose angle counts: positions behind the last 32-bit one, and angles next to whole half turns, where a sine or a cosine is small."""
import math

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, randn
from oracle import innerstep as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("first", [2 ** 31 - 4, 2 ** 31 - 1, 2 ** 31 - 300])
def test_counted_positions_go_on_behind_the_last_of_32_bits(first, dtype):
    """Token t stands at first_position + t, whatever that comes to."""
    x, f = randn((1, 300, 1, 8), dtype, 1), sdl.sdl_rotary_frequencies(8)
    out = torch.empty_like(x, device="cuda")
    sdl.sdl_rotary(x.cuda(), None, f.cuda(), out, first_position=first)
    torch.cuda.synchronize()
    want = ref.rotary(x, first + torch.arange(300)[None], f, False, 1.0, False)
    # the angle: 2^31 positions in fp64 are good to 2^31 times a few units of 2^-53, under one of 2^-20; the rest as everywhere: 8 u of the pair
    X = x.double().abs()
    pair = (X[..., :4] + X[..., 4:]).repeat(1, 1, 1, 2)
    close(out, want, U[dtype] * want.abs() + (8 * U32 + 4 * 2.0 ** 31 * 2.0 ** -53) * pair, f"first {first}")
