"""Attention where (sequence, key head)s have several blocks of rows and of keys each, as training micro-batches do: keys and values beyond what one die's cache
holds, workgroups of four and of eight wavefronts, nothing cut into chunks; and rows of all widths."""
import pytest

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32
from test_gpu_attention import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", [
    (4, 300, 300, 32, 32, 72, False, None, None),                  # eight wavefronts, two blocks each
    (8, 300, 300, 32, 32, 104, True, None, None),
    (8, 300, 333, 64, 16, 96, True, [300, 0, 1, 255, 256, 257, 299, 32], [333, 200, 5, 300, 20, 257, 128, 129]),
    (8, 300, 300, 32, 32, 64, True, None, None),                   # four wavefronts, three blocks each
    (4, 300, 300, 32, 8, 128, False, None, [300, 0, 257, 31]),      # ten blocks of a group's rows
    (7, 390, 390, 19, 19, 24, True, None, None)])                  # units that are no multiple of four
def test_several_blocks_of_rows_and_keys(dtype, case):
    assert 2 * case[0] * case[2] * case[4] * case[5] * (2 if dtype == BF16 else 4) > 4 << 20 or case[5] == 24
    _check(case, dtype, seed=21)


@pytest.mark.parametrize("case", [(2, 1100, 1100, 32, 32, 64, True, None, None), (4, 1100, 1100, 26, 26, 72, True, None, [1100, 1000, 17, 0]),
                                  (2, 2050, 2050, 16, 16, 80, False, None, None)])
def test_long_sequences_of_many_heads(case):
    assert sdl.sdl_attention_workspace_bytes(*case[:6], sdl.DTYPE_BF16) == 0
    _check(case, BF16, seed=22)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_of_every_kind_of_width(dtype):
    """Widths that are no multiple of eight, in many rows and in few, on and off their alignment."""
    for i, width in enumerate((3, 7, 8, 9, 12, 15, 31, 41, 62, 66, 95, 97, 100, 119, 127)):
        for how in ("dense", "odd"):
            print(f"attention width {width} {how} {dtype}", flush=True)
            _check((2, 70, 75, 2, 1, width, True, [70, 33], [75, 40]), dtype, how, seed=500 + i)
            _check((1, 1, 200, 4, 2, width, True, None, [131]), dtype, how, seed=600 + i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", [
    (8, 1, 8300, 8, 4, 128, True, None, [8300, 1, 0, 4000, 31, 32, 33, 8299]), (8, 2, 11000, 4, 4, 96, True, None, None),
    (8, 1, 16500, 4, 4, 64, False, None, [16500, 5, 0, 128, 129, 9000, 12345, 64]), (9, 1, 33000, 4, 4, 32, True, None, None)])
def test_caches_that_go_past_the_devices_own(dtype, case):
    """Single tokens over keys and values of 128 MB and more."""
    assert 2 * case[0] * case[2] * case[4] * case[5] * 2 >= 1 << 27
    for how in ("dense", "heads"):
        _check(case, dtype, how, seed=23)
