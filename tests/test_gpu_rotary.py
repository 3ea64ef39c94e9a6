"""GPU parity of sdl_rotary with the 64-bit oracle.

Bound: cosine and sine of the reduced angle are good to 4 u(fp32) (an angle in turns, rounded once, and a function of two units), the scale and the
two products and their sum cost a rounding each: 8 u (|a| + |b|) |scale|, and the type's own rounding."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, output, placed, randn
from oracle import innerstep as ref

pytestmark = pytest.mark.gpu


def _check(shape, dtype, rot, interleaved, positions, how="dense", scale=1.0, inverse=False, seed=0, frequencies=None, first=0):
    x = randn(shape, dtype, seed)
    f = sdl.sdl_rotary_frequencies(rot) if frequencies is None else frequencies
    out, alone = output(x, how)
    sdl.sdl_rotary(placed(x, how), None if positions is None else positions.cuda(), f.cuda(), out,
                   sdl.ROTARY_INTERLEAVED if interleaved else sdl.ROTARY_HALF, scale, inverse, first)
    torch.cuda.synchronize()
    p = first + torch.arange(shape[1]).expand(shape[:2]) if positions is None else positions
    want = ref.rotary(x, p, f, interleaved, scale, inverse)
    # the larger of a pair's two sums of absolute values
    size = ref.rotary(torch.ones(shape), torch.zeros_like(p), f, interleaved, 1.0, False)
    X = x.double().abs()
    half, pair = rot // 2, torch.zeros(shape, dtype=torch.float64)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    pair[..., a] = pair[..., b] = X[..., a] + X[..., b]
    assert size.shape == want.shape
    close(out, want, U[dtype] * want.abs() + 8 * U32 * abs(scale) * pair, f"rotary {shape} {rot}")
    assert torch.equal(out[..., rot:].cpu(), x[..., rot:]) and alone()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts_parts_and_sizes(dtype, interleaved):
    gen = torch.Generator().manual_seed(1)
    for i, (shape, rot) in enumerate([((1, 1, 1, 2), 2), ((2, 3, 2, 8), 8), ((1, 5, 3, 64), 64), ((3, 2, 5, 128), 128), ((2, 7, 1, 80), 20),
                                      ((2, 3, 4, 33), 18), ((1, 9, 2, 256), 96), ((2, 2, 3, 96), 2), ((1, 4, 40, 128), 128), ((2, 3, 2, 31), 30)]):
        for how in ("dense", "odd", "packed", "heads"):
            print(f"rotary {shape} {rot} {how}", flush=True)
            positions = torch.randint(-5, 3000, shape[:2], generator=gen, dtype=torch.int32)
            _check(shape, dtype, rot, interleaved, positions, how, 1.0 if i % 2 else 1.25, i % 3 == 0, seed=i)


def test_positions_far_out_and_counted():
    for first in (0, 1, 99999, 1 << 20, 2 ** 31 - 8, -(2 ** 31)):
        _check((1, 8, 2, 64), FP32, 64, False, None, first=first)
    _check((2, 3, 2, 64), FP32, 64, True, torch.tensor([[0, 10 ** 6, 2 ** 31 - 1], [-(2 ** 31), -1, 7]], dtype=torch.int32))


def test_scaled_frequencies():
    for scaling in (dict(scaling=sdl.ROTARY_LINEAR, factor=8.0), dict(scaling=sdl.ROTARY_PARTS, factor=32.0, low=1.0, high=4.0, trained_length=8192)):
        f = sdl.sdl_rotary_frequencies(128, 500000.0, **scaling)
        _check((2, 3, 4, 128), BF16, 128, False, torch.tensor([[1, 77, 131071], [5, 8192, 60000]], dtype=torch.int32), scale=1.1, frequencies=f)


def test_there_and_back_in_place_on_another_stream():
    x = randn((2, 300, 9, 96), FP32, 4).cuda()
    f = sdl.sdl_rotary_frequencies(64).cuda()
    positions = torch.arange(600, dtype=torch.int32).view(2, 300).cuda()
    out, y = torch.empty_like(x), x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sdl.sdl_rotary(x, positions, f, out)
    sdl.sdl_rotary(y, positions, f, y, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, y)
    sdl.sdl_rotary(y, positions, f, y, inverse=True)
    # two turns, 8 u (|a| + |b|) each, and the pair's length is kept
    assert float((y - x).abs().max()) < 2 * 8 * U32 * 2 * float(x.abs().max()) * 1.5


def test_nothing_to_turn():
    x = randn((2, 3, 1, 7), BF16, 5).cuda()
    out = torch.zeros_like(x)
    none = torch.empty(0, dtype=torch.float64, device="cuda")
    sdl.sdl_rotary(x, None, none, out)
    assert torch.equal(out, x)
    sdl.sdl_rotary(x, None, none, x)
    assert torch.equal(out, x)
    empty = torch.empty(0, 3, 1, 8, device="cuda")
    sdl.sdl_rotary(empty, None, sdl.sdl_rotary_frequencies(8).cuda(), empty)


def test_gradient_against_differences():
    """<J dy, way> of the inverse turn is <dy, J way> of the turn."""
    x = randn((1, 6, 2, 40), FP32, 6)
    dy, f = randn(x.shape, FP32, 7), sdl.sdl_rotary_frequencies(24)
    positions = torch.arange(50, 56, dtype=torch.int32).view(1, 6)
    dx = torch.empty(x.shape, device="cuda")
    sdl.sdl_rotary(dy.cuda(), positions.cuda(), f.cuda(), dx, sdl.ROTARY_INTERLEAVED, 1.5, inverse=True)
    way = randn(x.shape, torch.float64, 8)
    loss = lambda x: float((ref.rotary(x, positions, f, True, 1.5, False)[..., :24] * dy.double()[..., :24]).sum())  # noqa: E731
    slope = (loss(x.double() + 1e-4 * way) - loss(x.double() - 1e-4 * way)) / 2e-4
    mine = (dx.cpu().double() * way)[..., :24]
    assert abs(slope - float(mine.sum())) < 1e-5 * float(mine.abs().sum())
