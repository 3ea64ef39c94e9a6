"""GPU parity of sdl_orthogonalize with singular values and vectors in 64 bits.

Bounds are on the root of the sum of squares.  What the documented roundings cost (operands of 11 bits, or 22 for results in fp32 and of small matrices, but for the diagonals of
symmetric ones; sums held in 24, X in 19 or 24) is found by doing them in 64 bits; the kernels' are others of the same kind, so twice that, and the rounding of the results.  A sum of K terms
in fp32 has K roundings instead of the one that is done there, which add up as their root: so many times as much for results in fp32, where they count."""
import math

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, output, placed, randn
from oracle import training as ref

pytestmark = pytest.mark.gpu
QUINTIC, CUBIC = sdl.ORTHOGONALIZE_QUINTIC, sdl.ORTHOGONALIZE_CUBIC
SHAPES = [(1, 1, 1), (2, 1, 9), (1, 7, 1), (3, 5, 5), (1, 64, 64), (2, 33, 65), (1, 65, 64), (1, 100, 131), (4, 128, 96), (1, 129, 300), (2, 200, 70), (1, 257, 513)]


def momentum(shape, dtype, seed):
    """A few directions that count, falling off, and noise."""
    B, R, C = shape
    r = max(1, min(R, C) // 8)
    x = randn((B, R, r), torch.float64, seed) * torch.logspace(0, -2, r, dtype=torch.float64)
    return ((x @ randn((B, r, C), torch.float64, seed + 1) / math.sqrt(r) + randn(shape, torch.float64, seed + 2, 0.05)) * 1e-3).to(dtype)


def tiny_bound(x, coefficients, eps, scale):
    """What products of 22 bits may cost matrices of up to eight rows, to first order.  What a step rounds, with F = |X|^2 (all norms the root of the sum of squares) and u four
    roundings of fp32, as an operand of 22 bits has:
      A of sums of m/4 + 8 times u:      dA <= (m/4 + 8) u F
      B = b A + c A^2, n terms:          dB <= |b| dA + |c| (2 F dA + (n + 1) u F^2) + 3 u (|b| F + |c| F^2)
      X' = a X + B X:                    e  <= dB |X| + (n + 2) u |B| |X| + 2 u (|a| |X| + |X'|)
    An error's part from the i-th left to the j-th right singular vector goes on through p(s) = a s + b s^3 + c s^5 as (p(si) - p(sj)) / (si - sj) times its symmetric and
    (p(si) + p(sj)) / (si + sj) times its antisymmetric half; beside the square (j > n) it is p(si) / si."""
    u = 4 * U32
    a = x.double()
    n, m = min(a.shape), max(a.shape)
    s = torch.linalg.svdvals(a / (a.norm() + eps))
    errors, ways = [4 * u], []        # of the first X
    for ca, cb, cc in coefficients:
        f, p = float(s.square().sum()), s * (ca + cb * s ** 2 + cc * s ** 4)
        d_a = (m / 4 + 8) * u * f
        d_b = abs(cb) * d_a + abs(cc) * (2 * f * d_a + (n + 1) * u * f * f) + 3 * u * (abs(cb) * f + abs(cc) * f * f)
        b = float((cb * s ** 2 + cc * s ** 4).norm())
        errors.append(d_b * f ** 0.5 + (n + 2) * u * b * f ** 0.5 + 2 * u * (abs(ca) * f ** 0.5 + float(p.norm())))
        t, slope = s[:, None] - s[None], ca + 3 * cb * s ** 2 + 5 * cc * s ** 4
        minus = torch.where(t.abs() > 1e-9, (p[:, None] - p[None]) / torch.where(t.abs() > 1e-9, t, 1.0), slope[:, None]).abs()
        plus = ((p[:, None] + p[None]) / (s[:, None] + s[None]).clamp(min=1e-300)).abs()
        ways.append(torch.cat([torch.maximum(minus, plus), (p / s.clamp(min=1e-300)).abs()[:, None]], 1))
        s = p.abs()
    total, way = errors[-1], torch.ones_like(ways[0])
    for e, w in zip(errors[-2::-1], ways[::-1]):
        way = way * w
        total += e * float(way.max())
    return abs(scale) * total


def check(x, out_dtype, coefficients=QUINTIC, eps=1e-7, scale=1.0, how="dense"):
    out, alone = output(torch.empty(x.shape, dtype=out_dtype), how)
    xg = placed(x, how)
    space = sdl.alloc_orthogonalize(xg, out)
    space.fill_(0xff)               # NaN in every image that would be read before it is written
    sdl.sdl_orthogonalize(xg, out, space, coefficients, eps, scale)
    torch.cuda.synchronize()
    assert alone()
    for b in range(x.shape[0]):
        want = ref.orthogonalize(x[b], coefficients, eps, scale)
        split = out_dtype == FP32 or min(x.shape[1:]) <= 16 or x[b].numel() <= 2048
        rounded = ref.orthogonalize_rounded(x[b], coefficients, eps, scale, 22 if split else 11, 24, 24 if split else 19)
        cost = float((rounded - want).norm())
        times = 2.0 if out_dtype == BF16 else 2.0 + math.sqrt(max(x.shape[1:]))
        bound = times * cost + (U[out_dtype] + 16 * U32) * float(want.norm())
        if min(x.shape[1:]) <= 8 and x[b].numel() <= 2048:      # the roundings of so few products differ by more than twice
            bound = max(bound, tiny_bound(x[b], coefficients, eps, scale) + (U[out_dtype] + 16 * U32) * float(want.norm()))
        got = out[b].double().cpu()
        assert not torch.isnan(got).any(), (tuple(x.shape), b)
        off = float((got - want).norm())
        assert off <= bound, (tuple(x.shape), b, off, bound, cost)
        # no element is left out of the sum
        assert float((got - want).abs().max()) <= max(bound, 1e-30)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (FP32, FP32), (FP32, BF16), (BF16, FP32)])
def test_momentum(dtype, out):
    for i, shape in enumerate(SHAPES):
        print(f"orthogonalize {shape} {dtype} {out}", flush=True)
        check(momentum(shape, dtype, 10 * i), out, scale=(1.0, 0.2, -3.0)[i % 3])


@pytest.mark.parametrize("out", [BF16, FP32])
def test_every_launch_shape(out):
    """A workgroup a matrix of all kinds, up to what they hold; tiles of 64, of 128 and of 256; sums in slices."""
    for i, shape in enumerate([(3, 48, 80), (2, 16, 500), (3, 90, 90), (2, 112, 176), (1, 17, 1000), (2, 160, 180), (1, 32, 1300), (2, 200, 300), (1, 300, 520), (1, 180, 2100),
                               (40, 200, 400), (36, 385, 129), (2, 1024, 1100), (1, 513, 4000), (6, 700, 1600), (1, 2100, 180), (1, 900, 300), (2, 15, 2900), (2, 31, 2900), (1, 32, 1210),
                               (3, 1217, 16), (3, 1217, 17), (1, 1, 4099), (257, 40, 100), (257, 31, 40), (257, 50, 45), (3, 8, 256), (2, 8, 257), (3, 1, 2048),
                               (2, 1, 2049), (5, 300, 6), (300, 2, 2), (3, 9, 20)]):
        print(f"orthogonalize {shape} {out}", flush=True)
        check(momentum(shape, FP32, 10 * i), out)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_where_they_lie(dtype):
    for i, shape in enumerate([(2, 33, 70), (3, 90, 17), (1, 130, 129)]):
        check(momentum(shape, dtype, 50 + i), dtype, how="odd")


@pytest.mark.parametrize("out", [BF16, FP32])
def test_other_coefficients(out):
    x = momentum((2, 48, 80), FP32, 3)
    check(x, out, CUBIC)
    check(x, out, [(1.0, 0.0, 0.0)])
    check(x, out, [(0.0, 0.0, 0.0)])
    check(x, out, [(-1.5, 0.5, 0.0), (2.0, -1.5, 0.5), (1.0, 1e-9, -1e-9)])
    check(x, out, [(1.5, -0.5, 0.0)] * 30)
    check(x, out, eps=1.0)


def test_sizes_of_numbers():
    """Norms far from 1: their squares do not fit 32 bits."""
    x = randn((3, 20, 30), FP32, 4) * torch.tensor([1e30, 1e-28, 1.0])[:, None, None]
    check(x, FP32, eps=0.0)
    check(x[2:], FP32, eps=1e-7)
    tiny = torch.zeros(1, 20, 30)
    tiny[0, 3, 4] = 1e-40
    check(tiny, FP32)


def test_low_rank_and_orthogonal():
    a = randn((1, 60, 2), FP32, 1) @ randn((1, 2, 90), FP32, 2)
    check(a, FP32)
    check(a, BF16)
    check(randn((1, 300, 2), FP32, 1) @ randn((1, 2, 520), FP32, 2), BF16)
    q = torch.linalg.qr(randn((64, 64), torch.float64, 3))[0].float().contiguous()[None]
    check(q, FP32)
    got, space = torch.empty(1, 64, 64, device="cuda"), sdl.alloc_orthogonalize(q.cuda(), q.cuda())
    sdl.sdl_orthogonalize(q.cuda(), got, space, CUBIC * 2)
    # the cubic steps go to 1 from 1 / 8, quadratically: an orthogonal matrix comes back.  24 steps of about 64 u each on numbers of size 1
    assert float((got.cpu() - q).norm()) < 24 * 64 * U32 * 8


@pytest.mark.parametrize("shape", [(5, 40, 50), (5, 300, 520), (5, 700, 260)])
def test_zeros_and_what_is_not_finite(shape):
    x = momentum(shape, FP32, 5)
    x[1] = 0.0
    x[2, 3, 4], x[3, 39, 49] = math.nan, math.inf
    clean = x.clone()
    clean[2:4] = 0.0
    for out in (BF16, FP32):
        got, want = (torch.empty(shape, dtype=out, device="cuda") for _ in range(2))
        for eps in (1e-7, 0.0):
            sdl.sdl_orthogonalize(x.cuda(), got, sdl.alloc_orthogonalize(x.cuda(), got), eps=eps)
            sdl.sdl_orthogonalize(clean.cuda(), want, sdl.alloc_orthogonalize(x.cuda(), got), eps=eps)
            assert not got[1].any()
            assert torch.isnan(got.float()).flatten(1).any(1).tolist() == [False, False, True, True, False]
            assert torch.equal(got[[0, 1, 4]], want[[0, 1, 4]])


@pytest.mark.parametrize("shape", [(3, 100, 130), (300, 20, 30), (40, 256, 430), (1, 200, 2100)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_in_place_repeatable_on_another_stream_and_in_a_graph(shape, dtype):
    x = momentum(shape, dtype, 6).cuda()
    out, space = torch.empty_like(x), sdl.alloc_orthogonalize(x, x)
    sdl.sdl_orthogonalize(x, out, space)
    place = x.clone()
    sdl.sdl_orthogonalize(place, place, space)
    assert torch.equal(out, place)
    side, again = torch.cuda.Stream(), torch.empty_like(x)
    side.wait_stream(torch.cuda.current_stream())
    sdl.sdl_orthogonalize(x, again, torch.empty_like(space), stream=side)
    side.synchronize()
    assert torch.equal(out, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdl.sdl_orthogonalize(x, out, space, scale=0.5)
    for replay in range(3):
        x.copy_(momentum(shape, dtype, 60 + replay))
        space.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        sdl.sdl_orthogonalize(x, again, torch.empty_like(space), scale=0.5)
        assert torch.equal(out, again)


def test_a_matrix_alone_and_in_a_batch_of_no_rows():
    x = momentum((1, 30, 40), FP32, 7).cuda()
    out, flat = torch.empty_like(x), torch.empty(30, 40, device="cuda")
    space = sdl.alloc_orthogonalize(x, out)
    sdl.sdl_orthogonalize(x, out, space)
    sdl.sdl_orthogonalize(x[0], flat, space)
    assert torch.equal(out[0], flat)
    none = torch.empty(0, 30, 40, device="cuda")
    sdl.sdl_orthogonalize(none, none, None)
