"""How many bits sdl_orthogonalize's products have: a limit on its errors that one image where two belong goes beyond, shown here with the oracle's roundings (CPU only); the kernels are
held to it in test_gpu_orthogonalize_bits.py.

The limit is on the root mean square, over a batch, of |error| / |result|.  What is documented costs is found by rounding in 64 bits (oracle.training.orthogonalize_rounded), for the same
matrices; four times that, for other roundings of the same kind.  Beside it, the sums in fp32, which are rounded once there: a sum of squares on A's diagonal grows with N = K / 16
instructions, each rounding 0.42 u of what it has got to (u / sqrt(3) at most, and 1 / sqrt(2) of that for where between two powers of two it lies), in all 0.42 sqrt(N / 3) u of the sum.
B = b A + c A^2 of a row of X with singular values near 1 changes by (|b| s^2 + 2 |c| s^4) / p(s), 13 on average of 0.7 to 1.15 with the quintic coefficients, times as much, and what
the last two steps add counts: 13 sqrt(2) 0.42 sqrt(N / 3) u = 8 sqrt(N / 3) u, and as much again for the sums of B X."""
import math

import pytest
import torch

from operator_util import BF16, FP32, U32, randn
from oracle import training as ref

QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5
# matrices enough that a mean tells; a workgroup a matrix of every kind, and tiles
SHAPES = [(300, 2, 2), (200, 5, 5), (60, 3, 20), (60, 20, 9), (30, 8, 256), (30, 256, 8), (16, 5, 300), (16, 300, 6), (30, 16, 16), (30, 17, 17), (16, 17, 100), (270, 24, 24), (16, 31, 40),
          (8, 45, 45), (8, 64, 64), (8, 50, 45), (4, 100, 131), (4, 131, 100), (8, 16, 500), (2, 200, 300), (2, 129, 70), (1, 256, 700), (1, 257, 300), (1, 400, 801), (1, 385, 129)]
ROWS = [(200, 1, 9), (60, 12, 1), (60, 1, 100), (16, 1, 2048), (16, 1, 2049)]


def momentum(shape, dtype, seed):
    """A few directions that count, falling off, and noise."""
    B, R, C = shape
    r = max(1, min(R, C) // 8)
    x = randn((B, R, r), torch.float64, seed) * torch.logspace(0, -2, r, dtype=torch.float64)
    return ((x @ randn((B, r, C), torch.float64, seed + 1) / math.sqrt(r) + randn(shape, torch.float64, seed + 2, 0.05)) * 1e-3).to(dtype)


def is_split(shape, out):
    """Whether products have 22 bits, as the header says."""
    return out == FP32 or min(shape[1:]) <= 256


def exact(x, coefficients=QUINTIC):
    return torch.stack([ref.orthogonalize(m, coefficients, 1e-7, 1.0) for m in x])


def rms(off, want):
    return float((off.flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)).square().mean().sqrt())


def limit(x, want, split, coefficients=QUINTIC):
    """Of the results before they are rounded to their type."""
    rounded = torch.stack([ref.orthogonalize_rounded(m, coefficients, 1e-7, 1.0, 22 if split else 11, 24, 24 if split else 19) for m in x])
    return 4.0 * rms(rounded - want, want) + 16.0 * math.sqrt(math.ceil(max(x.shape[1:]) / 16.0) / 3.0) * U32


def limit_in_bf16(unrounded):
    """Of how far the results in bf16 are from the exact ones in bf16, which differ where an error goes over the middle of two neighbours: of an element in |error| / step, each by a step, at most
    2^-7 of the element.  The mean of error times step is at most the product of their roots of squares; twice that root, for a mean over the elements that there are."""
    return 2.0 * math.sqrt(unrounded * 2.0 ** -7)


def worse(x, coefficients, in_x, in_a, in_b):
    """The steps with operands of so many bits where X, A and B = b A + c A^2 are one."""
    def to(v, n):
        m, e = torch.frexp(v)
        return torch.ldexp((m * 2.0 ** n).round() * 2.0 ** -n, e)

    def cut(v, n):
        d = torch.diag(v.diagonal())
        return d, to(v - d, n)
    out = []
    for m in x:
        m = m.double()
        tall = m.shape[0] > m.shape[1]
        m = (m.T if tall else m) / (m.square().sum().sqrt() + 1e-7)
        for a, b, c in coefficients:
            low = to(m, in_x)
            d, gram = cut(low @ low.T, in_a)
            d, mix = cut(b * (d + gram) + c * (gram @ gram + d @ gram + gram @ d + d @ d), in_b)
            m = a * m + d @ m + mix @ low
        out.append(m.T if tall else m)
    return torch.stack(out)


@pytest.mark.parametrize("shape", SHAPES)
def test_fewer_bits_of_any_operand_go_beyond_the_limit(shape):
    x = momentum(shape, FP32, 7)
    want = exact(x)
    most = limit(x, want, True)
    assert rms(worse(x, QUINTIC, 22, 22, 22) - want, want) < most / 2
    for few in (11, 14):            # one image instead of two, and less than that
        for bits in ((few, 22, 22), (22, few, 22), (22, 22, few)):
            assert rms(worse(x, QUINTIC, *bits) - want, want) > most, (few, bits)


@pytest.mark.parametrize("shape", ROWS)
def test_fewer_bits_of_a_row_alone_go_beyond_the_limit(shape):
    """A and B have nothing but a diagonal."""
    x = momentum(shape, FP32, 7)
    want = exact(x)
    assert rms(worse(x, QUINTIC, 11, 22, 22) - want, want) > limit(x, want, True)


@pytest.mark.parametrize("shape", [s for s in SHAPES if is_split(s, BF16)])
def test_one_image_goes_beyond_the_limit_of_results_in_bf16(shape):
    x = momentum(shape, FP32, 7)
    want = exact(x)
    got = worse(x, QUINTIC, 11, 11, 11)
    assert rms(got.bfloat16().double() - want.bfloat16().double(), want) > limit_in_bf16(limit(x, want, True))
