"""sdl_orthogonalize of matrices of low rank: whatever rounding puts into the directions that are not there is lifted with every step, 480 times by the five quintic ones."""
import math

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32
from oracle import training as ref
from test_orthogonalize_bits import QUINTIC, exact, limit_in_bf16, rms

pytestmark = pytest.mark.gpu


def of_rank(r, shape, seed):
    gen = torch.Generator().manual_seed(seed)
    B, R, C = shape
    return torch.randn(B, R, r, generator=gen) @ torch.randn(B, r, C, generator=gen)


def run(x, out, coefficients):
    got, xg = torch.full(x.shape, float("nan"), dtype=out, device="cuda"), x.cuda()
    sdl.sdl_orthogonalize(xg, got, sdl.alloc_orthogonalize(xg, got), coefficients)
    return got.double().cpu()


@pytest.mark.parametrize("shape", [(2048, 2048), (2560, 2048)])
def test_x_between_steps_has_the_digits_of_fp32(shape):
    """Eight quintic steps of rank one lift what is there by chance 20000 times.  X kept with 20 bits between them (11 and what that leaves in 8) costs 1.4 times what the operands' 11 bits
    do by themselves in the oracle; its own sums in fp32 are a tenth of that, and the results' rounding is 2^-8 of an element at most."""
    x = of_rank(1, (1, *shape), 1)
    steps = QUINTIC[:1] * 8
    s = 1.0
    for a, b, c in steps:
        s = a * s + b * s ** 3 + c * s ** 5
    want = s * x.double() / (x.double().norm() + 1e-7)
    cost = rms(ref.orthogonalize_rounded(x[0], steps, 1e-7, 1.0, 11, 24, 24)[None] - want, want)
    off = rms(run(x, BF16, steps) - want, want)
    print(f"orthogonalize {shape} {off:.2e}, operands {cost:.2e}", flush=True)
    assert off <= ((1.2 * cost) ** 2 + 2.0 ** -18) ** 0.5


def limit(x, want):
    """What 22 bits cost in the oracle, where an element of a product is rounded once to 24 bits and one of X too.  In the kernels its sum has N = rows / 16 roundings of what it has got to,
    0.42 sqrt(N / 3) u together instead of 0.3 u, and all of that is lifted alike."""
    cost = rms(torch.stack([ref.orthogonalize_rounded(m, QUINTIC, 1e-7, 1.0, 22, 24, 24) for m in x]) - want, want)
    return (2.0 + 1.5 * math.sqrt(math.ceil(min(x.shape[1:]) / 16) / 3.0)) * cost


@pytest.mark.parametrize("rank", [1, 4])
@pytest.mark.parametrize("shape", [(8, 8, 2000), (16, 17, 100), (30, 24, 24), (8, 45, 46), (8, 64, 64), (8, 80, 48), (4, 100, 131), (2, 512, 128), (2, 200, 300), (2, 256, 256), (1, 256, 1024)])
def test_up_to_256_rows_are_off_by_little_more_than_the_results_rounding(shape, rank):
    x = of_rank(rank, shape, 10 + rank)
    want = exact(x)
    most = limit(x, want)
    off = rms(run(x, FP32, QUINTIC) - want, want), rms(run(x, BF16, QUINTIC) - want.bfloat16().double(), want)
    print(f"orthogonalize {shape} rank {rank} {off[0]:.2e} of {most:.2e}, {off[1]:.2e} of {limit_in_bf16(most):.2e}", flush=True)
    assert off[0] <= most
    assert off[1] <= limit_in_bf16(most)


@pytest.mark.parametrize("shape", [(2, 257, 300), (1, 384, 384), (1, 1000, 520), (1, 768, 768)])
def test_above_that_by_less_than_the_results_rounding(shape):
    """One image of 11 bits: 0.42 / rows of rank one, under 0.0017."""
    x = of_rank(1, shape, 20)
    want = exact(x)
    off = rms(run(x, BF16, QUINTIC) - want, want)
    print(f"orthogonalize {shape} {off:.2e}", flush=True)
    # half a step of bf16 is 2^-8 of an element at most, of all of them in the mean of squares 2^-9.2
    assert off <= ((1.2 * 0.42 / min(shape[1:])) ** 2 + 2.0 ** -18.4) ** 0.5
