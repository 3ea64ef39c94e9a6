"""sdl_orthogonalize of matrices of low rank: whatever rounding puts into the directions that are not there is lifted with every step, 480 times by the five quintic ones."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16
from oracle import training as ref
from test_orthogonalize_bits import QUINTIC, rms

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
