"""The products of sdl_orthogonalize have the bits that they are documented to have: errors over batches of matrices, under limits that fewer bits go beyond (test_orthogonalize_bits.py)."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32
from test_orthogonalize_bits import QUINTIC, ROWS, SHAPES, exact, is_split, limit, limit_in_bf16, momentum, rms

pytestmark = pytest.mark.gpu


def run(x, out):
    got, xg = torch.full(x.shape, float("nan"), dtype=out, device="cuda"), x.cuda()
    sdl.sdl_orthogonalize(xg, got, sdl.alloc_orthogonalize(xg, got), QUINTIC)
    return got.double().cpu()


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("shape", SHAPES + ROWS)
def test_results_in_fp32(shape, dtype):
    for seed in (7, 70):
        x = momentum(shape, dtype, seed)
        want = exact(x)
        off = rms(run(x, FP32) - want, want)
        print(f"orthogonalize {shape} {dtype} {off:.2e} of {limit(x, want, True):.2e}", flush=True)
        assert off <= limit(x, want, True)


@pytest.mark.parametrize("shape", SHAPES + ROWS)
def test_results_in_bf16(shape):
    for seed in (7, 70):
        x = momentum(shape, FP32, seed)
        want = exact(x)
        most = limit_in_bf16(limit(x, want, is_split(shape, BF16)))
        off = rms(run(x, BF16) - want.bfloat16().double(), want)
        print(f"orthogonalize {shape} {off:.2e} of {most:.2e}", flush=True)
        assert off <= most
