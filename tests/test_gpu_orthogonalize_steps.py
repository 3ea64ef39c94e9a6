"""sdl_orthogonalize with more steps than one launch of small matrices takes, against the 64-bit oracle and against the same steps in separate calls."""
import ctypes

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32
from test_gpu_orthogonalize import CUBIC, check, momentum

pytestmark = pytest.mark.gpu
# a workgroup a matrix of every kind, with one image and with two, wide and tall; and tiles
SHAPES = [(2, 6, 9), (3, 24, 24), (2, 40, 30), (1, 64, 64), (1, 100, 131), (300, 20, 30), (2, 112, 176), (1, 200, 300)]


@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("steps", [31, 32, 33, 64])
def test_many_steps(steps, out):
    for i, shape in enumerate(SHAPES):
        print(f"orthogonalize {shape} {out} {steps} steps", flush=True)
        check(momentum(shape, FP32, 10 * i)[:3] if shape[0] > 3 and steps != 33 else momentum(shape, FP32, 10 * i), out, [(1.5, -0.5, 0.0)] * steps, how="odd" if i % 3 == 1 else "dense")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("shape", [(5, 30, 50), (2, 50, 30), (2, 64, 64), (1, 100, 150)])
def test_steps_that_change_nothing_keep_the_bits(shape, dtype):
    """X = X: what 5 steps give is what they give among 32, 33, 70 and 200, in place too, with no more workspace than is asked for."""
    x = momentum(shape, dtype, 3).cuda()
    numbers = lambda steps: (ctypes.c_float * (3 * len(steps)))(*[v for s in steps for v in s])  # noqa: E731
    kind = {FP32: 0, BF16: 1}[dtype]
    size = sdl.sdl_orthogonalize_workspace_bytes(*shape, kind)
    want = None
    for steps in (5, 32, 33, 70, 200):
        for place in (False, True):
            out = x.clone() if place else torch.full_like(x, float("nan"))
            source = out if place else x
            space = torch.full((size + 256,), 0xff, dtype=torch.uint8, device="cuda")
            view = lambda t: sdl._View(t.data_ptr(), t.stride(0), t.stride(1), 0)  # noqa: E731
            # the real ones first, and once at the end of a launch and the start of the next
            todo = list(CUBIC[:5]) + [(1.0, 0.0, 0.0)] * (steps - 5)
            torch.cuda.synchronize()
            status = sdl._lib.sdl_orthogonalize(view(source), *shape, kind, numbers(todo), steps, 1e-7, 0.5, view(out), kind, space.data_ptr(), size, None)
            torch.cuda.synchronize()
            assert status == 0 and bool((space[size:] == 0xff).all())
            if want is None:
                want = out
            assert torch.equal(out, want), (steps, place)


def test_a_graph_of_many_steps():
    x = momentum((4, 40, 60), FP32, 5).cuda()
    out, again = torch.empty_like(x), torch.empty_like(x)
    space = sdl.alloc_orthogonalize(x, out)
    steps = [(1.5, -0.5, 0.0)] * 40
    sdl.sdl_orthogonalize(x, out, space, steps)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdl.sdl_orthogonalize(x, out, space, steps)
    for replay in range(3):
        x.copy_(momentum((4, 40, 60), FP32, 60 + replay))
        space.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        sdl.sdl_orthogonalize(x, again, torch.empty_like(space), steps)
        assert torch.equal(out, again)
