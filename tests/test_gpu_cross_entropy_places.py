"""sdl_cross_entropy with logits and gradients at different alignments and distances: what is grouped by where the gradient lies."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, close, output, placed, randn
from oracle import training as ref
from test_gpu_cross_entropy import bounds, targets_of

pytestmark = pytest.mark.gpu
# on both sides of where one of the two alignments takes the next launch shape, and short rows
VOCABS = [5, 513, 1017, 1020, 1024, 2045, 2048, 4092, 4096, 8189, 8192, 16380, 16384, 32700, 32768, 65535, 65536, 131068, 131072, 140001]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", VOCABS)
def test_logits_and_gradient_lie_apart(V, dtype):
    rows = (2, 3)
    for i, (where, to) in enumerate([("dense", "odd"), ("odd", "dense"), ("shifted", "dense"), ("dense", "shifted"), ("shifted", "odd")]):
        print(f"cross entropy {V} {dtype} {where} {to}", flush=True)
        x, t = randn((*rows, V), dtype, 10 * i, 3.0), targets_of(rows, V, i)
        smoothing, z = (0.0, 0.1, 1.0)[i % 3], (0.0, 1e-3)[i % 2]
        xg = of(x, where)
        if to == "shifted":
            d = of(torch.full(x.shape, float("nan"), dtype=dtype), "shifted")
            alone = lambda: bool(torch.isnan(d._base[:, :, V:].float()).all()) and bool(torch.isnan(d._base[:, -1:].float()).all())  # noqa: E731
        else:
            d, alone = output(x, to)
        weights = randn(rows, FP32, i).abs() + 0.1
        loss, lse, loss_alone, lse_alone = (torch.full(rows, float("nan"), device="cuda") for _ in range(4))
        sdl.sdl_cross_entropy(xg, t.cuda(), loss, lse, d, weights.cuda(), smoothing, z)
        sdl.sdl_cross_entropy(xg, t.cuda(), loss_alone, lse_alone, smoothing=smoothing, z=z)
        torch.cuda.synchronize()
        assert alone()
        there = (t >= 0) & (t < V)
        want_loss, want_lse = ref.cross_entropy(x, t, smoothing, z)
        e_loss, e_lse, e_d = bounds(x, t, torch.logsumexp(x.double(), -1), weights, smoothing, z)
        for got, got_lse in ((loss, lse), (loss_alone, lse_alone)):
            close(got_lse, want_lse, 1.01 * e_lse * there, "lse")
            close(got, want_loss, 1.01 * e_loss * there, "loss")
        want = ref.cross_entropy_backward(x, t, None, weights, smoothing, z)
        close(d, want, U[dtype] * want.abs() + 1.01 * e_d * there[..., None], "gradient")
        # the pass by itself, to the other place
        again = torch.full(x.shape, float("nan"), dtype=dtype, device="cuda")
        sdl.sdl_cross_entropy_backward(xg, t.cuda(), lse, again, weights.cuda(), smoothing, z)
        given = torch.where(there, lse.cpu().double(), want_lse)
        # from an lse that is rounded: off by its last half step once more, in exp(x - lse) and in the z term
        off = weights.double()[..., None] * torch.exp(x.double() - given[..., None]) * (1 + 2 * z * given.abs())[..., None]
        want = ref.cross_entropy_backward(x, t, given, weights, smoothing, z)
        close(again, want, U[dtype] * want.abs() + 1.01 * (e_d + (3 * 13.0 + 4) * 2.0 ** -24 * off) * there[..., None], "gradient from lse")


def of(x, where):
    """placed(), or rows that are 16 bytes from a cache line's start with the next sequence's further off ("shifted")."""
    if where != "shifted":
        return placed(x, where)
    step = 16 // x.element_size()
    big = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + step), float("nan"), dtype=x.dtype, device="cuda")
    view = big[:, :-1, :x.shape[2]]
    view.copy_(x)
    return view
