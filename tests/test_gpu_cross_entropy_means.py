"""sdl_cross_entropy of rows with numbers next to the largest ones: the mean of smoothed targets, and differences from the maximum, where sums of them are beyond fp32 and the
loss is not."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, close, output, placed, randn
from oracle import training as ref
from test_gpu_cross_entropy import bounds

pytestmark = pytest.mark.gpu
# every launch shape with and without gradients, and rows that are read twice
VOCABS = [2, 5, 40, 512, 700, 1500, 2500, 5003, 9001, 20000, 70001, 140001]


def check(x, t, smoothing, how="dense"):
    rows, dtype = x.shape[:-1], x.dtype
    xg, tg = placed(x, how), t.cuda()
    loss, lse = (torch.full(rows, float("nan"), device="cuda") for _ in range(2))
    d, alone = output(x, how)
    sdl.sdl_cross_entropy(xg, tg, loss, lse, d, None, smoothing)
    torch.cuda.synchronize()
    assert alone()
    want_loss, want_lse = ref.cross_entropy(x, t, smoothing, 0.0)
    e_loss, e_lse, e_d = bounds(x, t, torch.logsumexp(x.double(), -1), torch.ones(rows), smoothing, 0.0)
    close(lse, want_lse, 1.01 * e_lse, "lse")
    # a loss whose bound goes on to infinity may be infinite: that of one row, next to the largest number with smoothing 1
    sure = want_loss.abs() + 1.01 * e_loss < torch.finfo(FP32).max
    assert int((~sure).sum()) <= (smoothing == 1.0)
    close(loss[sure.cuda()], want_loss[sure], 1.01 * e_loss[sure], "loss")
    want = ref.cross_entropy_backward(x, t, None, torch.ones(rows), smoothing, 0.0)
    close(d, want, U[dtype] * want.abs() + 1.01 * e_d, "gradient")
    loss2 = torch.full(rows, float("nan"), device="cuda")
    sdl.sdl_cross_entropy(xg, tg, loss2, None, smoothing=smoothing)
    assert torch.equal(loss, loss2)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", VOCABS)
def test_tokens_masked_with_the_lowest_number(dtype, V):
    """The mean is -10^37 to -3 10^38, and the sum of two such logits is infinite."""
    low = torch.finfo(dtype).min
    gen = torch.Generator().manual_seed(V)
    x, t = randn((6, V), dtype, V, 2.0), torch.arange(6) % V
    for part in (0.01, 0.7):
        masked = torch.rand((6, V), generator=gen) < part
        masked[:, :3] = True
        masked[4] = True
        masked[torch.arange(6), t] = False
        y = torch.where(masked, torch.tensor(low, dtype=dtype), x)
        print(f"cross entropy {V} {dtype} {part}", flush=True)
        for smoothing in (0.1, 1.0):
            check(y, t, smoothing)
        check(y, t, 0.1, "odd")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", VOCABS)
def test_all_of_a_row_next_to_the_largest_number(dtype, V):
    """Sums of all of a row's logits, one by one, of either sign; and a maximum and a mean, or a target, at the two ends of the type."""
    top = torch.finfo(dtype).max
    x = torch.full((5, V), top).to(dtype)
    t = torch.full((5,), V // 2)
    x[1] = -x[1]
    x[2, ::2], t[2] = -top, 1       # a mean near 0: 0.25 top
    x[3] = -top                     # but for the target: 0.25 (top - mean)
    x[3, V // 2] = top
    x[4, V // 2] = -top             # the target: 0.25 (top + top), and little of the mean
    print(f"cross entropy {V} {dtype}", flush=True)
    check(x[:4], t[:4], 0.25)
    if V > 2:
        check(x[[0, 1, 4]], t[[0, 1, 4]], 0.75)
