"""GPU parity of sdl_cross_entropy and its backward pass with the 64-bit oracle.

Bounds, in u = u(fp32), M the row's maximum.  exp(x - M) is taken as a power of two of (x - M) log2(e): the difference, the constant and the product are off by u each, so the
result by (3 |x - M| + 2) u, relatively; on the way from a thread's maximum to the row's come at most 12 joins of 3 u each, and at most 130 additions: s is off by
E = (3 sum p (M - x) + 170) u.  log s: E + 2 u |log s|; lse: a rounding more.  An element's p: E + (3 (M - x) + 10) u."""
import math

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, output, placed, randn
from oracle import training as ref

pytestmark = pytest.mark.gpu
# on both sides of every launch shape's limits (which are seven elements lower for rows that start anywhere), and odd ones
VOCABS = [1, 2, 3, 8, 9, 63, 65, 511, 512, 513, 1018, 1024, 1025, 2042, 2047, 2048, 2049, 4090, 4096, 4097, 5003, 8186, 8192, 8193, 16378, 16384, 16385, 32000, 32762, 32768,
          32769, 65530, 65536, 65537, 131066, 131072, 131073, 200001]


def targets_of(shape, vocab, seed, index=torch.int64, padding=0.25):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randint(0, vocab, shape, generator=gen)
    out = torch.tensor([-1, vocab, -100] + ([2 ** 32, -2 ** 63] if index == torch.int64 else [2 ** 31 - 1]))
    which = out[torch.randint(0, len(out), shape, generator=gen)]
    return torch.where(torch.rand(shape, generator=gen) < padding, which, t).to(index)


def bounds(x, targets, lse, d_loss, smoothing, z):
    """Of loss, lse and the gradient before its last rounding."""
    X, V = x.double(), x.shape[-1]
    M = X.amax(-1)
    p = torch.softmax(X, -1)
    below = torch.where(p > 0, M[..., None] - X, torch.zeros(()).double())
    E = (3 * (p * below).sum(-1) + 170) * U32
    log_s = torch.logsumexp(X - M[..., None], -1).abs()
    e_lse = E + 2 * U32 * log_s + U32 * lse.double().abs()
    hit = (M - X.gather(-1, targets.long().clamp(0, V - 1)[..., None])[..., 0]).abs()
    e_loss = E + 4 * U32 * (log_s + hit) + z * (2 * lse.abs() * e_lse + 4 * U32 * lse.double() ** 2)
    if smoothing:
        e_loss = e_loss + smoothing * (170 * U32 * X.abs().mean(-1) + 4 * U32 * (M.abs() + X.mean(-1).abs()))
    g = d_loss.double().abs()[..., None]
    factor = (1 + 2 * z * lse.double()).abs()[..., None]
    e_d = g * (factor * p * (E[..., None] + (3 * below + 10) * U32) + 2 * z * e_lse[..., None] * p + 4 * U32 * (smoothing / V + p * factor))
    e_d.scatter_add_(-1, targets.long().clamp(0, V - 1)[..., None], 4 * U32 * g)
    return e_loss, e_lse, e_d


def check(x, targets, smoothing, z, how="dense", weighted=True, seed=0):
    dtype, rows = x.dtype, x.shape[:-1]
    d_loss = randn(rows, FP32, seed + 5).abs() + 0.1 if weighted else None
    one = torch.ones(rows) if d_loss is None else d_loss
    xg, tg, dg = placed(x, how), targets.cuda(), None if d_loss is None else d_loss.cuda()
    loss, lse = (torch.full(rows, float("nan"), device="cuda") for _ in range(2))
    d, alone = output(x, how)
    sdl.sdl_cross_entropy(xg, tg, loss, lse, d, dg, smoothing, z)
    torch.cuda.synchronize()
    assert alone()
    want_loss, want_lse = ref.cross_entropy(x, targets, smoothing, z)
    there = (targets >= 0) & (targets < x.shape[-1])
    full_lse = torch.logsumexp(x.double(), -1)
    e_loss, e_lse, e_d = bounds(x, targets, full_lse, one, smoothing, z)
    close(lse, want_lse, 1.01 * e_lse * there, "lse")
    close(loss, want_loss, 1.01 * e_loss * there, "loss")
    want = ref.cross_entropy_backward(x, targets, None, one, smoothing, z)
    close(d, want, U[dtype] * want.abs() + 1.01 * e_d * there[..., None], "gradient")
    # the passes by themselves: the forward one to the bit, the backward one from the lse that it is given
    loss2, lse2 = torch.empty_like(loss), torch.empty_like(lse)
    sdl.sdl_cross_entropy(xg, tg, loss2, None, smoothing=smoothing, z=z)
    sdl.sdl_cross_entropy(xg, tg, None, lse2, smoothing=smoothing, z=z)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    d2, alone = output(x, how)
    sdl.sdl_cross_entropy_backward(xg, tg, lse, d2, dg, smoothing, z)
    torch.cuda.synchronize()
    assert alone()
    given = torch.where(there, lse.cpu().double(), full_lse)
    want2 = ref.cross_entropy_backward(x, targets, given, one, smoothing, z)
    # x - lse is at most M - x and log V
    far = (3 * math.log(x.shape[-1]) + 4) * U32 * one.double().abs()[..., None] * torch.exp(x.double() - given[..., None]) * (1 + 2 * z * given.abs())[..., None]
    close(d2, want2, U[dtype] * want2.abs() + 1.01 * (e_d + far) * there[..., None], "gradient from lse")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_every_launch_shape(dtype):
    for i, V in enumerate(VOCABS):
        rows = (2, 3) if V > 3000 else (3, 11)
        print(f"cross entropy {rows} {V} {dtype}", flush=True)
        x = randn((*rows, V), dtype, 10 * i, 3.0)
        check(x, targets_of(rows, V, i, torch.int64 if i % 2 else torch.int32), (0.0, 0.1, 0.0, 1.0)[i % 4], (0.0, 1e-4, 1e-2)[i % 3], weighted=i % 2 == 0, seed=i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [7, 130, 2049, 5003, 33333])
def test_rows_where_they_lie(dtype, V):
    check(randn((2, 5, V), dtype, V, 2.0), targets_of((2, 5), V, 1), 0.1, 1e-3, "odd")
    # all but the last token of every sequence
    x = randn((3, 4, V), dtype, V + 1, 2.0)
    loss, d = torch.empty(3, 3, device="cuda"), torch.empty(3, 3, V, dtype=dtype, device="cuda")
    t = targets_of((3, 3), V, 2)
    sdl.sdl_cross_entropy(x.cuda()[:, :-1], t.cuda(), loss, None, d)
    alone, d2 = torch.empty(3, 3, device="cuda"), torch.empty_like(d)
    sdl.sdl_cross_entropy(x[:, :-1].contiguous().cuda(), t.cuda(), alone, None, d2)
    assert torch.equal(loss, alone) and torch.equal(d, d2)


def test_certain_targets_keep_their_digits():
    """Losses of 1e-6 beside logits of 30."""
    V = 4000
    x = randn((6, V), FP32, 1)
    t = torch.arange(6)
    x[t, t] = torch.tensor([30.0, 25.0, 22.0, 60.0, 1000.0, 10.0])
    check(x, t, 0.0, 0.0)


def test_large_logits_and_long_ways_to_the_maximum():
    x = randn((4, 3000), FP32, 2) * torch.tensor([1.0, 30.0, 1e4, 1e30])[:, None]
    check(x, targets_of((4,), 3000, 3, padding=0.0), 0.0, 0.0)
    check(randn((4, 3000), BF16, 2, 100.0), targets_of((4,), 3000, 4, padding=0.0), 0.0, 1e-4)


@pytest.mark.parametrize("V", [5, 700, 5003, 70001, 140001])
def test_maxima_of_every_size(V):
    """Rows around numbers that are large, with neighbours of the maximum that count, and far negative ones; in the logits' place too."""
    base = torch.tensor([0.0, 1e5, 2.0 ** 20 - 1, 2.0 ** 20 + 1, 2.0 ** 21 + 8, -2.0 ** 21 - 8, 1e7, -1e6, -3e6, 3e38, -3.3e38, 3.4028234e38, -3.4028234e38])
    t = torch.arange(len(base)) * 7 % V
    x = randn((len(base), V), FP32, V, 2.0)
    x = (x.double() + base.double()[:, None]).float().clamp(-3.4028234e38, 3.4028234e38)
    x[::2, V // 3] = -3.4028234e38                          # masked by the lowest number
    x[torch.arange(len(base)), t] = base                    # not at the target
    check(x, t, 0.0, 0.0)
    check(x[:9], t[:9], 0.1, 0.0)
    g = torch.ones(len(base), device="cuda")
    loss, d, place = torch.empty(len(base), device="cuda"), torch.empty_like(x, device="cuda"), x.cuda()
    sdl.sdl_cross_entropy(x.cuda(), t.cuda(), loss, None, d, g)
    sdl.sdl_cross_entropy(place, t.cuda(), loss, None, place, g)
    assert torch.equal(d, place)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [40, 2500, 70000, 140000])
def test_masked_logits(dtype, V):
    """Tokens that cannot come, as -infinity or as the type's lowest number."""
    x = randn((5, V), dtype, V, 2.0)
    gen = torch.Generator().manual_seed(V)
    masked = torch.rand((5, V), generator=gen) < 0.7
    t = torch.arange(5) * 3
    masked[torch.arange(5), t] = False
    masked[3] = True
    masked[3, t[3]] = False                                  # one token is left
    for low in (-math.inf, torch.finfo(dtype).min):
        y = torch.where(masked, torch.tensor(low, dtype=dtype), x)
        loss, lse = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
        d = torch.empty((5, V), dtype=dtype, device="cuda")
        sdl.sdl_cross_entropy(y.cuda(), t.cuda(), loss, lse, d, None, 0.0, 1e-4)
        want_loss, want_lse = ref.cross_entropy(torch.where(masked, torch.tensor(-1e30), x.float()), t, 0.0, 1e-4)
        e_loss, e_lse, e_d = bounds(torch.where(masked, torch.tensor(-1e30), x.float()), t, want_lse, torch.ones(5), 0.0, 1e-4)
        close(lse, want_lse, 1.01 * e_lse, "lse")
        close(loss, want_loss, 1.01 * e_loss, "loss")
        assert not d.cpu()[masked].any()
        want = ref.cross_entropy_backward(torch.where(masked, torch.tensor(-1e30), x.float()), t, want_lse, torch.ones(5), 0.0, 1e-4)
        close(d, want, U[dtype] * want.abs() + 1.01 * e_d, "gradient")


@pytest.mark.parametrize("V", [20, 600, 5000, 40000, 140000])
def test_what_is_not_finite_stays_in_its_row(V):
    x = randn((8, V), BF16, 5)
    t = torch.tensor([1, 2, -1, 3, 4, 5, V, 6])
    x[1, V // 2], x[3, 0] = math.nan, math.inf
    x[2] = math.nan                                          # no target: not looked at
    x[6, 3] = math.inf
    x[4] = -math.inf                                         # nothing can come
    x[5, 5] = -math.inf                                      # the target cannot come
    loss, lse = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    d = torch.empty((8, V), dtype=BF16, device="cuda")
    sdl.sdl_cross_entropy(x.cuda(), t.cuda(), loss, lse, d)
    for got in (d, d.clone()):
        bad = torch.isnan(got.float()).all(1).tolist()
        assert bad == [False, True, False, True, True, False, False, False]
        assert not torch.isnan(got.float()).any(1)[[0, 2, 5, 6, 7]].any() and not got[[2, 6]].any()
        sdl.sdl_cross_entropy_backward(x.cuda(), t.cuda(), lse, got)
    assert torch.isnan(loss).tolist() == [False, True, False, True, True, False, False, False]
    assert loss[2] == 0 and loss[6] == 0 and lse[2] == 0 and lse[6] == 0 and loss[5] == math.inf and lse[4] == -math.inf
    for smoothing in (0.1, 1.0):                             # a mean of logits with one that cannot come
        sdl.sdl_cross_entropy(x.cuda(), t.cuda(), loss, lse, smoothing=smoothing)
        assert loss[5] == math.inf and loss[2] == 0 and torch.isfinite(loss[[0, 7]]).all() and torch.isfinite(lse[5])


@pytest.mark.parametrize("V", [3, 100, 1001, 3000, 3003, 32000, 32001, 50257, 100000, 150000, 150001])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_in_place_repeatable_on_another_stream_and_in_a_graph(V, dtype):
    rows = 700 if V < 10000 else 30
    x, t = randn((rows, V), dtype, 1, 2.0).cuda(), targets_of((rows,), V, 2).cuda()
    loss, d, g = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.rand(rows, device="cuda")
    sdl.sdl_cross_entropy(x, t, loss, None, d, g, 0.1, 1e-4)
    place, loss2 = x.clone(), torch.empty_like(loss)
    sdl.sdl_cross_entropy(place, t, loss2, None, place, g, 0.1, 1e-4)
    assert torch.equal(loss, loss2) and torch.equal(d, place)
    lse, d2 = torch.empty_like(loss), torch.empty_like(d)
    sdl.sdl_cross_entropy(x, t, None, lse)
    sdl.sdl_cross_entropy_backward(x, t, lse, d2, g, 0.1, 1e-4)
    place.copy_(x)
    sdl.sdl_cross_entropy_backward(place, t, lse, place, g, 0.1, 1e-4)
    assert torch.equal(d2, place)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sdl.sdl_cross_entropy(x, t, loss2, None, d2, g, 0.1, 1e-4, stream=side)
    side.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(d, d2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdl.sdl_cross_entropy(x, t, loss2, lse, d2, g, 0.1, 1e-4)
        sdl.sdl_cross_entropy_backward(x, t, lse, place, g, 0.1, 1e-4)
    for replay in range(3):
        x.copy_(randn((rows, V), dtype, 10 + replay, 2.0))
        t.copy_(targets_of((rows,), V, 20 + replay))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b, c, e = torch.empty_like(loss), torch.empty_like(loss), torch.empty_like(d), torch.empty_like(d)
        sdl.sdl_cross_entropy(x, t, a, b, c, g, 0.1, 1e-4)
        sdl.sdl_cross_entropy_backward(x, t, b, e, g, 0.1, 1e-4)
        assert torch.equal(a, loss2) and torch.equal(b, lse) and torch.equal(c, d2) and torch.equal(e, place)


def test_gradient_against_differences():
    x, t, g = randn((5, 60), FP32, 1), torch.tensor([3, 59, -1, 0, 60]), torch.rand(5, generator=torch.Generator().manual_seed(1))
    d = torch.empty(5, 60, device="cuda")
    sdl.sdl_cross_entropy(x.cuda(), t.cuda(), None, None, d, g.cuda(), 0.2, 0.01)
    loss = lambda y: float((ref.cross_entropy(y, t, 0.2, 0.01)[0] * g.double()).sum())  # noqa: E731
    for seed in range(3):
        way = randn((5, 60), torch.float64, seed)
        slope = (loss(x.double() + 1e-5 * way) - loss(x.double() - 1e-5 * way)) / 2e-5
        # central differences are good to 1e-9 here, the fp32 gradient to 1e-5 of the sum of absolute values
        assert abs(slope - float((d.cpu().double() * way).sum())) < 1e-5 * float((d.cpu().double() * way).abs().sum())


def test_more_rows_than_workgroups_and_none():
    x, t = randn((70000, 5), FP32, 1), targets_of((70000,), 5, 1)
    check(x, t, 0.0, 0.0)
    none = torch.empty(0, 5, device="cuda")
    sdl.sdl_cross_entropy(none, torch.empty(0, dtype=torch.int64, device="cuda"), None, None, none)
