"""sdl_embedding and its backward pass where their teams, merges and accesses end: rows that are one more than a team's, wide rows, places of three and four merges."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, randn
from oracle import training as ref
from test_gpu_embedding import check, tokens_of

pytestmark = pytest.mark.gpu


def inside(rows, width, dtype, more=5):
    """rows of NaN with as many more behind the last one, and what says whether those are untouched."""
    big = torch.full((rows + more, width), float("nan"), dtype=dtype, device="cuda")
    return big[:rows], lambda: bool(torch.isnan(big[rows:].float()).all())


@pytest.mark.parametrize("table,dtype", [(BF16, BF16), (FP32, FP32), (FP32, BF16)])
@pytest.mark.parametrize("n,width", [(2047, 300), (2049, 300), (2049, 257), (4095, 2048), (4097, 2048), (4099, 2049), (2051, 1021), (9, 64), (33, 63), (31, 65), (7, 256), (13, 5)])
def test_a_place_more_than_a_team_has(n, width, table, dtype):
    print(f"embedding {n} of {width} {table} {dtype}", flush=True)
    V = 60
    weights, t = randn((V, width), table, 1), tokens_of((n,), V, "padded", 2)
    out, untouched = inside(n, width, dtype)
    sdl.sdl_embedding(weights.cuda(), t.cuda(), out, 3.0)
    torch.cuda.synchronize()
    assert untouched()
    want = ref.embedding(weights, t, 3.0)
    close(out, want, (U[dtype] + 2 * U32) * want.abs(), "out")
    d, (d_table, untouched) = randn((n, width), dtype, 3), inside(V, width, table)
    sdl.sdl_embedding_backward(d.cuda(), t.cuda(), d_table, sdl.alloc_embedding(t.cuda(), width), 3.0)
    torch.cuda.synchronize()
    assert untouched()
    want, size, count = ref.embedding_backward(d, t, V, 3.0)
    close(d_table, want, U[table] * want.abs() + 1.01 * (count + 2) * U32 * size, "d_table")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("width", [2049, 2500, 4097, 8191, 16388, 65535, 65536])
def test_wide_rows(width, dtype):
    for i, (shape, place) in enumerate([((1, 3, 5, width), "dense"), ((2, 9, 7, width), "odd")]):
        print(f"embedding {shape} {dtype} {place}", flush=True)
        check(shape, dtype, dtype, "padded" if i else "uniform", place=place, scale=0.5, seed=i)


@pytest.mark.parametrize("n,width", [(1 << 20, 1), ((1 << 20) + 1, 3), (1100003, 8), ((1 << 25) + 5, 1)])
@pytest.mark.parametrize("how", ["words", "uniform", "one"])
def test_places_of_more_than_two_merges(n, width, how):
    """Whole numbers, exact in any order: a place that is lost, or comes twice, is seen."""
    V = 5000
    print(f"embedding {n} places of {width}", flush=True)
    t = tokens_of((n,), V, how, 5, torch.int32).cuda()
    # sums stay under 2^24
    d = (torch.arange(n * width, device="cuda") * 7 % 11 == 0).float().view(n, width)
    got = torch.full((V, width), float("nan"), device="cuda")
    space = sdl.alloc_embedding(t, width)
    space.fill_(0xab)
    sdl.sdl_embedding_backward(d, t, got, space)
    torch.cuda.synchronize()
    print("summed", flush=True)
    want = torch.zeros((V, width), dtype=torch.float64).index_add_(0, t.cpu(), d.double().cpu())       # (one row's atomics on the device take minutes)
    assert float(want.max()) < 2 ** 24
    assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,width", [(9, 5), (700, 64), (2500, 300), (40000, 40)])
def test_what_is_not_finite_in_padded_places_goes_nowhere(n, width, dtype):
    """d_out of padding is not looked at; elsewhere it stays in its token's row and column."""
    V = 70
    t, d = tokens_of((n,), V, "padded", 6), randn((n, width), dtype, 7)
    clean = d.clone()
    there = (t >= 0) & (t < V)
    d[~there] = float("nan")
    d[~there, :2] = float("inf")
    at = int(there.nonzero()[0])
    d[at, 3] = float("nan")
    got, want = (torch.full((V, width), -1.0, dtype=dtype, device="cuda") for _ in range(2))
    sdl.sdl_embedding_backward(d.cuda(), t.cuda(), got, sdl.alloc_embedding(t.cuda(), width))
    sdl.sdl_embedding_backward(clean.cuda(), t.cuda(), want, sdl.alloc_embedding(t.cuda(), width))
    assert torch.isnan(got[t[at], 3])
    got[t[at], 3] = want[t[at], 3]
    assert torch.equal(got, want)
