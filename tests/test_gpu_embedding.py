"""GPU parity of sdl_embedding and its backward pass with the 64-bit oracle.

Bounds.  Forward: one product in fp32 and a rounding to the result's type.  Backward: a row is a sum of k terms in fp32 and a product, off by at most
(k + 2) u(fp32) times the sum of its terms' absolute values, and rounded to the table's type."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, output, placed, randn
from oracle import training as ref

pytestmark = pytest.mark.gpu
# batch, tokens, vocab, width: one place and many, widths on both sides of what a wavefront takes, two chunks of places and one more, more chunks than are merged at once
SHAPES = [(1, 1, 5, 3), (2, 3, 7, 8), (1, 17, 100, 64), (3, 5, 33, 65), (2, 40, 300, 257), (1, 2048, 50, 33), (1, 2049, 1000, 16), (2, 1500, 777, 100), (3, 700, 64, 520),
          (1, 5000, 3, 1021), (8, 1, 50, 768), (1, 300, 1, 40), (5, 13, 2000, 2048)]


def tokens_of(shape, vocab, how, seed, dtype=torch.int64):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randint(0, vocab, shape, generator=gen)
    if how == "words":
        t = (vocab ** torch.rand(shape, generator=gen)).long() - 1
    elif how == "one":
        t = torch.full(shape, vocab - 1)
    elif how == "none":
        t = torch.full(shape, -1)
    elif how == "padded":           # everything that is not in the table
        out = [-1, vocab, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, 2 ** 40 + 1, -2 ** 63, 2 ** 63 - 1] if dtype == torch.int64 else [])
        which = torch.tensor(out)[torch.randint(0, len(out), shape, generator=gen)]
        t = torch.where(torch.rand(shape, generator=gen) < 0.4, which, t)
    elif how == "sorted":
        t = t.flatten().sort()[0].view(shape)
    return t.to(dtype)


def check(shape, table_dtype, dtype, how="words", index=torch.int64, place="dense", scale=1.0, seed=0):
    B, L, V, W = shape
    t = tokens_of((B, L), V, how, seed, index)
    table = randn((V, W), table_dtype, seed + 1)
    out, alone = output(torch.empty(B, L, W, dtype=dtype), place)
    sdl.sdl_embedding(placed(table, place), t.cuda(), out, scale)
    torch.cuda.synchronize()
    assert alone()
    want = ref.embedding(table, t, scale)
    close(out, want, (U[dtype] + 2 * U32) * want.abs(), "out")
    d_out = randn((B, L, W), dtype, seed + 2)
    d_table, alone = output(torch.empty(V, W, dtype=table_dtype), place)
    d, ids = placed(d_out, place), t.cuda()
    space = sdl.alloc_embedding(ids, W)
    space.fill_(0xab)
    sdl.sdl_embedding_backward(d, ids, d_table, space, scale)
    torch.cuda.synchronize()
    assert alone()
    want, size, count = ref.embedding_backward(d_out, t, V, scale)
    close(d_table, want, U[table_dtype] * want.abs() + 1.01 * (count + 2) * U32 * size, "d_table")
    return d_table, (d, ids, space)


@pytest.mark.parametrize("table,dtype", [(BF16, BF16), (FP32, FP32), (FP32, BF16), (BF16, FP32)])
def test_forward_and_backward(table, dtype):
    for i, shape in enumerate(SHAPES):
        print(f"embedding {shape} {table} {dtype}", flush=True)
        check(shape, table, dtype, "words" if i % 2 else "uniform", torch.int64 if i % 3 else torch.int32, scale=(1.0, 45.25, -0.5)[i % 3], seed=10 * i)


@pytest.mark.parametrize("how", ["one", "none", "padded", "sorted"])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_tokens_of_every_kind(how, index):
    for i, shape in enumerate([(1, 1, 4, 8), (2, 9, 30, 72), (1, 2100, 90, 24), (3, 1000, 17, 600), (1, 16, 8, 8), (1, 17, 8, 8)]):
        print(f"embedding {shape} {how} {index}", flush=True)
        check(shape, FP32, FP32, how, index, seed=100 + 10 * i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_where_they_lie(dtype):
    for i, shape in enumerate([(2, 5, 9, 64), (3, 70, 40, 33), (2, 1100, 12, 300), (1, 4, 100, 1030)]):
        print(f"embedding {shape} {dtype}", flush=True)
        check(shape, dtype, dtype, "padded", place="odd", seed=200 + 10 * i)


@pytest.mark.parametrize("vocab", [(1 << 22) - 2, (1 << 22) - 1, 1 << 22, 5000011])
def test_tables_longer_than_short_keys_name(vocab):
    """Tokens from both ends of the table; all of its rows are looked at."""
    for n, how in ((1500, "padded"), (40, "one")):
        print(f"embedding {n} places of {vocab}", flush=True)
        t = tokens_of((n,), vocab, how, n).to(torch.int64)
        t[::7], t[1::7] = vocab - 1, 0
        t = t.cuda()
        d = (torch.arange(n * 3, device="cuda") % 11).float().view(n, 3)
        got = torch.full((vocab, 3), float("nan"), device="cuda")
        sdl.sdl_embedding_backward(d, t, got, sdl.alloc_embedding(t, 3))
        there = (t >= 0) & (t < vocab)
        want = torch.zeros((vocab, 3), device="cuda").index_add_(0, t[there], d[there])          # whole numbers: exact in any order
        assert torch.equal(got, want)


def test_more_places_than_are_merged_at_once():
    """The sum of a column of ones counts the places of a token, exactly."""
    for n in (65536, 65537, 150000):
        print(f"embedding {n} places", flush=True)
        t = tokens_of((n,), 5000, "words", n).cuda()
        space = sdl.alloc_embedding(t, 8)
        d = torch.zeros((n, 8), device="cuda")
        d[:, 0], d[:, 1] = 1.0, torch.arange(n, device="cuda") % 7
        got = torch.empty((5000, 8), device="cuda")
        sdl.sdl_embedding_backward(d, t, got, space)
        want = torch.zeros((5000, 8), dtype=torch.float64).index_add_(0, t.cpu(), d.cpu().double())
        assert torch.equal(got.cpu().double(), want)


def test_repeatable_on_another_stream_and_in_a_graph():
    got, (d, ids, space) = check((4, 900, 500, 768), BF16, BF16, seed=7)
    again = torch.empty_like(got)
    sdl.sdl_embedding_backward(d, ids, again, space)
    assert torch.equal(got, again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    third = torch.empty_like(got)
    sdl.sdl_embedding_backward(d, ids, third, torch.empty_like(space), stream=side)
    side.synchronize()
    assert torch.equal(got, third)
    graph, table, out = torch.cuda.CUDAGraph(), randn((500, 768), BF16, 3).cuda(), torch.empty_like(d)
    with torch.cuda.graph(graph):
        sdl.sdl_embedding_backward(d, ids, again, space)
        sdl.sdl_embedding(table, ids, out, 2.0)
    for replay in range(4):
        # other tokens and other rows in the same places
        ids.copy_(tokens_of((4, 900), 500, ("words", "one", "padded", "uniform")[replay], replay))
        d.copy_(randn(d.shape, BF16, 40 + replay))
        space.fill_(replay)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        sdl.sdl_embedding_backward(d, ids, third, torch.empty_like(space))
        assert torch.equal(again, third), replay
        sdl.sdl_embedding(table, ids, d, 2.0)
        assert torch.equal(out, d), replay


def test_gradient_is_the_lookups_transpose():
    """sum of d_out * lookup(table) = sum of lookup's gradient * table, whatever the table is."""
    B, L, V, W = 3, 50, 40, 96
    t, table, d = tokens_of((B, L), V, "padded", 1).cuda(), randn((V, W), FP32, 2).cuda(), randn((B, L, W), FP32, 3).cuda()
    out, d_table = torch.empty_like(d), torch.empty_like(table)
    sdl.sdl_embedding(table, t, out, 3.0)
    sdl.sdl_embedding_backward(d, t, d_table, sdl.alloc_embedding(t, W), 3.0)
    a, b = (d.double() * out.double()), (d_table.double() * table.double())
    # at most 50 terms a sum: 52 roundings of the absolute values, and the lookup's own
    assert abs(float(a.sum() - b.sum())) <= 55 * U32 * float(a.abs().sum())


def test_nothing_to_do():
    table, out = torch.ones(5, 16, device="cuda"), torch.empty(0, 16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    sdl.sdl_embedding(table, none, out)
    sdl.sdl_embedding_backward(out, none, table, None)
    assert not table.any()                                  # no token: all rows are zeros
    rows = torch.ones(3, 16, device="cuda")
    sdl.sdl_embedding(torch.empty(0, 16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), rows)
    assert not rows.any()                                   # no table: every token is outside
