"""GPU parity of sdl_attention and its backward pass with the 64-bit oracle.

Bounds, with u = u(fp32) and r the rounding of probabilities and of their gradients as operands (u(type)):
  P     is off by d P, d = 2 u ((D + 4) max |S| + 8 (1 + |lse|) + 8 + keys): scores are sums of D products, lse is rounded to fp32, sums run over the keys
  out   (r + d) P |v|, and the type's rounding
  dv    (r + d) P^T |d_out| + u rows P^T |d_out|
  dS    P (d |dP - D| + (D + 4) u |d_out||v| + (D + 4) u |d_out||out| + |d_out| out's error) + r |dS|, summed with |k| and |q| for dq and dk"""
import math

import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, output, placed, randn
from oracle import innerstep as ref

pytestmark = pytest.mark.gpu

# batch, queries, keys, heads, kv_heads, width, causal, valid queries, valid keys
CASES = [
    (1, 1, 1, 1, 1, 1, False, None, None),
    (1, 1, 1, 1, 1, 64, True, None, None),
    (2, 3, 3, 2, 1, 8, True, None, None),
    (1, 1, 77, 4, 2, 64, True, None, None),
    (2, 1, 300, 8, 1, 128, True, None, [300, 1]),
    (1, 32, 32, 1, 1, 32, False, None, None),
    (1, 33, 65, 2, 2, 64, True, None, None),
    (1, 64, 31, 2, 1, 64, True, None, None),                       # more queries than keys: the first see nothing
    (2, 127, 127, 3, 1, 96, True, None, None),
    (1, 129, 129, 2, 2, 128, True, None, None),
    (1, 200, 200, 1, 1, 128, False, None, None),
    (3, 70, 70, 2, 2, 80, True, [70, 0, 33], [70, 0, 33]),           # an empty sequence, one that ends inside a tile
    (3, 70, 90, 6, 2, 33, False, [1, 70, 64], [90, 0, 63]),          # valid queries over no keys
    (2, 50, 60, 4, 4, 72, True, [50, 20], [10, 60]),                 # fewer valid keys than queries, and more
    (1, 260, 260, 2, 1, 40, True, [257], [257]),
    (1, 5, 700, 6, 2, 128, True, None, [699]),
    (1, 17, 1100, 3, 3, 64, True, None, None),
    (2, 2, 1500, 4, 1, 127, False, None, [1400, 3]),
    (1, 300, 513, 1, 1, 64, True, None, None),
    (2, 130, 131, 5, 5, 16, True, [140, -3], [1000, 131]),           # lengths out of range
]


def _inputs(case, dtype, seed=0, std=1.0):
    B, Lq, Lk, H, G, D = case[:6]
    q, do = randn((B, Lq, H, D), dtype, seed, std), randn((B, Lq, H, D), dtype, seed + 1)
    k, v = randn((B, Lk, G, D), dtype, seed + 2, std), randn((B, Lk, G, D), dtype, seed + 3)
    return q, k, v, do


def _lengths(case):
    return [None if n is None else torch.tensor(n, dtype=torch.int32) for n in case[7:9]]


def _run(case, q, k, v, do, how="dense", scale=None, poison=True, stream=None):
    """out, lse, dq, dk, dv of the library; what lies behind a length is NaN."""
    causal, (q_len, k_len) = case[6], _lengths(case)
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    if poison:
        q, k, v, do = (t.clone() for t in (q, k, v, do))
        for n, ts in ((q_len, (q, do)), (k_len, (k, v))):
            for b in range(len(q) if n is not None else 0):
                for t in ts:
                    t[b, max(0, int(n[b])):] = float("nan")
    qg, kg, vg, dg = (placed(t, how) for t in (q, k, v, do))
    ql, kl = cuda(q_len), cuda(k_len)
    out, out_alone = output(q, how)
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), device="cuda")
    space = sdl.alloc_attention(qg, kg, backward=True)
    mask = dict(scale=scale, causal=causal, q_len=ql, k_len=kl, stream=stream)
    sdl.sdl_attention(qg, kg, vg, out, lse, space, **mask)
    grads = [output(t, how) for t in (q, k, v)]
    sdl.sdl_attention_backward(dg, qg, kg, vg, out, lse, *[g for g, _ in grads], space, **mask)
    torch.cuda.synchronize()
    assert out_alone() and all(alone() for _, alone in grads)
    return out, lse, *[g for g, _ in grads]


def _check(case, dtype, how="dense", seed=0, std=1.0, scale=None):
    B, Lq, Lk, H, G, D = case[:6]
    q, k, v, do = _inputs(case, dtype, seed, std)
    out, lse, dq, dk, dv = _run(case, q, k, v, do, how, scale)
    s = D ** -0.5 if scale is None else scale
    w = ref.attention(q, k, v, s, case[6], *_lengths(case), d_out=do)
    some = w["lse"][torch.isfinite(w["lse"])]
    top = float(some.abs().max()) if some.numel() else 0.0
    d = 2 * U32 * ((D + 4) * w["score_abs"] + 8 * (1 + top) + 8 + Lk)
    r, name = U[dtype], f"attention {case} {dtype} {how}"
    r_in = r if dtype == BF16 else 0.0
    close(lse, w["lse"], d + U32 * w["lse"].abs().nan_to_num(0, 0, 0), name + " lse")
    e_out = r * w["out"].abs() + 1.01 * (r_in + d) * w["out_abs"]
    close(out, w["out"], e_out, name + " out")
    close(dv, w["dv"], r * w["dv"].abs() + 1.01 * (r_in + d + U32 * Lq * (H // G)) * w["dv_abs"], name + " dv")
    e_q, e_k, a_q, a_k = (torch.zeros(t.shape, dtype=torch.float64) for t in (q, k, q, k))
    for b, h, g, nq, nk, p in w["p"]:
        qq, kk, vv, dd = (t.double() for t in (q[b, :nq, h], k[b, :nk, g], v[b, :nk, g], do[b, :nq, h]))
        oo, eo = w["out"][b, :nq, h], e_out[b, :nq, h]
        ds = p * (dd @ vv.T - (dd * oo).sum(1, keepdim=True))
        e = d * ds.abs() + p * ((D + 4) * U32 * (dd.abs() @ vv.abs().T + (dd * oo).abs().sum(1, keepdim=True)) + (dd.abs() * eo).sum(1, keepdim=True))
        e = 1.01 * e + r_in * ds.abs()
        e_q[b, :nq, h] = s * (e @ kk.abs())
        a_q[b, :nq, h] = s * (ds.abs() @ kk.abs())
        e_k[b, :nk, g] += s * (e.T @ qq.abs())
        a_k[b, :nk, g] += s * (ds.abs().T @ qq.abs())
    close(dq, w["dq"], r * w["dq"].abs() + 1.01 * (e_q + U32 * (Lk + 2) * a_q), name + " dq")
    close(dk, w["dk"], r * w["dk"].abs() + 1.01 * (e_k + U32 * (Lq * (H // G) + 2) * a_k), name + " dk")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_forward_and_backward(dtype):
    for i, case in enumerate(CASES):
        print(f"attention {case} {dtype}", flush=True)
        _check(case, dtype, seed=10 * i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("how", ["odd", "packed", "heads"])
def test_arrays_where_they_lie(dtype, how):
    for i in (0, 2, 3, 7, 8, 9, 11, 12, 15, 17):
        print(f"attention {CASES[i]} {dtype} {how}", flush=True)
        _check(CASES[i], dtype, how, seed=300 + 10 * i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scores_far_apart_and_other_scales(dtype):
    case = (1, 90, 150, 2, 1, 64, True, None, None)
    _check(case, dtype, seed=1, std=4.0)                   # scores up to a hundred and more: most probabilities are 0
    _check(case, dtype, seed=2, scale=1e-3)                 # all alike
    _check(case, dtype, seed=3, scale=1.7)


def test_maximum_that_grows_with_every_tile():
    B, L, D = 1, 400, 64
    q = torch.ones(B, L, 1, D)
    k = (torch.arange(L).float() / 16)[None, :, None, None].expand(B, L, 1, D).contiguous() / D
    v, do = randn((B, L, 1, D), FP32, 1), randn((B, L, 1, D), FP32, 2)
    case = (B, L, L, 1, 1, D, False, None, None)
    out, lse = _run(case, q, k, v, do, scale=1.0)[:2]
    w = ref.attention(q, k, v, 1.0)
    d = 2 * U32 * (70 * 25 + 8 * 30 + 8 + L)
    close(out, w["out"], d * w["out_abs"] + U32 * w["out"].abs(), "out")
    close(lse, w["lse"], d, "lse")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_split_keys_give_what_one_pass_gives(dtype):
    """Few rows over many keys go through several workgroups; the same rows among many others do not."""
    B, Lk, H, G, D = 2, 3000, 4, 2, 64
    case = (B, 3, Lk, H, G, D, True, None, [3000, 1203])
    assert sdl.sdl_attention_workspace_bytes(B, 3, Lk, H, G, D, sdl.DTYPE_BF16 if dtype == BF16 else sdl.DTYPE_FP32) > 0
    _check(case, dtype, seed=9)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_few_rows_over_caches_of_different_lengths(dtype):
    """The tiles of many keys' caches are shared out evenly among the workgroups; those of fewer keys, and of more than 256 sequences times key heads, go another way."""
    for i, (B, Lq, Lk, H, G, D, causal, lens) in enumerate([
            (7, 1, 6300, 6, 3, 128, True, [0, 1, 128, 129, 6300, 31, 4700]), (40, 1, 2000, 4, 2, 32, True, [(7 * b * b) % 2001 for b in range(40)]),
            (70, 1, 700, 3, 3, 16, True, [(11 * b) % 701 for b in range(70)]), (128, 2, 600, 2, 2, 24, True, [(37 * b) % 601 for b in range(128)]),
            (1, 3, 140000, 2, 1, 16, True, [139999]), (3, 5, 50000, 3, 1, 8, False, [50000, 2, 0]), (2, 1, 66000, 16, 1, 64, True, [0, 0]),
            (130, 1, 600, 2, 2, 24, True, [(13 * b) % 601 for b in range(130)]), (3, 2, 900, 8, 2, 64, True, [900, 2, 0])]):
        print(f"few rows {B} {Lq} {Lk} {H} {G} {D} {dtype}", flush=True)
        _check((B, Lq, Lk, H, G, D, causal, None, lens), dtype, seed=400 + 10 * i)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_many_heads_at_once(dtype):
    """As many (sequence, key head) as fill the chip with workgroups of 256 rows."""
    _check((8, 200, 300, 32, 32, 128, False, None, [300, 0, 1, 127, 128, 129, 256, 290]), dtype, seed=13)
    _check((16, 70, 190, 32, 32, 104, True, [70, 0, 1, 33, 70, 64, 31, 32] * 2, [190, 100, 0, 20, 128, 129, 31, 190] * 2), dtype, seed=14)
    _check((16, 20, 140, 96, 32, 90, True, None, None), dtype, seed=15)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_heads_of_a_group_go_to_several_workgroups(dtype):
    """Many query heads over few blocks of keys: the gradients of keys and values are sums over workgroups that have some of the heads each."""
    _check((2, 300, 300, 64, 16, 72, True, [300, 170], [300, 170]), dtype, seed=11)
    _check((1, 40, 290, 96, 32, 24, False, None, None), dtype, seed=12)


def test_calls_repeat_bit_for_bit_also_on_another_stream_and_in_a_graph():
    case = (2, 150, 150, 4, 2, 64, True, [150, 99], [150, 99])
    q, k, v, do = _inputs(case, BF16, 5)
    first = _run(case, q, k, v, do)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for again in (_run(case, q, k, v, do), _run(case, q, k, v, do, stream=side)):
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    # one token over a cache, captured: the lengths are read on the device, so that a replay sees new ones
    q, k, v, _ = (t.cuda() for t in _inputs((2, 1, 2000, 4, 2, 64), BF16, 6))
    lens = torch.tensor([2000, 5], dtype=torch.int32, device="cuda")
    out, want, space = torch.empty_like(q), torch.empty_like(q), sdl.alloc_attention(q, k)
    sdl.sdl_attention(q, k, v, out, None, space, causal=True, k_len=lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdl.sdl_attention(q, k, v, out, None, space, causal=True, k_len=lens)
    for n in (1, 700, 1999, 256):
        lens.copy_(torch.tensor([n, 2000 - n], dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        sdl.sdl_attention(q, k, v, want, None, space, causal=True, k_len=lens)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_one_key_head_for_all_by_a_stride_of_zero():
    q, k, v, _ = (t.cuda() for t in _inputs((1, 40, 50, 4, 1, 32), BF16, 8))
    kb, vb = (t.expand(1, 50, 4, 32) for t in (k, v))
    out, want = torch.empty_like(q), torch.empty_like(q)
    sdl.sdl_attention(q, kb, vb, out, None, sdl.alloc_attention(q, kb))
    sdl.sdl_attention(q, k, v, want, None, sdl.alloc_attention(q, k))
    # the rows meet other tiles in the other layout, and the sums another order: two roundings to bf16
    torch.cuda.synchronize()
    assert float((out.float() - want.float()).abs().max()) <= 2 * U[BF16] * float(v.abs().max()) * 1.1


def test_offsets_past_32_bits():
    """Keys 2^21 elements apart: the last ones lie more than 2^32 bytes behind the first."""
    n, far, D = 1100, 1 << 21, 64
    big = torch.empty((n - 1) * far + 2 * D, dtype=BF16, device="cuda")
    k, v = (big.as_strided((1, n, 1, D), (0, far, D, 1), at) for at in (0, D))
    q, kk, vv, do = _inputs((1, 3, n, 1, 1, D), BF16, 3)
    k.copy_(kk)
    v.copy_(vv)
    dk = torch.empty((n - 1) * far + 2 * D, dtype=BF16, device="cuda")
    dkk, dvv = (dk.as_strided((1, n, 1, D), (0, far, D, 1), at) for at in (0, D))
    res = []
    for kx, vx, a, b in ((k, v, dkk, dvv), (kk.cuda(), vv.cuda(), torch.empty_like(kk.cuda()), torch.empty_like(vv.cuda()))):
        qg, out, lse, dq = q.cuda(), torch.empty_like(q.cuda()), torch.empty(1, 1, 3, device="cuda"), torch.empty_like(q.cuda())
        space = sdl.alloc_attention(qg, kx, backward=True)
        sdl.sdl_attention(qg, kx, vx, out, lse, space, causal=True)
        sdl.sdl_attention_backward(do.cuda(), qg, kx, vx, out, lse, dq, a, b, space, causal=True)
        res.append((out, lse, dq, a, b))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*res))


def test_without_keys_or_queries():
    q, k, v, do = _inputs((2, 3, 0, 2, 1, 16), FP32)
    out, lse, dq, dk, dv = _run((2, 3, 0, 2, 1, 16, True, None, None), q, k, v, do)
    assert not out.any() and bool((lse == -math.inf).all()) and not dq.any() and dk.numel() == 0
    q, k, v, do = _inputs((2, 0, 5, 2, 1, 16), FP32)
    out, lse, dq, dk, dv = _run((2, 0, 5, 2, 1, 16, True, None, None), q, k, v, do)
    assert out.numel() == 0 and not dk.any() and not dv.any()


def test_gradient_against_differences():
    case = (1, 20, 24, 2, 1, 24, True, None, None)
    q, k, v, do = _inputs(case, FP32, 4)
    grads = _run(case, q, k, v, do)[2:]
    loss = lambda *t: float((ref.attention(*t, 24 ** -0.5, True)["out"] * do.double()).sum())  # noqa: E731
    args = [t.double() for t in (q, k, v)]
    for i, grad in enumerate(grads):
        way = randn(args[i].shape, torch.float64, 30 + i)
        there, back = (loss(*[t + s * 1e-5 * way if j == i else t for j, t in enumerate(args)]) for s in (1, -1))
        mine = grad.cpu().double() * way
        assert abs((there - back) / 2e-5 - float(mine.sum())) < 1e-5 * float(mine.abs().sum())
