"""Attention that goes one way against the same problem going another: chunks of keys against one pass, D of short rows against the stored result's, a stream of
its own against the current one."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, placed
from oracle import innerstep as ref
from test_gpu_attention import _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("queries,lens", [(3, None), (3, [3000, 1203]), (20, [3000, 7])])
def test_chunks_of_keys_against_one_pass(dtype, queries, lens):
    """The same sequences alone, in chunks, and among 512 copies of themselves, which are not cut: both within the bound, so at most two bounds apart."""
    B, Lk, H, G, D, copies = 2, 3000, 4, 2, 64, 512
    t = sdl.DTYPE_BF16 if dtype == BF16 else sdl.DTYPE_FP32
    assert sdl.sdl_attention_workspace_bytes(B, queries, Lk, H, G, D, t) > 0 and sdl.sdl_attention_workspace_bytes(B * copies, queries, Lk, H, G, D, t) == 0
    q, k, v, _ = _inputs((B, queries, Lk, H, G, D), dtype, 31)
    got = []
    for n in (1, copies):
        many = lambda x: x.cuda()[None].expand(n, *x.shape)  # noqa: E731
        qg = many(q).reshape(n * B, *q.shape[1:])
        # two sequences side by side, every copy the same memory: one call a sequence
        outs, lses = [], []
        for b in range(B):
            kg, vg = (x[b:b + 1].cuda().expand(n * B, *x.shape[1:]) for x in (k, v))
            kl = None if lens is None else torch.full((n * B,), lens[b], dtype=torch.int32, device="cuda")
            out, lse = torch.empty_like(qg), torch.empty(n * B, H, queries, device="cuda")
            sdl.sdl_attention(qg, kg, vg, out, lse, sdl.alloc_attention(qg, kg), causal=True, k_len=kl)
            torch.cuda.synchronize()
            outs.append(out[b])
            lses.append(lse[b])
        got.append((torch.stack(outs), torch.stack(lses)))
    w = ref.attention(q, k, v, D ** -0.5, True, None, None if lens is None else torch.tensor(lens))
    some = w["lse"][torch.isfinite(w["lse"])]
    d = 2 * U32 * ((D + 4) * w["score_abs"] + 8 * (1 + float(some.abs().max())) + 8 + Lk)
    e = U[dtype] * w["out"].abs() + 1.01 * ((U[dtype] if dtype == BF16 else 0.0) + d) * w["out_abs"]
    for out, lse in got:
        close(out, w["out"], e, "out")
    close(got[0][0], got[1][0].cpu().double(), 2 * e, "chunks and one pass")
    close(got[0][1], got[1][1].cpu().double(), 2 * (d + U32 * w["lse"].abs().nan_to_num(0, 0, 0)), "lse of chunks and one pass")


@pytest.mark.parametrize("case", [(2, 5, 5, 2, 2, 64, False, None, None), (2, 100, 100, 4, 2, 128, True, None, None), (1, 128, 128, 2, 1, 40, True, [111], [120]),
                                  (3, 60, 64, 2, 1, 96, True, None, [64, 1, 0]), (2, 128, 128, 3, 3, 30, False, None, None)])
def test_short_rows_take_the_sum_of_p_dp_and_not_the_rounded_result(case):
    """Values with a large part in common: d_out out and d_out v agree in it, and the rounding of the stored result would be many times larger than what is left.

    As in the module that the other bounds are from, with D's error from its own sum: P |dP| off by d each and by u a term, and dP's products."""
    B, Lq, Lk, H, G, D = case[:6]
    q, k, v, do = _inputs(case, BF16, 41)
    v = (v.float() + 128.0).bfloat16()
    lens = [None if n is None else torch.tensor(n, dtype=torch.int32) for n in case[7:9]]
    qg, kg, vg, dg = (placed(t) for t in (q, k, v, do))
    out, lse = torch.empty_like(qg), torch.empty(B, H, Lq, device="cuda")
    mask = dict(causal=case[6], q_len=None if lens[0] is None else lens[0].cuda(), k_len=None if lens[1] is None else lens[1].cuda())
    space = sdl.alloc_attention(qg, kg, backward=True)
    sdl.sdl_attention(qg, kg, vg, out, lse, space, **mask)
    dq, dk, dv = (torch.empty_like(t) for t in (qg, kg, vg))
    sdl.sdl_attention_backward(dg, qg, kg, vg, out, lse, dq, dk, dv, space, **mask)
    torch.cuda.synchronize()
    s, r = D ** -0.5, U[BF16]
    w = ref.attention(q, k, v, s, case[6], *lens, d_out=do)
    some = w["lse"][torch.isfinite(w["lse"])]
    d = 2 * U32 * ((D + 4) * w["score_abs"] + 8 * (1 + float(some.abs().max())) + 8 + Lk)
    e_q, e_k, a_q, a_k = (torch.zeros(t.shape, dtype=torch.float64) for t in (q, k, q, k))
    for b, h, g, nq, nk, p in w["p"]:
        qq, kk, vv, dd = (t.double() for t in (q[b, :nq, h], k[b, :nk, g], v[b, :nk, g], do[b, :nq, h]))
        dp, size = dd @ vv.T, dd.abs() @ vv.abs().T
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        e_d = (p * ((d + Lk * U32) * dp.abs() + (D + 4) * U32 * size)).sum(1, keepdim=True)
        # dk and dv start a sum from -D, of D's size: a rounding of |D| for every 16 products of it
        e = 1.01 * (d * ds.abs() + p * ((D + 4) * U32 * (size + (p * dp).sum(1, keepdim=True).abs()) + e_d)) + r * ds.abs()
        e_q[b, :nq, h] = s * (e @ kk.abs())
        a_q[b, :nq, h] = s * (ds.abs() @ kk.abs())
        e_k[b, :nk, g] += s * (e.T @ qq.abs())
        a_k[b, :nk, g] += s * (ds.abs().T @ qq.abs())
    close(dq, w["dq"], r * w["dq"].abs() + 1.01 * (e_q + U32 * (Lk + 2) * a_q), "dq")
    close(dk, w["dk"], r * w["dk"].abs() + 1.01 * (e_k + U32 * (Lq * (H // G) + 2) * a_k), "dk")


def test_calls_on_another_stream_that_waits_for_their_arrays():
    case = (2, 150, 150, 4, 2, 64, True, None, None)
    q, k, v, do = (t.cuda() for t in _inputs(case, BF16, 5))
    res = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        out, dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, q, k, v))
        lse, space = torch.full((2, 4, 150), float("nan"), device="cuda"), sdl.alloc_attention(q, k, backward=True)
        stream.wait_stream(torch.cuda.current_stream())         # everything the calls read and write is there
        sdl.sdl_attention(q, k, v, out, lse, space, causal=True, stream=stream)
        sdl.sdl_attention_backward(do, q, k, v, out, lse, dq, dk, dv, space, causal=True, stream=stream)
        torch.cuda.synchronize()
        res.append((out, lse, dq, dk, dv))
    assert all(torch.equal(a, b) for a, b in zip(*res)) and not any(torch.isnan(t.float()).any() for t in res[0])
