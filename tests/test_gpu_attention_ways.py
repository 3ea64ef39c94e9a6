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
