"""Attention at the edges of its sizes."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, output, placed, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("queries", [0, 3])
def test_gradients_of_keys_that_no_query_head_reads_are_zero(dtype, queries):
    q, k = torch.empty(2, queries, 0, 24), randn((2, 70, 3, 24), dtype, 1)
    qg, kg = q.to(dtype).cuda(), placed(k, "odd")
    dk, dk_alone = output(k, "odd")
    dv, dv_alone = output(k)
    lse = torch.empty(2, 0, queries, device="cuda")
    lens = torch.tensor([70, 11], dtype=torch.int32, device="cuda")
    sdl.sdl_attention(qg, kg, kg, qg, lse, None, causal=True, k_len=lens)
    sdl.sdl_attention_backward(qg, qg, kg, kg, qg, lse, qg, dk, dv, sdl.alloc_attention(qg, kg, backward=True), causal=True, k_len=lens)
    torch.cuda.synchronize()
    assert not dk.any() and not dv.any() and dk_alone() and dv_alone()


def test_as_many_sequences_as_one_row_of_workgroups_cannot_hold():
    """2^24 (sequence, head) of 17 queries and 2^26 of one: a launch of that many workgroups side by side would be 2^32 threads.  One key each: the result is its value."""
    for batch, queries, heads in ((1 << 20, 17, 16), (1 << 26, 1, 1), ((1 << 22) + 5, 1, 1)):
        print(f"attention {batch} {queries} {heads}", flush=True)
        gen = torch.Generator("cuda").manual_seed(batch % 1000)
        v = torch.randn(batch, 1, heads, 1, device="cuda", generator=gen).bfloat16()
        q, k = torch.ones(1, 1, 1, 1, device="cuda", dtype=BF16).expand(batch, queries, heads, 1), v
        out, lse = torch.full((batch, queries, heads, 1), 9.0, device="cuda", dtype=BF16), torch.empty(batch, heads, queries, device="cuda")
        sdl.sdl_attention(q, k, v, out, lse, None, scale=1.0)
        torch.cuda.synchronize()
        assert torch.equal(out, v.expand_as(out))
        # the score is k; the logarithm of a sum of one term, a product and a sum in fp32
        assert float((lse - k.float()[:, :, :, 0].transpose(1, 2)).abs().max()) <= 4 * 2.0 ** -24 * float(k.abs().max())
        del q, k, v, out, lse


def test_gradients_of_as_many_sequences_as_one_row_of_workgroups_cannot_hold():
    batch, heads = 1 << 20, 16
    one = torch.ones(1, 1, 1, 1, device="cuda", dtype=BF16).expand(batch, 1, heads, 1)
    gen = torch.Generator("cuda").manual_seed(3)
    v, do = (torch.randn(batch, 1, heads, 1, device="cuda", generator=gen).bfloat16() for _ in range(2))
    out, lse = torch.empty_like(v), torch.empty(batch, heads, 1, device="cuda")
    sdl.sdl_attention(one, v, v, out, lse, None, scale=1.0)
    dq, dk, dv = (torch.full_like(v, 9.0) for _ in range(3))
    sdl.sdl_attention_backward(do, one, v, v, out, lse, dq, dk, dv, sdl.alloc_attention(one, v, backward=True), scale=1.0)
    torch.cuda.synchronize()
    # one probability, of 1 but for the roundings of lse (|lse| under 8): 1 in bf16; the gradients through it are those roundings times |d_out v| under 64
    assert torch.equal(dv, do)
    assert float(dq.abs().max()) <= 64 * 8 * 8 * 2.0 ** -24 * 8 and float(dk.abs().max()) <= 64 * 8 * 8 * 2.0 ** -24
