"""The example that trains replicas of a small decoder with the operators and the engine, and lets the result answer token by token."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def test_replicas_learn_and_the_cache_answers_as_the_whole_prompt_does():
    import inner_steps as ex
    losses, shape, flat, frequencies = ex.train(steps=60, say=lambda *_: None)
    first, last = sum(losses[0]) / 2, sum(sum(row) for row in losses[-5:]) / 10
    assert 4.0 < first < 6.0                    # ln 96 = 4.6: nothing is known
    assert last < 0.6 * first                   # the rule of three jumps leaves ln 3 = 1.1 at most
    params, prompt = shape.views(flat), ex.text(shape, 3, 12, seed=7)
    with torch.no_grad():
        tokens, logits = ex.answer(shape, params, prompt, frequencies, 6)
        L = tokens.shape[1] - 1
        positions = torch.arange(L, dtype=torch.int32, device="cuda").expand(3, L).contiguous()
        whole = ex.decoder(shape, params, tokens[:, :-1], frequencies, positions)[:, -6:]
    # bf16 activations of two blocks: the products of one token and of many may round differently, by a few units of 2^-8
    assert float((whole.float() - logits.float()).abs().max()) < 16 * 2.0 ** -8 * float(whole.float().abs().max())


def test_gradients_of_the_decoder_against_torch():
    """One loss, its gradient by the operators and by torch's own functions in fp32, from the same bf16 parameters."""
    import inner_steps as ex
    shape = ex.Shape()
    gen = torch.Generator("cuda").manual_seed(1)
    flat = torch.randn(sum(shape.numel), device="cuda", generator=gen) * 0.05
    for name, view in shape.views(flat).items():
        if name.endswith("norm"):
            view.add_(1.0)
    flat = flat.bfloat16()
    tokens = ex.text(shape, 4, 33, seed=3)
    f = ex.sdl.sdl_rotary_frequencies(shape.head).cuda()
    positions = torch.arange(32, dtype=torch.int32, device="cuda").expand(4, 32).contiguous()
    mine = flat.clone().requires_grad_()
    loss = torch.nn.functional.cross_entropy(ex.decoder(shape, shape.views(mine), tokens[:, :-1], f, positions).float().flatten(0, 1), tokens[:, 1:].flatten())
    grad = torch.autograd.grad(loss, mine)[0].float()

    def plain(shape, p, tokens):
        B, L = tokens.shape
        H, G, D = shape.heads, shape.kv_heads, shape.head
        norm = lambda x, w: torch.nn.functional.layer_norm(x, x.shape[-1:], eps=ex.EPS) * w  # noqa: E731
        angle = positions.double()[:, :, None, None] * f
        cos, sin = angle.cos().float(), angle.sin().float()

        def turn(x):
            a, b = x.chunk(2, -1)
            return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        x = p["embed"][tokens]
        for b in range(shape.blocks):
            q, k, v = (norm(x, p[f"{b}.norm"]) @ p[f"{b}.qkv"].T).view(B, L, H + 2 * G, D).split([H, G, G], 2)
            q, k = turn(norm(q, p[f"{b}.q_norm"])), turn(norm(k, p[f"{b}.k_norm"]))
            k, v = k.repeat_interleave(H // G, 2), v.repeat_interleave(H // G, 2)
            s = (q.transpose(1, 2) @ k.permute(0, 2, 3, 1).contiguous()) * D ** -0.5
            s = s.masked_fill(torch.ones(L, L, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
            a = (s.softmax(-1) @ v.transpose(1, 2).contiguous()).transpose(1, 2).reshape(B, L, -1)
            x = x + a @ p[f"{b}.out"].T
            x = x + torch.nn.functional.gelu(norm(x, p[f"{b}.ffn_norm"]) @ p[f"{b}.up"].T) @ p[f"{b}.down"].T
        return norm(x, p["final_norm"]) @ p["head"].T
    ref = flat.float().requires_grad_()
    want_loss = torch.nn.functional.cross_entropy(plain(shape, shape.views(ref), tokens[:, :-1]).flatten(0, 1), tokens[:, 1:].flatten())
    want = torch.autograd.grad(want_loss, ref)[0]
    # about forty bf16 roundings of 2^-9 on average (rms 2^-9 / sqrt 3 each) on the way there and back: sqrt(40) 2^-9 / sqrt 3 = 0.7 %; twice that and a half
    assert abs(float(loss) - float(want_loss)) < 0.02 * float(want_loss)
    for name, got in shape.views(grad).items():
        w = shape.views(want)[name]
        assert float((got - w).norm()) < 0.025 * float(w.norm()), name
