"""Inner steps of M replicas of a small decoder with the outer step between them, and what comes out answering token by token.

The replicas are the flat bf16 arrays that the outer step works on; the decoder's parameters are views of them.  One inner step of a
replica: embedding, blocks of [norm, q k v projection, norm of q and k per head, rotary positions, attention, output projection; norm,
feed-forward], final norm, head, cross entropy, backward, Adam.  Norms, rotary positions and attention are this library's calls, the
products torch's.  The engine sends and receives what its schedule says after every step.  Then the mean of the replicas answers a
prompt: once as a whole, and once token by token over a cache of keys and values.

    python examples/inner_steps.py [--steps 60] [--replicas 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_18512_amd as sdl  # noqa: E402

EPS = 1e-5


# ---------------------------------------------------------------- the operators, as torch's autograd sees them

class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) for _ in range(2))
        sdl.sdl_layer_norm(x, weight, None, EPS, y, mean, rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dweight = torch.empty(x.shape, dtype=x.dtype, device=x.device), torch.empty_like(weight)
        workspace = torch.empty(sdl.sdl_layer_norm_workspace_bytes(x.shape[-1]), dtype=torch.uint8, device=x.device)
        sdl.sdl_layer_norm_backward(dy.contiguous(), x, weight, mean, rstd, dx, dweight, None, workspace)
        return dx, dweight


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, frequencies):
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        sdl.sdl_rotary(x, positions, frequencies, out)
        ctx.save_for_backward(positions, frequencies)
        return out

    @staticmethod
    def backward(ctx, dy):
        positions, frequencies = ctx.saved_tensors
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        sdl.sdl_rotary(dy.contiguous(), positions, frequencies, dx, inverse=True)
        return dx, None, None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        sdl.sdl_attention(q, k, v, out, lse, sdl.alloc_attention(q, k), causal=True)
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, out, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        sdl.sdl_attention_backward(d_out.contiguous(), q, k, v, out, lse, dq, dk, dv, sdl.alloc_attention(q, k, backward=True), causal=True)
        return dq, dk, dv


# ------------------------------------------------------------------------------------------------ the decoder

class Shape:
    """Width, blocks, heads, and the parameter groups in the order of the flat array."""

    def __init__(self, vocab=96, width=128, blocks=2, heads=4, kv_heads=2):
        self.vocab, self.width, self.blocks, self.heads, self.kv_heads, self.head = vocab, width, blocks, heads, kv_heads, width // heads
        qkv = (heads + 2 * kv_heads) * self.head
        self.groups = [("embed", (vocab, width), sdl.UNIT_PRE)]
        for b in range(blocks):
            for name, shape in (("norm", (width,)), ("qkv", (qkv, width)), ("q_norm", (self.head,)), ("k_norm", (self.head,)),
                                ("out", (width, width)), ("ffn_norm", (width,)), ("up", (4 * width, width)), ("down", (width, 4 * width))):
                self.groups.append((f"{b}.{name}", shape, b))
        self.groups += [("final_norm", (width,), sdl.UNIT_POST), ("head", (vocab, width), sdl.UNIT_POST)]
        self.numel = [torch.Size(s).numel() for _, s, _ in self.groups]

    def views(self, flat):
        """Parameters by name, as views of a flat array."""
        out, at = {}, 0
        for (name, shape, _), n in zip(self.groups, self.numel):
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out


def decoder(shape, params, tokens, frequencies, positions, cache=None):
    """Logits of tokens [batch, tokens].  cache: (keys, values, lengths) per block; the new tokens are put behind the valid ones."""
    B, L = tokens.shape
    H, G, D = shape.heads, shape.kv_heads, shape.head
    x = params["embed"][tokens]
    for b in range(shape.blocks):
        p = {n: params[f"{b}.{n}"] for n in ("norm", "qkv", "q_norm", "k_norm", "out", "ffn_norm", "up", "down")}
        qkv = (LayerNorm.apply(x, p["norm"]) @ p["qkv"].T).view(B, L, H + 2 * G, D)
        q = Rotary.apply(LayerNorm.apply(qkv[:, :, :H], p["q_norm"]), positions, frequencies)
        k = Rotary.apply(LayerNorm.apply(qkv[:, :, H:H + G], p["k_norm"]), positions, frequencies)
        v = qkv[:, :, H + G:]
        if cache is None:
            a = Attention.apply(q, k, v)
        else:
            keys, values, lengths = cache[b]
            rows = torch.arange(B, device=tokens.device)[:, None]
            keys[rows, positions.long()], values[rows, positions.long()] = k, v
            lengths.copy_(positions[:, -1] + 1)
            a = torch.empty_like(q)
            sdl.sdl_attention(q, keys, values, a, None, sdl.alloc_attention(q, keys), causal=True, k_len=lengths)
        x = x + a.reshape(B, L, -1) @ p["out"].T
        h = LayerNorm.apply(x, p["ffn_norm"]) @ p["up"].T
        x = x + torch.nn.functional.gelu(h) @ p["down"].T
    return LayerNorm.apply(x, params["final_norm"]) @ params["head"].T


class Replica:
    """One worker's inner optimizer over a flat bf16 array (Adam's moments in fp32)."""

    def __init__(self, shape, flat, lr):
        self.shape, self.flat, self.lr, self.t = shape, flat, lr, 0
        self.m, self.v = (torch.zeros(flat.numel(), dtype=torch.float32, device=flat.device) for _ in range(2))

    def step(self, tokens, frequencies, positions):
        flat = self.flat.detach().requires_grad_()
        logits = decoder(self.shape, self.shape.views(flat), tokens[:, :-1], frequencies, positions)
        loss = torch.nn.functional.cross_entropy(logits.float().flatten(0, 1), tokens[:, 1:].flatten())
        grad = torch.autograd.grad(loss, flat)[0].float()
        self.t += 1
        self.m.lerp_(grad, 0.1)
        self.v.lerp_(grad * grad, 0.05)
        step = (self.m / (1 - 0.9 ** self.t)) / ((self.v / (1 - 0.95 ** self.t)).sqrt() + 1e-8)
        with torch.no_grad():
            self.flat.copy_(self.flat.float() - self.lr * step)
        return loss.detach()


def text(shape, batch, length, seed):
    """Sequences with something to learn: every token follows from the one before, by one of a few rules a sequence keeps to."""
    gen = torch.Generator().manual_seed(seed)
    jump = torch.randint(1, 4, (batch, 1), generator=gen)
    return ((torch.randint(0, shape.vocab, (batch, 1), generator=gen) + jump * torch.arange(length)) % shape.vocab).cuda()


def answer(shape, params, prompt, frequencies, new):
    """Greedy tokens behind a prompt, over a cache, and the logits that each was chosen by."""
    B, L = prompt.shape
    cache = [(torch.zeros(B, L + new, shape.kv_heads, shape.head, dtype=torch.bfloat16, device="cuda"),
              torch.zeros(B, L + new, shape.kv_heads, shape.head, dtype=torch.bfloat16, device="cuda"),
              torch.zeros(B, dtype=torch.int32, device="cuda")) for _ in range(shape.blocks)]
    positions = torch.arange(L, dtype=torch.int32, device="cuda").expand(B, L).contiguous()
    logits = [decoder(shape, params, prompt, frequencies, positions, cache)[:, -1]]
    tokens = [prompt]
    for i in range(new):
        tokens.append(logits[-1].argmax(-1, keepdim=True))
        if i + 1 < new:
            at = torch.full((B, 1), L + i, dtype=torch.int32, device="cuda")
            logits.append(decoder(shape, params, tokens[-1], frequencies, at, cache)[:, -1])
    return torch.cat(tokens, 1), torch.stack(logits, 1)


def train(steps=60, replicas=2, batch=16, length=65, H=20, tau=2, lr=3e-3, seed=0, say=print):
    """Returns the losses [steps][replicas], the shape, the mean of the replicas as bf16 and the frequencies."""
    shape = Shape()
    plan = sdl.sdl_fragment_plan(shape.numel, [u for _, _, u in shape.groups], shape.blocks, 2, sdl.PATTERN_STRIDED, H, tau)
    total = plan.total_numel
    g, mom, w, _, pool = sdl.alloc_flat_model(total, replicas, False)
    gen = torch.Generator("cuda").manual_seed(seed)
    g.copy_(torch.randn(total, device="cuda", generator=gen) * 0.05)
    for name, view in shape.views(g).items():
        if name.endswith("norm"):
            view.fill_(1.0)
    mom.zero_()
    for x in w:
        x.copy_(g)
    messages = [sdl.sdl_plan_message_bytes(plan, p, sdl.FMT_E3M0) for p in range(plan.num_fragments)]
    buffers = [[torch.empty(max(m[i], 16), dtype=torch.uint8, device="cuda") for m in messages for _ in range(replicas)] for i in range(2)]
    engine = sdl.sdl_engine_create(plan, H, [tau] * replicas, sdl.FMT_E3M0, 0.7, 0.9, 0.5)
    sdl.sdl_engine_bind(engine, g, mom, w, *buffers)
    workers = [Replica(shape, x, lr) for x in w]
    frequencies = sdl.sdl_rotary_frequencies(shape.head).cuda()
    positions = torch.arange(length - 1, dtype=torch.int32, device="cuda").expand(batch, length - 1).contiguous()
    losses = []
    for t in range(1, steps + 1):
        losses.append([r.step(text(shape, batch, length, seed * 1000003 + t * replicas + m), frequencies, positions) for m, r in enumerate(workers)])
        sent, received = sdl.sdl_engine_step(engine, t)
        if sent or received or t == 1:
            say(f"step {t}: loss " + " ".join(f"{float(x):.3f}" for x in losses[-1]) + f", {sent} fragments sent, {received} received")
    out = torch.empty(total, dtype=torch.bfloat16, device="cuda")
    sdl.sdl_evaluation_params(sdl.EVAL_REPLICA_MEAN, None, w, total, out)
    del pool
    return [[float(x) for x in row] for row in losses], shape, out, frequencies


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--replicas", type=int, default=2)
    a = parser.parse_args()
    _, shape, flat, frequencies = train(a.steps, a.replicas)
    prompt = text(shape, 4, 12, seed=99)
    with torch.no_grad():
        tokens, _ = answer(shape, shape.views(flat), prompt, frequencies, 8)
    for row in tokens.tolist():
        print("prompt", row[:12], "answer", row[12:])


if __name__ == "__main__":
    main()
