"""The operators at the decoder's two ends and the update of its matrices together, in the example's inner step."""
import os
import sys

import pytest
import torch

from oracle import training as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def setting(seed):
    import inner_steps as ex
    shape = ex.Shape()
    gen = torch.Generator("cuda").manual_seed(seed)
    flat = torch.randn(sum(shape.numel), device="cuda", generator=gen) * 0.05
    for name, view in shape.views(flat).items():
        if name.endswith("norm"):
            view.add_(1.0)
    f = ex.sdl.sdl_rotary_frequencies(shape.head).cuda()
    positions = torch.arange(32, dtype=torch.int32, device="cuda").expand(4, 32).contiguous()
    return ex, shape, flat.bfloat16(), ex.text(shape, 4, 33, seed=3), f, positions


def test_loss_and_gradients_with_the_z_term_against_torch():
    """The decoder's loss and gradient by the library's embedding and cross entropy, and by torch's lookup and fp32 arithmetic around the same blocks."""
    ex, shape, flat, tokens, f, positions = setting(1)
    loss, grad = ex.Replica(shape, flat, 1e-3).gradient(tokens, f, positions)
    lookup = ex.Embedding.apply
    mine = flat.clone().requires_grad_()
    try:
        ex.Embedding.apply = lambda table, t: table[t]
        logits = ex.decoder(shape, shape.views(mine), tokens[:, :-1], f, positions).float()
    finally:
        ex.Embedding.apply = lookup
    lse = torch.logsumexp(logits, -1)
    want_loss = (lse - logits.gather(-1, tokens[:, 1:, None])[..., 0] + ex.Z * lse * lse).mean()
    want = torch.autograd.grad(want_loss, mine)[0].float()
    # the same blocks in the same arithmetic: what differs is the order of sums in fp32, and roundings of d_logits and of the table's gradient that fall the other way, 2^-9 on average
    # each; a few of them on the way back
    assert abs(float(loss.detach()) - float(want_loss.detach())) < 1e-4 * float(want_loss.detach())
    for name, got in shape.views(grad).items():
        w = shape.views(want)[name]
        assert float((got - w).norm()) < 8 * 2.0 ** -9 * float(w.norm()), name


def test_an_orthogonal_step_of_the_flat_array():
    """One step: the blocks' matrices move by the orthogonalised momentum, by the oracle's singular values, and nothing else than without it."""
    ex, shape, flat, tokens, f, positions = setting(2)
    steps = {}
    for update in ("adam", "orthogonal"):
        replica = ex.Replica(shape, flat.clone(), 1e-2, update)
        replica.step(tokens, f, positions)
        steps[update] = (replica.flat.clone(), replica.m.clone())
    assert torch.equal(steps["adam"][1], steps["orthogonal"][1])
    before = shape.views(flat)
    for (name, a), o, m in zip(shape.views(steps["adam"][0]).items(), shape.views(steps["orthogonal"][0]).values(), shape.views(steps["adam"][1]).values()):
        if not (name[0].isdigit() and a.dim() == 2):
            assert torch.equal(a, o), name
            continue
        step = ref.orthogonalize(m.cpu(), ex.sdl.ORTHOGONALIZE_QUINTIC, 1e-7, 0.2 * max(m.shape) ** 0.5)
        want = before[name].cpu().double() - 1e-2 * step
        # the parameters are bf16: half a step of theirs, on a step that is good to 1e-5
        off = (o.cpu().double() - want).abs()
        assert bool((off <= 2.0 ** -8 * want.abs() + 1e-4 * step.abs().max()).all()), name


def test_replicas_run_with_orthogonal_updates():
    """Forty steps of two replicas with the engine between them: everything stays finite, and the replicas move."""
    import inner_steps as ex
    losses, shape, flat, _ = ex.train(steps=40, say=lambda *_: None, update="orthogonal")
    assert all(x == x and x < 100 for row in losses for x in row)
    assert bool(torch.isfinite(flat.float()).all()) and len(losses) == 40


def test_two_captured_graphs_share_a_workspace():
    """Lookup, loss, both gradients and an update in two graphs of other sizes over one workspace, replayed in turn."""
    import paper_2501_18512_amd as sdl
    gen = torch.Generator("cuda").manual_seed(5)

    def part(places, vocab, width, rows):
        t = dict(tokens=torch.randint(-1, vocab, (places,), device="cuda", generator=gen), table=torch.randn(vocab, width, device="cuda", generator=gen).bfloat16(),
                 m=torch.randn(2, rows, width, device="cuda", generator=gen))
        t.update(x=torch.empty(places, width, dtype=torch.bfloat16, device="cuda"), logits=torch.randn(places, vocab, device="cuda", generator=gen).bfloat16(),
                 loss=torch.empty(places, device="cuda"), d_table=torch.empty_like(t["table"]), step=torch.empty_like(t["m"]))
        t["d"] = torch.empty_like(t["logits"])
        return t

    def run(t, space):
        sdl.sdl_embedding(t["table"], t["tokens"], t["x"])
        sdl.sdl_cross_entropy(t["logits"], t["tokens"], t["loss"], None, t["d"], z=1e-4)
        sdl.sdl_embedding_backward(t["x"], t["tokens"], t["d_table"], space)
        sdl.sdl_orthogonalize(t["m"], t["step"], space)

    parts = [part(2500, 300, 260, 200), part(70, 5000, 512, 700)]
    space = torch.empty(max(max(sdl.alloc_embedding(t["tokens"], t["x"].shape[1]).numel(), sdl.alloc_orthogonalize(t["m"], t["step"]).numel()) for t in parts),
                        dtype=torch.uint8, device="cuda")
    graphs = []
    for t in parts:
        run(t, space)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(t, space)
    for replay in range(3):
        for t, graph in zip(parts, graphs):
            t["tokens"].copy_(torch.randint(-1, t["table"].shape[0], t["tokens"].shape, device="cuda", generator=gen))
            t["m"].normal_(generator=gen)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for t in parts:
            want = {k: torch.empty_like(v) if k in ("x", "loss", "d", "d_table", "step") else v for k, v in t.items()}
            run(want, torch.empty_like(space))
            for name in ("x", "loss", "d", "d_table", "step"):
                assert torch.equal(t[name], want[name]), (replay, name)
