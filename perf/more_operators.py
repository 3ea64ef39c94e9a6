"""What the operators at the two ends of a decoder, and the update of its matrices, are measured on.

Between two outer steps every replica of the decoder (widths 768 and 2048, 32,000 tokens, see workloads) takes inner steps: tokens are
looked up in a table, the last layer's logits meet the next tokens in a cross entropy (with the z term of the method's paper), the table gets its
gradient, and the matrices of the blocks get an update.  Three operators, each a case's `op`:

  embedding      out[t] = scale * table[tokens[t]], and the table's gradient: scale * the sum of d_out[t] over the places t of a token.
                 A token outside the table (padding, -1) gives a row of zeros and no gradient
  cross_entropy  loss = lse - (1 - smoothing) x[target] - smoothing * mean(x) + z lse^2,  lse = log sum exp(x), and its gradient times the
                 row's weight.  A target outside the vocabulary gives 0 and no gradient
  orthogonalize  X = x / (norm(x) + eps), of a tall matrix the transpose, then for every (a, b, c):  A = X X^T,  X = a X + (b A + c A^2) X

A case's `pass` is what one pass does: "forward", "backward", or "train", both.
`own` chooses between the plain forms below, in elementary torch operations in fp32, and the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TOKENS = {"int32": torch.int32, "int64": torch.int64}
EPS = 1e-7
QUINTIC = (3.4445, -4.7750, 2.0315)     # of the Muon optimizer: lifts small singular values fast, and leaves all of them near 1
STEPS = 5
NUMEL_MOST = 1 << 28                    # drawn cases: logits, and elements of a table, at most
FLOPS_MOST = 7.0e11                     # drawn cases: operations of a matrix case at most


# ------------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the first layer of the 1B shape, one micro-batch of four sequences
        {"name": "embedding_1b", "op": "embedding", "pass": "forward", "batch": 4, "tokens": 2048, "vocab": 32000, "width": 2048, "table": "bf16",
         "dtype": "bf16", "index": "int64", "padding": 0.0, "hot": 0.0},
        # one new token for each of eight requests, 100M shape
        {"name": "embedding_token", "op": "embedding", "pass": "forward", "batch": 8, "tokens": 1, "vocab": 32000, "width": 768, "table": "bf16",
         "dtype": "bf16", "index": "int64", "padding": 0.0, "hot": 0.0},
        # its gradient, of tokens that are as frequent as words are
        {"name": "embedding_back_1b", "op": "embedding", "pass": "backward", "batch": 4, "tokens": 2048, "vocab": 32000, "width": 2048, "table": "bf16",
         "dtype": "bf16", "index": "int64", "padding": 0.0, "hot": 0.0},
        # documents padded to one length in fp32, sizes that are multiples of nothing, a separator that is every third token
        {"name": "embedding_odd_fp32", "op": "embedding", "pass": "backward", "batch": 3, "tokens": 1517, "vocab": 5003, "width": 1021, "table": "fp32",
         "dtype": "fp32", "index": "int32", "padding": 0.2, "hot": 0.33},
        # the loss of a micro-batch of the 1B shape, with its gradient
        {"name": "loss_1b", "op": "cross_entropy", "pass": "train", "batch": 4, "tokens": 2048, "vocab": 32000, "dtype": "bf16", "index": "int64",
         "smoothing": 0.0, "z": 1e-4, "padding": 0.0, "shifted": False},
        # a large vocabulary, smoothed targets, the logits of all but the last token
        {"name": "loss_wide", "op": "cross_entropy", "pass": "train", "batch": 2, "tokens": 511, "vocab": 131072, "dtype": "bf16", "index": "int64",
         "smoothing": 0.1, "z": 0.0, "padding": 0.0, "shifted": True},
        # what answers cost in evaluation: prompts and padding have no loss
        {"name": "loss_evaluation", "op": "cross_entropy", "pass": "forward", "batch": 8, "tokens": 1024, "vocab": 32000, "dtype": "bf16", "index": "int64",
         "smoothing": 0.0, "z": 0.0, "padding": 0.5, "shifted": False},
        # a debugging run in fp32, sizes that are multiples of nothing
        {"name": "loss_odd_fp32", "op": "cross_entropy", "pass": "train", "batch": 3, "tokens": 517, "vocab": 5003, "dtype": "fp32", "index": "int32",
         "smoothing": 0.1, "z": 1e-4, "padding": 0.2, "shifted": False},
        # the four attention matrices of a block, 1B shape
        {"name": "update_block_1b", "op": "orthogonalize", "pass": "forward", "batch": 4, "rows": 2048, "cols": 2048, "dtype": "bf16", "out": "bf16",
         "rank": 128},
        # one matrix of a feed-forward layer of the 1B shape, momentum and update in fp32
        {"name": "update_ffn_1b_fp32", "op": "orthogonalize", "pass": "forward", "batch": 1, "rows": 8192, "cols": 2048, "dtype": "fp32", "out": "fp32",
         "rank": 128},
        # all attention matrices of the 100M shape in one call, momentum in fp32
        {"name": "update_all_100m", "op": "orthogonalize", "pass": "forward", "batch": 48, "rows": 768, "cols": 768, "dtype": "fp32", "out": "bf16",
         "rank": 64},
        # a projection of a small decoder, of an odd width
        {"name": "update_small", "op": "orthogonalize", "pass": "forward", "batch": 1, "rows": 100, "cols": 131, "dtype": "fp32", "out": "fp32", "rank": 8},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["embedding", "embedding", "cross_entropy", "cross_entropy", "orthogonalize", "orthogonalize"])
    kind = lambda: rng.choice(["bf16", "bf16", "fp32"])  # noqa: E731
    index = rng.choice(["int64", "int64", "int32"])
    if op == "embedding":
        vocab, width = _log(rng, 16, 131072), rng.choice([_log(rng, 1, 8192), 64 * _log(rng, 1, 64)])
        width = min(width, NUMEL_MOST // vocab)
        batch = rng.randint(1, 8)
        dtype = kind()
        return {"op": op, "pass": rng.choice(["forward", "backward", "backward"]), "batch": batch, "tokens": _log(rng, 1, min(16384, NUMEL_MOST // (4 * batch * width))),
                "vocab": vocab, "width": width, "table": rng.choice([dtype, "bf16", "fp32"]), "dtype": dtype, "index": index,
                "padding": rng.choice([0.0, 0.0, rng.random() * 0.5]), "hot": rng.choice([0.0, 0.0, rng.random()])}
    if op == "cross_entropy":
        vocab, batch = _log(rng, 2, 200000), rng.randint(1, 8)
        return {"op": op, "pass": rng.choice(["train", "train", "forward", "backward"]), "batch": batch,
                "tokens": _log(rng, 1, max(1, min(4096, NUMEL_MOST // (batch * vocab) - 1))), "vocab": vocab, "dtype": kind(), "index": index,
                "smoothing": rng.choice([0.0, 0.0, 0.1, rng.random() * 0.5]), "z": rng.choice([0.0, 1e-4, 1e-3]),
                "padding": rng.choice([0.0, rng.random() * 0.5]), "shifted": rng.random() < 0.3}
    while True:
        rows, cols = _log(rng, 1, 4096), _log(rng, 1, 8192)
        if rng.random() < 0.5:
            rows, cols = 64 * max(1, rows // 64), 64 * max(1, cols // 64)
        if rng.random() < 0.5:
            rows, cols = cols, rows
        n, m, batch = min(rows, cols), max(rows, cols), _log(rng, 1, 64)
        if 2.0 * batch * STEPS * n * n * (2 * m + n) <= FLOPS_MOST and batch * n * m <= 1 << 26:
            return {"op": op, "pass": "forward", "batch": batch, "rows": rows, "cols": cols, "dtype": kind(), "out": kind(), "rank": rng.randint(1, max(1, n // 8))}


# ----------------------------------------------------------------------------------------------------- inputs

def _randn(shape, gen, std=1.0):
    return torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen) * std


def _words(shape, vocab, index, padding, gen, hot=0.0):
    """Tokens whose frequency falls with their rank, as words' does; `padding` of them are -1, and `hot` of the others one separator."""
    u = torch.rand(shape, device="cuda", generator=gen, dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)
    # ranks are spread over the table
    t = (t * 7919 + 13) % vocab if vocab % 7919 else t
    t = torch.where(torch.rand(shape, device="cuda", generator=gen) < hot, vocab // 3, t)
    return torch.where(torch.rand(shape, device="cuda", generator=gen) < padding, -1, t).to(TOKENS[index])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] == "embedding":
        shape = (case["batch"], case["tokens"])
        state["ids"] = _words(shape, case["vocab"], case["index"], case["padding"], gen, case["hot"])
        state["scale"] = math.sqrt(case["width"])
        if case["pass"] == "forward":
            state["table"] = _randn((case["vocab"], case["width"]), gen, 0.02).to(DTYPES[case["table"]])
        else:
            state["d_out"] = _randn(shape + (case["width"],), gen, 1e-3).to(DTYPES[case["dtype"]])
    elif case["op"] == "cross_entropy":
        shape = (case["batch"], case["tokens"])
        targets = _words(shape, case["vocab"], case["index"], case["padding"], gen)
        x = _randn((case["batch"], case["tokens"] + case["shifted"], case["vocab"]), gen, 2.0)
        # the target is somewhere between unknown and certain
        lift = torch.rand(shape, device="cuda", generator=gen) * 16.0
        x[:, :case["tokens"]].scatter_add_(2, targets.long().clamp(min=0)[..., None], lift[..., None])
        x = x.to(DTYPES[case["dtype"]])
        state["logits"], state["targets"] = x[:, :case["tokens"]], targets
        # the mean over the targets
        state["d_loss"] = torch.full(shape, 1.0, device="cuda") / (targets >= 0).sum().clamp(min=1)
        if case["pass"] == "backward":      # the forward pass has left it
            state["lse"] = torch.where(targets >= 0, torch.logsumexp(state["logits"].double(), -1), 0.0).float()
    else:
        B, R, C, r = case["batch"], case["rows"], case["cols"], case["rank"]
        # a gradient's momentum: a few directions that count, falling off, and noise
        fall = torch.logspace(0, -2, r, device="cuda")
        x = torch.matmul(_randn((B, R, r), gen) * fall, _randn((B, r, C), gen)) * (1.0 / math.sqrt(r)) + _randn((B, R, C), gen, 0.05)
        state["x"] = (x * 1e-3).to(DTYPES[case["dtype"]])
        # an update as large as that of a square matrix' rows
        state["scale"] = math.sqrt(max(1.0, R / C))
    return state


# ------------------------------------------------------------------------------------------------ plain forms

def _embedding(state):
    case, ids = state["case"], state["ids"].long()
    there = (ids >= 0) & (ids < case["vocab"])
    if case["pass"] == "forward":
        rows = state["table"][torch.where(there, ids, 0)].float() * state["scale"]
        return torch.where(there[..., None], rows, 0.0).to(DTYPES[case["dtype"]])
    d_out = state["d_out"].float().reshape(-1, case["width"])
    # rows without a place in the table go into one more row
    total = torch.zeros((case["vocab"] + 1, case["width"]), device="cuda").index_add_(0, torch.where(there, ids, case["vocab"]).reshape(-1), d_out)
    return (total[:-1] * state["scale"]).to(DTYPES[case["table"]])


def _cross_entropy(state):
    case, targets = state["case"], state["targets"].long()
    V, smoothing, z = case["vocab"], case["smoothing"], case["z"]
    there = (targets >= 0) & (targets < V)
    at = torch.where(there, targets, 0)[..., None]
    x = state["logits"].float()
    out = {}
    if case["pass"] == "backward":
        lse = state["lse"]
    else:
        top = x.amax(-1, keepdim=True)
        lse = (top + (x - top).exp().sum(-1, keepdim=True).log())[..., 0]
        loss = lse - (1.0 - smoothing) * x.gather(-1, at)[..., 0] + z * lse * lse
        if smoothing:
            loss = loss - smoothing * x.mean(-1)
        out = {"loss": torch.where(there, loss, 0.0), "lse": torch.where(there, lse, 0.0)}
    if case["pass"] != "forward":
        d = (x - lse[..., None]).exp() * (1.0 + 2.0 * z * lse)[..., None]
        d.scatter_add_(-1, at, torch.full_like(d[..., :1], smoothing - 1.0))
        if smoothing:
            d = d - smoothing / V
        out["d_logits"] = torch.where(there[..., None], d * state["d_loss"][..., None], 0.0).to(state["logits"].dtype)
    return out


def _orthogonalize(state):
    case, x = state["case"], state["x"].float()
    tall = case["rows"] > case["cols"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if tall:
        x = x.transpose(1, 2)
    return (x * state["scale"]).to(DTYPES[case["out"]]).contiguous()


# ------------------------------------------------------------------------------------------- the framework's calls

def _own_embedding(state):
    import paper_2501_18512_amd as sdl
    case, ids = state["case"], state["ids"]
    if case["pass"] == "forward":
        out = torch.empty((*ids.shape, case["width"]), dtype=DTYPES[case["dtype"]], device=ids.device)
        sdl.sdl_embedding(state["table"], ids, out, state["scale"])
        return out
    if "space" not in state:
        state["space"] = sdl.alloc_embedding(ids, case["width"])
    d_table = torch.empty((case["vocab"], case["width"]), dtype=DTYPES[case["table"]], device=ids.device)
    sdl.sdl_embedding_backward(state["d_out"], ids, d_table, state["space"], state["scale"])
    return d_table


def _own_cross_entropy(state):
    import paper_2501_18512_amd as sdl
    case, logits, targets = state["case"], state["logits"], state["targets"]
    how = {"smoothing": case["smoothing"], "z": case["z"]}
    d_logits = None if case["pass"] == "forward" else torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    if case["pass"] == "backward":
        sdl.sdl_cross_entropy_backward(logits, targets, state["lse"], d_logits, state["d_loss"], **how)
        return {"d_logits": d_logits}
    loss, lse = (torch.empty(targets.shape, dtype=torch.float32, device=logits.device) for _ in range(2))
    if case["pass"] == "forward":
        sdl.sdl_cross_entropy(logits, targets, loss, lse, **how)
        return {"loss": loss, "lse": lse}
    sdl.sdl_cross_entropy(logits, targets, loss, lse, d_logits, state["d_loss"], **how)
    return {"loss": loss, "lse": lse, "d_logits": d_logits}


def _own_orthogonalize(state):
    import paper_2501_18512_amd as sdl
    case, x = state["case"], state["x"]
    out = torch.empty(x.shape, dtype=DTYPES[case["out"]], device=x.device)
    if "space" not in state:
        state["space"] = sdl.alloc_orthogonalize(x, out)
    sdl.sdl_orthogonalize(x, out, state["space"], [QUINTIC] * STEPS, EPS, state["scale"])
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"embedding": _own_embedding, "cross_entropy": _own_cross_entropy, "orthogonalize": _own_orthogonalize}[op](state)
    return {"embedding": _embedding, "cross_entropy": _cross_entropy, "orthogonalize": _orthogonalize}[op](state)


# --------------------------------------------------------------------------------------------------- yardsticks

def work(case):
    size = {"bf16": 2, "fp32": 4, "int32": 4, "int64": 8}
    if case["op"] == "embedding":
        n, W = case["batch"] * case["tokens"], case["width"]
        if case["pass"] == "forward":       # about as many rows of the table as there are places; one that comes again is in the caches
            return {"bytes": n * W * (size[case["table"]] + size[case["dtype"]]) + n * size[case["index"]], "flops": n * W}
        return {"bytes": n * W * size[case["dtype"]] + n * size[case["index"]] + case["vocab"] * W * size[case["table"]], "flops": n * W}
    if case["op"] == "cross_entropy":       # rows without a target are not read, and their gradient is written all the same
        n, V = case["batch"] * case["tokens"], case["vocab"]
        read = n * V * size[case["dtype"]] * (1.0 - case["padding"])
        return {"bytes": read + n * (size[case["index"]] + 12) + (0 if case["pass"] == "forward" else n * V * size[case["dtype"]]),
                "flops": n * V * (4 if case["pass"] == "forward" else 8)}
    B, n, m = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # A and A^2 are symmetric: half of each
    return {"bytes": B * n * m * (size[case["dtype"]] + size[case["out"]]), "flops": STEPS * B * (n * (n + 1) * m + n * n * (n + 1) + 2 * n * n * m)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "embedding":
        ids = state["ids"].reshape(-1).long()
        valid = ids.ge(0) & ids.lt(case["vocab"])
        if case["pass"] == "forward":
            out = torch.zeros((ids.numel(), case["width"]), dtype=torch.float64, device="cuda")
            out[valid] = state["table"].double()[ids[valid]] * state["scale"]
            return out.view(case["batch"], case["tokens"], case["width"])
        grad = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
        rows = state["d_out"].double().reshape(-1, case["width"])[valid] * state["scale"]
        return grad.index_put_((ids[valid],), rows, accumulate=True)
    if case["op"] == "cross_entropy":
        V, e = case["vocab"], case["smoothing"]
        x, t = state["logits"].double(), state["targets"].long()
        valid = t.ge(0) & t.lt(V)
        logp = torch.log_softmax(x, -1)
        lse = torch.logsumexp(x, -1)
        hit = torch.zeros(x.shape, dtype=torch.bool, device="cuda").scatter_(-1, t.clamp(0, V - 1)[..., None], True)
        out = {}
        if case["pass"] != "backward":
            loss = -(1.0 - e) * logp.masked_select(hit).view(t.shape) - e * logp.mean(-1) + case["z"] * lse.square()
            out = {"loss": loss.masked_fill(~valid, 0.0), "lse": lse.masked_fill(~valid, 0.0)}
        if case["pass"] != "forward":
            q = hit.double() * (1.0 - e) + e / V
            d = (logp.exp() - q + logp.exp() * (2.0 * case["z"] * lse)[..., None]) * state["d_loss"].double()[..., None]
            out["d_logits"] = d.masked_fill(~valid[..., None], 0.0)
        return out
    # everything that the steps do is a polynomial of the first Gram matrix: its powers, and the product with x at the end
    x = state["x"].double()
    if case["rows"] > case["cols"]:
        x = x.mT.contiguous()
    x = x / (torch.linalg.matrix_norm(x)[:, None, None] + EPS)
    a, b, c = QUINTIC
    one = torch.eye(x.shape[1], dtype=torch.float64, device="cuda").expand(x.shape[0], -1, -1)
    g, q = torch.bmm(x, x.mT.contiguous()), one.clone()
    for _ in range(STEPS):
        p = torch.baddbmm(a * one + b * g, g, g, alpha=c)
        q, g = torch.bmm(p, q), torch.bmm(torch.bmm(p, g), p)
    x = torch.bmm(q, x) * state["scale"]
    return x.mT.contiguous() if case["rows"] > case["cols"] else x
