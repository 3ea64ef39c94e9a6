"""What the operators of a decoder's inner step and evaluation are measured on.

The outer step synchronises replicas of a decoder (widths 768 and 2048, sequences of 1,024 and 2,048 tokens, see workloads); between two
of them every replica is trained, and what came out is evaluated on prompts and token by token.  Three operators of that
decoder, each a case's `op`:

  norm       layer norm of rows of `width` elements, [batch, tokens, heads, width]
  rotary     rotary positions of [batch, tokens, heads, width]: the first `rot` elements of every head are rotated
  attention  softmax(scale q k^T + mask) v of [batch, tokens, heads, width], keys and values with `kv_heads` heads

A case's `pass` is what one pass does: "train" is the forward and the backward pass, "forward" and "backward" are one of the two.
`own` chooses between the plain forms below, in elementary torch operations in fp32, and the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5
COST_MOST = 2.0e12        # drawn cases: operations of a pass at most (an fp32 one counts as 16 bf16 ones)
NUMEL_MOST = 1 << 26      # drawn cases of the operators that only stream: elements at most


# ------------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the norm before each half of a block of the 1B shape, one micro-batch of four sequences
        {"name": "norm_block_1b", "op": "norm", "pass": "train", "batch": 4, "tokens": 2048, "heads": 1, "width": 2048, "dtype": "bf16",
         "params": "bf16", "bias": False, "packed": False},
        # the norm of queries per head, where they lie in a fused projection's output; 100M shape
        {"name": "norm_heads_100m", "op": "norm", "pass": "train", "batch": 8, "tokens": 1024, "heads": 12, "width": 64, "dtype": "bf16",
         "params": "bf16", "bias": True, "packed": True},
        # a debugging run in fp32 with a width and a number of rows that are multiples of nothing
        {"name": "norm_odd_fp32", "op": "norm", "pass": "train", "batch": 3, "tokens": 517, "heads": 1, "width": 1021, "dtype": "fp32",
         "params": "fp32", "bias": True, "packed": False},
        # one new token for each of eight requests
        {"name": "norm_token", "op": "norm", "pass": "forward", "batch": 8, "tokens": 1, "heads": 1, "width": 768, "dtype": "bf16",
         "params": "bf16", "bias": True, "packed": False},
        # queries and keys of a fused projection, 1B shape, one micro-batch
        {"name": "rotary_1b", "op": "rotary", "pass": "forward", "batch": 4, "tokens": 2048, "heads": 32, "width": 128, "dtype": "bf16",
         "rot": 128, "layout": "half", "scaling": "none", "first": 0, "packed": True},
        # the gradient through neighbouring pairs in a quarter of an odd number of heads, fp32
        {"name": "rotary_part_back", "op": "rotary", "pass": "backward", "batch": 3, "tokens": 517, "heads": 7, "width": 80, "dtype": "fp32",
         "rot": 20, "layout": "interleaved", "scaling": "linear", "first": 0, "packed": False},
        # new tokens far into a long context
        {"name": "rotary_token_long", "op": "rotary", "pass": "forward", "batch": 16, "tokens": 1, "heads": 20, "width": 128, "dtype": "bf16",
         "rot": 128, "layout": "half", "scaling": "parts", "first": 120000, "packed": False},
        # a training micro-batch of the 1B shape
        {"name": "attention_train_1b", "op": "attention", "pass": "train", "batch": 4, "queries": 2048, "keys": 2048, "heads": 16, "kv_heads": 16,
         "width": 128, "dtype": "bf16", "causal": True, "shortest": 2048, "packed": True, "cache": "tokens"},
        # the 100M shape
        {"name": "attention_train_100m", "op": "attention", "pass": "train", "batch": 8, "queries": 1024, "keys": 1024, "heads": 12, "kv_heads": 12,
         "width": 64, "dtype": "bf16", "causal": True, "shortest": 1024, "packed": True, "cache": "tokens"},
        # documents of different lengths padded to one, shared heads, fp32
        {"name": "attention_ragged_fp32", "op": "attention", "pass": "train", "batch": 4, "queries": 517, "keys": 517, "heads": 6, "kv_heads": 2,
         "width": 80, "dtype": "fp32", "causal": True, "shortest": 1, "packed": False, "cache": "tokens"},
        # a long prompt, forward only
        {"name": "attention_prompt", "op": "attention", "pass": "forward", "batch": 1, "queries": 8192, "keys": 8192, "heads": 16, "kv_heads": 4,
         "width": 128, "dtype": "bf16", "causal": True, "shortest": 8192, "packed": False, "cache": "tokens"},
        # one new token for each of 16 requests of different lengths, over their caches
        {"name": "attention_token", "op": "attention", "pass": "forward", "batch": 16, "queries": 1, "keys": 8192, "heads": 16, "kv_heads": 4,
         "width": 128, "dtype": "bf16", "causal": True, "shortest": 1, "packed": False, "cache": "heads"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "rotary", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "norm":
        heads = rng.choice([1, 1, _log(rng, 2, 32)])
        width = _log(rng, 4, 8192) if heads == 1 else rng.choice([32, 64, 80, 128, 200])
        batch = rng.randint(1, 8)
        most = max(1, min(4096, NUMEL_MOST // (batch * heads * width)))
        return {"op": op, "pass": rng.choice(["train", "train", "forward"]), "batch": batch, "tokens": _log(rng, 1, most), "heads": heads,
                "width": width, "dtype": dtype, "params": rng.choice([dtype, "bf16", "fp32"]), "bias": rng.random() < 0.5,
                "packed": rng.random() < 0.3}
    if op == "rotary":
        batch, heads, width = rng.randint(1, 16), _log(rng, 1, 48), rng.choice([32, 64, 80, 96, 128, 128, 256, 2 * rng.randint(1, 128) + 1])
        most = max(1, min(4096, NUMEL_MOST // (batch * heads * width)))
        return {"op": op, "pass": rng.choice(["forward", "backward"]), "batch": batch, "tokens": _log(rng, 1, most), "heads": heads, "width": width,
                "dtype": dtype, "rot": rng.choice([width // 2 * 2, width // 2 * 2, max(2, width // 4 * 2)]), "layout": rng.choice(["half", "interleaved"]),
                "scaling": rng.choice(["none", "linear", "parts"]), "first": rng.choice([0, _log(rng, 1, 500000)]), "packed": rng.random() < 0.5}
    while True:
        kv_heads = _log(rng, 1, 16)
        c = {"op": op, "pass": rng.choice(["train", "train", "forward"]), "batch": _log(rng, 1, 16), "queries": _log(rng, 1, 8192), "keys": 0,
             "heads": kv_heads * rng.choice([1, 1, 2, 3, 4, 8]), "kv_heads": kv_heads, "width": rng.choice([32, 64, 64, 80, 96, 128, 128, 128, rng.randint(1, 128)]),
             "dtype": dtype, "causal": rng.random() < 0.8, "shortest": 0, "packed": False, "cache": rng.choice(["tokens", "heads"])}
        if c["pass"] == "train":
            # a lone key's probability is 1 whatever the scores are, and the gradients through it are 0
            c["queries"] = max(c["queries"], 8)
            c["keys"], c["packed"] = c["queries"], rng.random() < 0.5
        else:
            c["queries"] = rng.choice([1, 1, rng.randint(2, 16), c["queries"]])
            c["keys"] = max(c["queries"], _log(rng, 1, 65536))
        c["shortest"] = rng.choice([c["keys"], rng.randint(0, c["keys"])])
        if c["pass"] == "train" and c["batch"] == 1:
            c["shortest"] = c["keys"]
        scores = c["batch"] * c["heads"] * c["queries"] * c["keys"]
        cost = scores * c["width"] * (14 if c["pass"] == "train" else 4) * (16 if dtype == "fp32" else 1)
        if cost <= COST_MOST and scores <= 1.1e9 and c["batch"] * c["keys"] * kv_heads * c["width"] <= 1 << 28:
            return c


def _lengths(case):
    """Valid tokens of every sequence of an attention case, from `shortest` to all of them: (queries, keys)."""
    B, longest, shortest = case["batch"], case["keys"], case["shortest"]
    keys = [longest if B == 1 and shortest == longest else shortest + (longest - shortest) * b // max(1, B - 1) for b in range(B)]
    if case["pass"] == "train":
        return keys, keys
    return [case["queries"]] * B, keys


def _randn(shape, dtype, gen, std=1.0):
    return (torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen) * std).to(DTYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] == "norm":
        shape = (case["batch"], case["tokens"], case["heads"], case["width"])
        if case["packed"]:      # the first of three equal parts of a fused projection's output
            x = _randn(shape[:2] + (3,) + shape[2:], case["dtype"], gen)[:, :, 0]
        else:
            x = _randn(shape, case["dtype"], gen)
        x.mul_(2.0).add_(_randn((1, 1, 1, case["width"]), case["dtype"], gen, 0.5))
        state["x"] = x
        state["weight"] = (1.0 + _randn((case["width"],), "fp32", gen, 0.1)).to(DTYPES[case["params"]])
        state["bias"] = _randn((case["width"],), case["params"], gen, 0.1) if case["bias"] else None
        if case["pass"] == "train":
            state["dy"] = _randn(shape, case["dtype"], gen)
    elif case["op"] == "rotary":
        B, L, H, D, R = case["batch"], case["tokens"], case["heads"], case["width"], case["rot"]
        if case["packed"]:      # queries and keys in front of the values in a fused projection's output
            state["x"] = _randn((B, L, H + (H + 1) // 2, D), case["dtype"], gen)[:, :, :H]
        else:
            state["x"] = _randn((B, L, H, D), case["dtype"], gen)
        f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
        state["scale"] = 1.0
        if case["scaling"] == "linear":
            f = f / 8.0
        elif case["scaling"] == "parts":
            # wave lengths over 8192 positions 32 times slower, those under 8192 / 4 as they are, in between a blend
            turns = 8192.0 * f / (2.0 * math.pi)
            keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
            f = f * (keep + (1.0 - keep) / 32.0)
            state["scale"] = 1.0 + 0.1 * math.log(32.0)
        state["frequencies"] = f.cuda()
        start = torch.randint(0, 64, (B, 1), device="cuda", generator=gen, dtype=torch.int32)
        state["positions"] = case["first"] + start + torch.arange(L, device="cuda", dtype=torch.int32)
    else:
        B, Lq, Lk, H, G, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "width"))
        if case["packed"]:
            qkv = _randn((B, Lq, H + 2 * G, D), case["dtype"], gen)
            q, k, v = qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:]
        else:
            q = _randn((B, Lq, H, D), case["dtype"], gen)
            k, v = (_randn((B, G, Lk, D), case["dtype"], gen).transpose(1, 2) if case["cache"] == "heads" else
                    _randn((B, Lk, G, D), case["dtype"], gen) for _ in range(2))
        queries, keys = _lengths(case)
        ragged = min(keys) < Lk
        state.update(q=q, k=k, v=v, scale=1.0 / math.sqrt(D), k_len=torch.tensor(keys, dtype=torch.int32).cuda() if ragged else None,
                     q_len=torch.tensor(queries, dtype=torch.int32).cuda() if ragged and case["pass"] == "train" else None)
        if case["pass"] == "train":
            state["d_out"] = _randn((B, Lq, H, D), case["dtype"], gen)
    return state


# ------------------------------------------------------------------------------------------------ plain forms

def _norm(state):
    case, x, w, b = state["case"], state["x"].float(), state["weight"].float(), state["bias"]
    mean = x.mean(-1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / ((centred * centred).mean(-1, keepdim=True) + EPS).sqrt()
    h = centred * rstd
    y = h * w
    if b is not None:
        y = y + b.float()
    out = {"y": y.to(state["x"].dtype)}
    if case["pass"] == "train":
        dy = state["dy"].float()
        a = dy * w
        dx = rstd * (a - a.mean(-1, keepdim=True) - h * (a * h).mean(-1, keepdim=True))
        out.update(dx=dx.to(state["x"].dtype), dweight=(dy * h).sum((0, 1, 2)).to(state["weight"].dtype))
        if b is not None:
            out["dbias"] = dy.sum((0, 1, 2)).to(b.dtype)
    return out


def _rotary(state):
    case, x = state["case"], state["x"].float()
    R = case["rot"]
    # the angles in 64 bits, as the frequencies are: an fp32 angle of 10^5 radians is good to three digits
    angle = state["positions"].double()[:, :, None, None] * state["frequencies"]
    cos, sin = (angle.cos() * state["scale"]).float(), (angle.sin() * state["scale"]).float()
    if case["pass"] == "backward":
        sin = -sin
    if case["layout"] == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1).to(state["x"].dtype)


def _visible(state):
    """[batch, 1, 1, queries, keys]: which keys a query sees.  The last valid query stands at the last valid key."""
    q, k = state["q"], state["k"]
    B, Lq, Lk = q.shape[0], q.shape[1], k.shape[1]
    full = torch.ones(B, dtype=torch.int32, device=q.device)
    q_len = (full * Lq if state["q_len"] is None else state["q_len"]).view(B, 1, 1)
    k_len = (full * Lk if state["k_len"] is None else state["k_len"]).view(B, 1, 1)
    i = torch.arange(Lq, device=q.device).view(1, Lq, 1)
    j = torch.arange(Lk, device=q.device).view(1, 1, Lk)
    seen = (i < q_len) & (j < k_len)
    if state["case"]["causal"]:
        seen = seen & (j <= i + k_len - q_len)
    return seen[:, None, None]


def _attention(state):
    q, k, v, scale = state["q"], state["k"], state["v"], state["scale"]
    B, Lq, H, D = q.shape
    Lk, G = k.shape[1], k.shape[2]

    def of_queries(x):          # [batch, kv head, head of the group, query, width]
        return x.float().transpose(1, 2).reshape(B, G, H // G, Lq, D)

    def back(x, like):
        return x.reshape(B, -1, x.shape[-2], D).transpose(1, 2).to(like.dtype).contiguous()

    def times_keys(x, y):       # [.., queries, width] x [.., keys, width]^T, heads of a group in one product
        return (x.reshape(B, G, -1, D) @ y.transpose(-1, -2)).view(B, G, H // G, Lq, Lk)

    def times(x, y):            # [.., queries, keys] x [.., keys, width]
        return (x.reshape(B, G, -1, Lk) @ y).view(B, G, H // G, Lq, D)

    qf, kf, vf = of_queries(q), k.float().transpose(1, 2).contiguous(), v.float().transpose(1, 2).contiguous()
    s = (times_keys(qf, kf) * scale).masked_fill(~_visible(state), -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (s - top).exp()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).view(B, H, Lq)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = times(p, vf)
    out = {"out": back(o, q), "lse": lse}
    if state["case"]["pass"] == "train":
        do = of_queries(state["d_out"])
        ds = p * (times_keys(do, vf) - (do * o).sum(-1, keepdim=True)) * scale
        out.update(dq=back(times(ds, kf), q), dk=back(ds.reshape(B, G, -1, Lk).transpose(-1, -2) @ qf.reshape(B, G, -1, D), k),
                   dv=back(p.reshape(B, G, -1, Lk).transpose(-1, -2) @ do.reshape(B, G, -1, D), v))
    return out


# ------------------------------------------------------------------------------------------- the framework's calls

def _own_norm(state):
    import paper_2501_18512_amd as sdl
    case, x, w, b = state["case"], state["x"], state["weight"], state["bias"]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if case["pass"] != "train":
        sdl.sdl_layer_norm(x, w, b, EPS, y)
        return {"y": y}
    if "space" not in state:
        state["space"] = sdl.alloc_layer_norm(x)
    mean, rstd, workspace = state["space"]
    sdl.sdl_layer_norm(x, w, b, EPS, y, mean, rstd)
    dx, dw = torch.empty_like(y), torch.empty_like(w)
    db = None if b is None else torch.empty_like(b)
    sdl.sdl_layer_norm_backward(state["dy"], x, w, mean, rstd, dx, dw, db, workspace)
    out = {"y": y, "dx": dx, "dweight": dw}
    if db is not None:
        out["dbias"] = db
    return out


def _own_rotary(state):
    import paper_2501_18512_amd as sdl
    case, x = state["case"], state["x"]
    out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    sdl.sdl_rotary(x, state["positions"], state["frequencies"], out, sdl.ROTARY_HALF if case["layout"] == "half" else sdl.ROTARY_INTERLEAVED,
                   state["scale"], inverse=case["pass"] == "backward")
    return out


def _own_attention(state):
    import paper_2501_18512_amd as sdl
    case, q, k, v = state["case"], state["q"], state["k"], state["v"]
    train = case["pass"] == "train"
    if "space" not in state:
        state["space"] = sdl.alloc_attention(q, k, backward=train)
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
    mask = {"causal": case["causal"], "q_len": state["q_len"], "k_len": state["k_len"]}
    sdl.sdl_attention(q, k, v, out, lse, state["space"], state["scale"], **mask)
    res = {"out": out, "lse": lse}
    if train:
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        sdl.sdl_attention_backward(state["d_out"], q, k, v, out, lse, dq, dk, dv, state["space"], state["scale"], **mask)
        res.update(dq=dq, dk=dk, dv=dv)
    return res


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "rotary": _own_rotary, "attention": _own_attention}[op](state)
    return {"norm": _norm, "rotary": _rotary, "attention": _attention}[op](state)


# --------------------------------------------------------------------------------------------------- yardsticks

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        rows, C = case["batch"] * case["tokens"] * case["heads"], case["width"]
        param = C * (2 if case["params"] == "bf16" else 4) * (2 if case["bias"] else 1)
        if case["pass"] == "train":     # x, y, dy, dx; the parameters and their gradients
            return {"bytes": 4 * rows * C * size + 2 * param, "flops": 20 * rows * C}
        return {"bytes": 2 * rows * C * size + param, "flops": 8 * rows * C}
    if case["op"] == "rotary":
        n = case["batch"] * case["tokens"] * case["heads"]
        return {"bytes": 2 * n * case["width"] * size + 4 * case["batch"] * case["tokens"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    H, G, D = case["heads"], case["kv_heads"], case["width"]
    pairs = rows = keys = 0             # (query, key) pairs that see each other, valid queries, valid keys
    for nq, nk in zip(*_lengths(case)):
        if case["causal"]:              # query i sees min(nk, i + 1 + nk - nq) keys, none where that is negative
            short = max(0, nq - nk)
            n = nq - short
            pairs += n * (nk - nq + short) + n * (n + 1) // 2
        else:
            pairs += nq * nk
        rows, keys = rows + nq, keys + nk
    every = case["batch"] * case["queries"]
    # q is read and out written, k and v are read, lse is written
    nbytes = (rows + every) * H * D * size + 2 * keys * G * D * size + 4 * every * H
    if case["pass"] == "train":         # d_out is read; dq, dk and dv are written
        nbytes += (rows + every) * H * D * size + 2 * case["batch"] * case["keys"] * G * D * size
    return {"bytes": nbytes, "flops": pairs * H * D * (14 if case["pass"] == "train" else 4)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        x, w = state["x"].double(), state["weight"].double()
        n = case["width"]
        mu = x.sum(-1, keepdim=True) / n
        var = ((x - mu) ** 2).sum(-1, keepdim=True) / n
        h = (x - mu) / torch.sqrt(var + EPS)
        out = {"y": torch.addcmul(torch.zeros_like(w) if state["bias"] is None else state["bias"].double(), h, w)}
        if case["pass"] == "train":
            dy = state["dy"].double()
            dh = dy * w
            out["dx"] = (n * dh - dh.sum(-1, keepdim=True) - h * (dh * h).sum(-1, keepdim=True)) / (n * torch.sqrt(var + EPS))
            out["dweight"] = (dy * h).reshape(-1, n).sum(0)
            if state["bias"] is not None:
                out["dbias"] = dy.reshape(-1, n).sum(0)
        return out
    if case["op"] == "rotary":
        R = case["rot"]
        angle = torch.outer(state["positions"].reshape(-1).double(), state["frequencies"]).view(*state["positions"].shape, 1, R // 2)
        turn = torch.polar(torch.full_like(angle, state["scale"]), -angle if case["pass"] == "backward" else angle)
        x = state["x"].double()
        out = x.clone()
        first, second = (slice(0, R // 2), slice(R // 2, R)) if case["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        out[..., first], out[..., second] = z.real, z.imag
        return out
    q, k, v = (state[n].double() for n in ("q", "k", "v"))
    B, Lq, H, D = q.shape
    share = H // k.shape[2]
    train = case["pass"] == "train"
    res = {"out": torch.zeros_like(q), "lse": torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device=q.device)}
    if train:
        do = state["d_out"].double()
        res.update(dq=torch.zeros_like(q), dk=torch.zeros(k.shape, dtype=k.dtype, device=k.device), dv=torch.zeros(v.shape, dtype=v.dtype, device=v.device))
    for b, (nq, nk) in enumerate(zip(*_lengths(case))):
        if nq == 0 or nk == 0:
            continue
        hidden = torch.ones((nq, nk), dtype=torch.bool, device=q.device).triu(nk - nq + 1) if case["causal"] else None
        for h in range(H):
            g = h // share
            kk, vv = k[b, :nk, g].contiguous(), v[b, :nk, g].contiguous()
            s = torch.mm(q[b, :nq, h], kk.T) * state["scale"]
            if hidden is not None:
                s[hidden] = -math.inf
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
            res["lse"][b, h, :nq] = lse
            o = torch.mm(p, vv)
            res["out"][b, :nq, h] = o
            if train:
                d = do[b, :nq, h].contiguous()
                dp = torch.mm(d, vv.T)
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * state["scale"]
                res["dq"][b, :nq, h] = torch.mm(ds, kk)
                res["dk"][b, :nk, g] += torch.mm(ds.T.contiguous(), q[b, :nq, h].contiguous())
                res["dv"][b, :nk, g] += torch.mm(p.T.contiguous(), d)
    return res
