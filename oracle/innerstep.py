"""Layer norm, rotary positions and attention with their gradients, in 64 bits on the CPU, as the formulas have them
(test infrastructure only: loops over rows or heads, nothing shared with the GPU path)."""
import math

import torch


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) of x [..., width]."""
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    y = (x - mean) * rstd
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean[..., 0], rstd[..., 0]


def layer_norm_backward(dy, x, weight, eps):
    """(dx, dweight, dbias)."""
    dy, (h, _, rstd) = dy.double(), layer_norm(x, None, None, eps)
    a = dy if weight is None else dy * weight.double()
    dx = rstd[..., None] * (a - a.mean(-1, keepdim=True) - h * (a * h).mean(-1, keepdim=True))
    rows = tuple(range(dy.dim() - 1))
    return dx, (dy * h).sum(rows), dy.sum(rows)


def rotary(x, positions, frequencies, interleaved, scale, inverse):
    """x [batch, tokens, heads, width], positions [batch, tokens], frequencies [rot / 2]."""
    x, half = x.double(), len(frequencies)
    out = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = positions.double()[..., None] * float(frequencies[i]) * (-1.0 if inverse else 1.0)
        out[..., a] = scale * (x[..., a] * torch.cos(angle) - x[..., b] * torch.sin(angle))
        out[..., b] = scale * (x[..., a] * torch.sin(angle) + x[..., b] * torch.cos(angle))
    return out


def seen(queries, keys, nq, nk, causal):
    """Boolean [queries, keys]: which keys a query sees, of nq valid queries and nk valid keys."""
    return torch.tensor([[i < nq and j < nk and (not causal or j <= i + nk - nq) for j in range(keys)] for i in range(queries)],
                        dtype=torch.bool).reshape(queries, keys)


def attention(q, k, v, scale, causal=False, q_len=None, k_len=None, d_out=None):
    """A dict: out, lse, with d_out also dq, dk, dv; and what error bounds are made of: for every output the same sums over absolute
    values (`out_abs`, `dv_abs`), and per head the largest sum of |q||k| (`score_abs`)."""
    B, Lq, H, D = q.shape
    Lk, G = k.shape[1], k.shape[2]
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64)  # noqa: E731
    r = {"out": zeros(q), "lse": torch.full((B, H, Lq), -math.inf, dtype=torch.float64), "out_abs": zeros(q), "p": [], "score_abs": 0.0}
    if d_out is not None:
        r.update(dq=zeros(q), dk=zeros(k), dv=zeros(v), dv_abs=zeros(v))
    for b in range(B):
        nq = Lq if q_len is None else max(0, min(Lq, int(q_len[b])))
        nk = Lk if k_len is None else max(0, min(Lk, int(k_len[b])))
        see = seen(Lq, Lk, nq, nk, causal)[:nq, :nk]
        for h in range(H):
            g = h * G // H
            qq, kk, vv = q[b, :nq, h].double(), k[b, :nk, g].double(), v[b, :nk, g].double()
            s = scale * (qq @ kk.T)
            e = torch.where(see, torch.exp(s - torch.where(see, s, -math.inf).amax(1, keepdim=True).clamp(min=-1e300) if nk else s), 0.0)
            total = e.sum(1, keepdim=True)
            p = e / torch.where(total == 0, 1.0, total)
            any_key = see.any(1)
            if nk:
                r["lse"][b, h, :nq] = torch.where(any_key, torch.logsumexp(torch.where(see, s, -math.inf), 1), -math.inf)
                r["score_abs"] = max(r["score_abs"], float((scale * (qq.abs() @ kk.abs().T)).max()) if nq else 0.0)
            r["out"][b, :nq, h] = o = p @ vv
            r["out_abs"][b, :nq, h] = p @ vv.abs()
            r["p"].append((b, h, g, nq, nk, p))
            if d_out is not None:
                do = d_out[b, :nq, h].double()
                ds = p * (do @ vv.T - (do * o).sum(1, keepdim=True))
                r["dq"][b, :nq, h] = scale * (ds @ kk)
                r["dk"][b, :nk, g] += scale * (ds.T @ qq)
                r["dv"][b, :nk, g] += p.T @ do
                r["dv_abs"][b, :nk, g] += p.T @ do.abs()
    return r
