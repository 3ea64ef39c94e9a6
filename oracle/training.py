"""The operators at the decoder's two ends and the update of its matrices, in 64 bits on the CPU, from their definitions.  Inputs of any type are taken as the
values they stand for."""
import torch

F64 = torch.float64


def embedding(table, tokens, scale):
    V = table.shape[0]
    out = torch.zeros((*tokens.shape, table.shape[1]), dtype=F64)
    for place in (tokens.ge(0) & tokens.lt(V)).nonzero().tolist():
        out[tuple(place)] = scale * table[int(tokens[tuple(place)])].double()
    return out


def embedding_backward(d_out, tokens, vocab, scale):
    """The gradient of the table, the sum of absolute values of its terms, and how many there are."""
    d, t = d_out.double().reshape(-1, d_out.shape[-1]), tokens.reshape(-1).tolist()
    total, size, count = (torch.zeros((vocab, d.shape[1]), dtype=F64) for _ in range(3))
    for i, v in enumerate(t):
        if 0 <= v < vocab:
            total[v] += scale * d[i]
            size[v] += abs(scale) * d[i].abs()
            count[v] += 1
    return total, size, count


def cross_entropy(x, targets, smoothing, z):
    """(loss, lse) of rows; 0 without a target."""
    x, V = x.double(), x.shape[-1]
    there = targets.ge(0) & targets.lt(V)
    # around the row's maximum: log 5 is lost in 64 bits, too, beside logits of 10^38
    top = x.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, torch.zeros(()).double())
    lse = top[..., 0] + torch.logsumexp(x - top, -1)
    hit = (x - top).gather(-1, targets.long().clamp(0, V - 1)[..., None])[..., 0]
    loss = torch.logsumexp(x - top, -1) - (1.0 - smoothing) * hit + z * lse ** 2
    if smoothing:
        loss = loss - smoothing * (x - top).mean(-1)
    return loss.where(there, torch.zeros(())), lse.where(there, torch.zeros(()))


def cross_entropy_backward(x, targets, lse, d_loss, smoothing, z):
    """The gradient of the rows' losses, weighted by d_loss, from lse; lse None: from the probabilities themselves."""
    x, V = x.double(), x.shape[-1]
    p = torch.softmax(x, -1) if lse is None else torch.exp(x - lse.double()[..., None])
    lse = torch.logsumexp(x, -1) if lse is None else lse.double()
    there = targets.ge(0) & targets.lt(V)
    want = torch.full(x.shape, smoothing / V, dtype=F64)
    want.scatter_add_(-1, targets.long().clamp(0, V - 1)[..., None], torch.full((*targets.shape, 1), 1.0 - smoothing, dtype=F64))
    d = (1.0 + 2.0 * z * lse)[..., None] * p - want
    return (d * d_loss.double()[..., None]).where(there[..., None], torch.zeros(()))


def orthogonalize(x, coefficients, eps, scale):
    """U p(S) V^T of one matrix' singular values and vectors."""
    x = x.double()
    u, s, vt = torch.linalg.svd(x / (x.square().sum().sqrt() + eps), full_matrices=False)
    for a, b, c in coefficients:
        s = a * s + b * s ** 3 + c * s ** 5
    return scale * (u * s) @ vt


def orthogonalize_rounded(x, coefficients, eps, scale, bits, held, held_x):
    """The steps themselves with operands of `bits` bits, X of `held_x`, the products' results and the diagonals of the symmetric ones, which are kept apart, of `held` bits,
    everything else in 64: what these roundings cost is how far this is from orthogonalize()."""
    def to(v, n):
        m, e = torch.frexp(v)
        return torch.ldexp((m * 2.0 ** n).round() * 2.0 ** -n, e)
    def cut(v):
        d = v.diagonal()
        return d, to(v - torch.diag(d), bits)
    x = x.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = to(x / (x.square().sum().sqrt() + eps), held_x)
    for a, b, c in coefficients:
        low = to(x, bits)
        d, gram = cut(to(low @ low.T, held))
        whole = gram + torch.diag(d)
        square = to(gram @ gram, held) + (d[:, None] + d[None]) * gram + torch.diag(d * d)
        d, mix = cut(to(b * whole + c * square, held))
        x = to((a + d)[:, None] * x + to(mix @ low, held), held_x)
    return scale * (x.T if tall else x)
