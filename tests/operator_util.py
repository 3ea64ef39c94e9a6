"""What the tests of the inner step's operators share: inputs in odd places, and bounds on their errors.

u(type) is half a unit in the last place of 1: what one rounding to the type costs, relatively.  A sum of n terms in fp32 is off by at most
n u(fp32) times the sum of their absolute values, whatever its order."""
import torch

BF16, FP32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24
U = {BF16: 2.0 ** -8, FP32: U32}
TINY = 1e-37              # results under the least normal numbers may be flushed


def randn(shape, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(dtype)


def placed(t, how="dense"):
    """t on the GPU with the same values: dense; with every row one element off its alignment and gaps between them ("odd"); one of three
    parts of a fused projection's output ("packed"); or with heads in front of tokens ("heads", four dimensions)."""
    if how == "dense":
        return t.cuda()
    if how == "heads":
        return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    if how == "odd":
        big = torch.full((*t.shape[:-1], t.shape[-1] + 3), float("nan"), dtype=t.dtype, device="cuda")
        view = big[..., 1:1 + t.shape[-1]]
    else:
        big = torch.full((*t.shape[:-2], 3, *t.shape[-2:]), float("nan"), dtype=t.dtype, device="cuda")
        view = big.select(-3, 1)
    view.copy_(t)
    return view


def output(like, how="dense"):
    """An uninitialised output (NaN everywhere) and a function that says whether what lies around it is untouched."""
    t = placed(torch.full(like.shape, float("nan"), dtype=like.dtype), how)
    base = t._base if t._base is not None else t

    def untouched():
        inside = torch.zeros_like(base, dtype=torch.bool)
        inside.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(True)
        return bool(torch.isnan(base[~inside].float()).all())
    return t, untouched


def close(got, want, bound, what):
    """|got - want| <= bound, element by element (bound may be a tensor); infinities have to be equal."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert not torch.isnan(got).any(), f"{what}: NaN"
    same = got == want
    off = (got - want).abs()
    bad = ~same & ~(off <= torch.as_tensor(bound, dtype=torch.float64) + TINY)
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bound, first at {i}: got {got[i]!r} want {want[i]!r}")
