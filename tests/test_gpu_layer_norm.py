"""GPU parity of sdl_layer_norm and its backward pass with the 64-bit oracle.

Bounds.  The mean is off by at most (n + 1) u mean|x| =: m, h by e = rstd (m + 2 u (|x| + |mean|)) + |h| (n + 8) u, as the sum of squares has n terms and
the root, the division and the products a rounding each.  y: |w| e + 2 u (|h w| + |b|) and the type's rounding.  dx: the two means over n
products, with h's error in each, are off by (n + 4) u mean|a| and (n + 4) u mean|a h| + mean(|a| e).  dweight: sum |dy| e + rows u sum |dy h|."""
import pytest
import torch

import paper_2501_18512_amd as sdl
from operator_util import BF16, FP32, U, U32, close, output, placed, randn
from oracle import innerstep as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5
# widths on both sides of every launch shape's limit, odd ones, the smallest; row counts under and over a workgroup's
SHAPES = [(1, 1), (3, 1), (5, 2), (33, 7), (9, 8), (130, 64), (17, 65), (70, 128), (5, 200), (260, 256), (3, 257), (11, 512), (9, 513), (2, 768),
          (40, 1021), (7, 1024), (6, 1025), (300, 2048), (3, 2049), (2, 4096), (4, 4097), (2, 8192), (2, 8193), (1, 16384), (600, 33)]


def _case(shape, dtype, params, how, seed, bias=True, weight=True):
    x = randn(shape, dtype, seed, 2.0) + randn((shape[-1],), dtype, seed + 1, 0.5)
    w = (1.0 + randn((shape[-1],), torch.float64, seed + 2, 0.1)).to(params) if weight else None
    b = randn((shape[-1],), params, seed + 3, 0.1) if bias else None
    return x, w, b, randn(shape, dtype, seed + 4), placed(x, how)


def _check(x, w, b, dy, xg, how, eps=EPS):
    dtype, n = x.dtype, x.shape[-1]
    rows = x.numel() // n
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    y, y_alone = output(x, how)
    mean, rstd, workspace = sdl.alloc_layer_norm(xg)
    wg, bg = cuda(w), cuda(b)
    sdl.sdl_layer_norm(xg, wg, bg, eps, y, mean, rstd)
    dx, dx_alone = output(x, how)
    dw = torch.full((n,), float("nan"), dtype=FP32 if w is None else w.dtype, device="cuda")
    db = torch.full_like(dw, float("nan"))
    sdl.sdl_layer_norm_backward(placed(dy, how), xg, wg, mean, rstd, dx, dw, db, workspace)
    torch.cuda.synchronize()
    assert y_alone() and dx_alone()
    want_y, want_mean, want_rstd = ref.layer_norm(x, w, b, eps)
    want_dx, want_dw, want_db = ref.layer_norm_backward(dy, x, w, eps)
    X, D = x.double(), dy.double()
    W = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    m = (n + 1) * U32 * X.abs().mean(-1, keepdim=True)
    h = (X - want_mean[..., None]) * want_rstd[..., None]
    e = want_rstd[..., None] * (m + 2 * U32 * (X.abs() + want_mean[..., None].abs())) + h.abs() * (n + 8) * U32
    # a row of equal elements has rstd = 1 / sqrt(eps), and the mean's own error squared under the root
    rel = (n + 8) * U32 + (want_rstd * m[..., 0]) ** 2
    close(mean, want_mean, m[..., 0], "mean")
    close(rstd, want_rstd, want_rstd * rel, "rstd")
    e = e + h.abs() * rel[..., None]
    B = torch.zeros(n, dtype=torch.float64) if b is None else b.double()
    close(y, want_y, U[dtype] * want_y.abs() + 1.01 * (W.abs() * e + 2 * U32 * ((h * W).abs() + B.abs())), "y")
    a = (D * W).abs()
    e1 = (n + 4) * U32 * a.mean(-1, keepdim=True)
    e2 = (n + 4) * U32 * (a * h.abs()).mean(-1, keepdim=True) + (a * e).mean(-1, keepdim=True)
    c2 = (D * W * h).mean(-1, keepdim=True).abs()
    inner = 4 * U32 * (a + (h * c2).abs() + a.mean(-1, keepdim=True)) + e1 + h.abs() * e2 + e * (c2 + e2)
    close(dx, want_dx, U[dtype] * want_dx.abs() + 1.01 * (want_rstd[..., None] * inner + want_dx.abs() * (rel[..., None] + 2 * U32)), "dx")
    up, flat = U[dw.dtype], tuple(range(x.dim() - 1))
    close(dw, want_dw, up * want_dw.abs() + 1.01 * ((D.abs() * e).sum(flat) + (rows + 4) * U32 * (D * h).abs().sum(flat)), "dweight")
    close(db, want_db, up * want_db.abs() + 1.01 * (rows + 4) * U32 * D.abs().sum(flat), "dbias")


@pytest.mark.parametrize("dtype,params", [(BF16, BF16), (FP32, FP32), (BF16, FP32), (FP32, BF16)])
def test_forward_and_backward(dtype, params):
    for i, shape in enumerate(SHAPES):
        print(f"norm {shape} {dtype} {params}", flush=True)
        _check(*_case(shape, dtype, params, "dense", 10 * i), "dense")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("how", ["odd", "packed", "heads"])
def test_rows_where_they_lie(dtype, how):
    for i, shape in enumerate([(2, 5, 3, 64), (1, 7, 4, 33), (3, 2, 5, 128), (2, 3, 1, 1030), (4, 1, 6, 80), (1, 3, 2, 5000)]):
        print(f"norm {shape} {dtype} {how}", flush=True)
        _check(*_case(shape, dtype, dtype, how, 100 + 10 * i), how)


def test_without_parameters_and_with_eps_that_matters():
    _check(*_case((9, 96), BF16, BF16, "dense", 1, bias=False), "dense")
    _check(*_case((9, 96), FP32, FP32, "dense", 2, bias=False, weight=False), "dense")
    x, w, b, dy, _ = _case((6, 300), FP32, FP32, "dense", 3)
    x = x * 1e-3 + 0.25 * (torch.arange(6) % 2)[:, None]          # rows whose variance is under eps, and rows of large equal parts
    x[4] = 3.0                                                     # a row of equal elements
    _check(x, w, b, dy, x.cuda(), "dense", eps=1e-3)


def test_more_rows_than_workgroups_hold_at_a_time():
    _check(*_case((20011, 40), BF16, FP32, "dense", 5), "dense")
    _check(*_case((4000, 600), FP32, FP32, "dense", 6), "dense")


def test_in_place_repeatable_and_on_another_stream():
    x, w, b, dy, xg = _case((700, 768), BF16, BF16, "dense", 7)
    w, b, dy = w.cuda(), b.cuda(), dy.cuda()
    y, other = torch.empty_like(xg), xg.clone()
    sdl.sdl_layer_norm(xg, w, b, EPS, y)
    sdl.sdl_layer_norm(other, w, b, EPS, other)
    assert torch.equal(y, other)
    got = []
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        stream.wait_stream(torch.cuda.current_stream())
        mean, rstd, workspace = sdl.alloc_layer_norm(xg)
        dx, dw, db = torch.empty_like(xg), torch.empty_like(w), torch.empty_like(b)
        sdl.sdl_layer_norm(xg, w, b, EPS, y, mean, rstd, stream=stream)
        sdl.sdl_layer_norm_backward(dy, xg, w, mean, rstd, dx, dw, db, workspace, stream=stream)
        torch.cuda.synchronize()
        got.append((dx, dw, db))
    assert all(torch.equal(a, c) for a, c in zip(*got))
    sdl.sdl_layer_norm_backward(dy, xg, w, mean, rstd, dy, dw, db, workspace)          # dx in dy's place
    assert torch.equal(dy, got[0][0]) and torch.equal(dw, got[0][1])


def test_no_rows_and_no_sums():
    x = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    mean, rstd, workspace = sdl.alloc_layer_norm(x)
    dw, db = torch.full_like(w, 7.0), torch.full_like(w, 7.0)
    sdl.sdl_layer_norm(x, w, None, EPS, x, mean, rstd)
    sdl.sdl_layer_norm_backward(x, x, w, mean, rstd, x, dw, db, workspace)
    assert not dw.any() and not db.any()
    x = randn((5, 64), FP32, 1).cuda()
    mean, rstd, _ = sdl.alloc_layer_norm(x)
    y, dx, dx2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    sdl.sdl_layer_norm(x, w, None, EPS, y, mean, rstd)
    sdl.sdl_layer_norm_backward(x, x, w, mean, rstd, dx, None, None, None)
    sdl.sdl_layer_norm_backward(x, x, w, mean, rstd, dx2, None, db, sdl.alloc_layer_norm(x)[2])
    assert torch.equal(dx, dx2) and torch.allclose(db, x.sum(0), atol=1e-5)


def test_gradient_against_differences():
    x, w, b, dy, xg = _case((4, 50), FP32, FP32, "dense", 11)
    mean, rstd, workspace = sdl.alloc_layer_norm(xg)
    y, dx, dw, db = torch.empty_like(xg), torch.empty_like(xg), torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    sdl.sdl_layer_norm(xg, w.cuda(), b.cuda(), EPS, y, mean, rstd)
    sdl.sdl_layer_norm_backward(dy.cuda(), xg, w.cuda(), mean, rstd, dx, dw, db, workspace)
    loss = lambda x, w, b: float((ref.layer_norm(x, w, b, EPS)[0] * dy.double()).sum())  # noqa: E731
    args = [t.double() for t in (x, w, b)]
    for k, grad in enumerate((dx, dw, db)):
        way = randn(args[k].shape, torch.float64, 20 + k)
        there, back = (loss(*[t + s * 1e-5 * way if i == k else t for i, t in enumerate(args)]) for s in (1, -1))
        slope = (there - back) / 2e-5
        # central differences are good to about 1e-10 here, the fp32 gradient to 1e-6 of the sum of absolute values
        assert abs(slope - float((grad.cpu().double() * way).sum())) < 1e-5 * float((grad.cpu().double() * way).abs().sum())


def test_values_that_are_not_finite_stay_in_their_row():
    x = randn((6, 200), BF16, 3).cuda()
    x[2, 50], x[4, 199] = float("inf"), float("nan")
    y = torch.empty_like(x)
    sdl.sdl_layer_norm(x, None, None, EPS, y)
    bad = torch.isnan(y.float()).any(1).tolist()
    assert bad == [False, False, True, False, True, False]
