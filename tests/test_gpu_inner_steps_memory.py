"""What the example's operators keep from the forward to the backward pass: their inputs, results and statistics, and no workspace."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def _bytes(*tensors):
    return sum(t.numel() * t.element_size() for t in tensors)


def test_no_workspace_is_kept_for_the_backward_pass():
    import inner_steps as ex
    x, w = torch.randn(2, 30, 4, 256, device="cuda").bfloat16(), torch.ones(256, device="cuda").bfloat16()
    y = ex.LayerNorm.apply(x.requires_grad_(), w.requires_grad_())
    assert _bytes(*y.grad_fn.saved_tensors) == _bytes(x, w) + 2 * 4 * 2 * 30 * 4
    q, k, v = (torch.randn(2, 30, n, 64, device="cuda").bfloat16().requires_grad_() for n in (4, 2, 2))
    out = ex.Attention.apply(q, k, v)
    assert _bytes(*out.grad_fn.saved_tensors) == _bytes(q, k, v, out) + 4 * 2 * 4 * 30
    grads = torch.autograd.grad(out.float().sum() + y.float().sum(), (x, w, q, k, v))
    assert all(bool(torch.isfinite(g.float()).all()) for g in grads)
