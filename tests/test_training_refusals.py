"""What the operators at the decoder's two ends and of its matrices' update refuse, before anything is launched (CPU only: no refused call touches an address)."""
import ctypes
import functools
import math

import pytest
import torch

import paper_2501_18512_amd as sdl

INVALID, UNSUPPORTED, ALIGNMENT, OK = -1, -2, -3, 0
INF, NAN = math.inf, math.nan


def view(data=0x10000, batch=1 << 20, token=1 << 10, head=0):
    return sdl._View(data, batch, token, head)


def numbers(*x):
    return (ctypes.c_float * len(x))(*x)


def call(name, **change):
    """The C entry point with arguments that would be launched, but for `change`."""
    loss = dict(logits=view(), batch=2, tokens=3, vocab=100, dtype=1, targets=0x20000, index=1, smoothing=0.1, z=1e-4)
    good = {
        "sdl_embedding": dict(table=0x10000, stride=64, vocab=100, width=64, table_dtype=1, tokens=0x20000, index=1, batch=2, count=3, scale=1.0, out=view(0x30000), dtype=1),
        "sdl_embedding_backward": dict(d_out=view(), dtype=1, tokens=0x20000, index=1, batch=2, count=3, scale=1.0, d_table=0x30000, stride=64, vocab=100, width=64,
                                       table_dtype=1, workspace=0x40000, workspace_bytes=1 << 24),
        "sdl_cross_entropy": dict(**loss, loss=0x30000, lse=0x40000, d_loss=0x50000, d_logits=view(0x60000)),
        "sdl_cross_entropy_backward": dict(**loss, lse=0x40000, d_loss=0x50000, d_logits=view(0x60000)),
        "sdl_orthogonalize": dict(x=view(), batch=2, rows=30, cols=40, dtype=1, coefficients=numbers(1.5, -0.5, 0.0), steps=1, eps=1e-7, scale=1.0, out=view(0x40000),
                                  out_dtype=1, workspace=0x80000, workspace_bytes=1 << 30),
    }[name]
    assert set(change) <= set(good)
    return getattr(sdl._lib, name)(*{**good, **change}.values(), None)


EMBEDDING = [
    (INVALID, dict(width=0)), (INVALID, dict(dtype=2)), (INVALID, dict(table_dtype=-1)), (INVALID, dict(index=2)), (INVALID, dict(index=-1)), (INVALID, dict(scale=NAN)),
    (INVALID, dict(scale=INF)), (INVALID, dict(tokens=None)), (UNSUPPORTED, dict(width=65537)), (UNSUPPORTED, dict(vocab=1 << 31)),
    (UNSUPPORTED, dict(batch=1 << 16, count=1 << 15)), (UNSUPPORTED, dict(batch=1 << 31, count=1 << 31)), (ALIGNMENT, dict(tokens=0x20004)), (ALIGNMENT, dict(index=0, tokens=0x20002)),
]


@pytest.mark.parametrize("status,change", EMBEDDING + [
    (INVALID, dict(table=None)), (INVALID, dict(out=None)), (INVALID, dict(out=view(0))), (INVALID, dict(out=view(0x30000, batch=0))), (INVALID, dict(out=view(0x30000, token=0))),
    (ALIGNMENT, dict(table=0x10001)), (ALIGNMENT, dict(out=view(0x30001))), (ALIGNMENT, dict(dtype=0, out=view(0x30002))), (ALIGNMENT, dict(table_dtype=0, table=0x10002)),
    (OK, dict(batch=0)), (OK, dict(count=0, out=None, tokens=None))])
def test_embedding(status, change):
    assert call("sdl_embedding", **change) == status


@pytest.mark.parametrize("status,change", EMBEDDING + [
    (INVALID, dict(d_out=None)), (INVALID, dict(d_table=None)), (INVALID, dict(stride=0)), (INVALID, dict(workspace=None)), (INVALID, dict(workspace_bytes=8)),
    (UNSUPPORTED, dict(batch=1, count=(1 << 28) + 1, workspace_bytes=1 << 62)), (ALIGNMENT, dict(d_out=view(0x10001))), (ALIGNMENT, dict(d_table=0x30001)),
    (ALIGNMENT, dict(workspace=0x40004)), (OK, dict(vocab=0, d_table=None))])
def test_embedding_backward(status, change):
    assert call("sdl_embedding_backward", **change) == status


CROSS_ENTROPY = [
    (INVALID, dict(logits=None)), (INVALID, dict(logits=view(0))), (INVALID, dict(vocab=0)), (INVALID, dict(dtype=2)), (INVALID, dict(targets=None)), (INVALID, dict(index=3)),
    (INVALID, dict(smoothing=-0.1)), (INVALID, dict(smoothing=1.5)), (INVALID, dict(smoothing=NAN)), (INVALID, dict(z=NAN)), (INVALID, dict(z=INF)), (INVALID, dict(z=-1e-4)),
    (INVALID, dict(d_logits=view(0))), (INVALID, dict(d_logits=view(0x60000, token=0))), (INVALID, dict(d_logits=view(0x60000, batch=0))),
    (INVALID, dict(d_logits=view(0x10000, token=512))), (UNSUPPORTED, dict(vocab=(1 << 24) + 1)), (UNSUPPORTED, dict(batch=1 << 16, tokens=1 << 15)),
    (UNSUPPORTED, dict(batch=1 << 31, tokens=1 << 31)), (ALIGNMENT, dict(logits=view(0x10001))), (ALIGNMENT, dict(targets=0x20004)), (ALIGNMENT, dict(lse=0x40002)),
    (ALIGNMENT, dict(d_loss=0x50001)), (ALIGNMENT, dict(d_logits=view(0x60001))), (OK, dict(batch=0)), (OK, dict(tokens=0, logits=None, d_logits=None)),
]


@pytest.mark.parametrize("status,change", CROSS_ENTROPY + [(INVALID, dict(loss=None, lse=None, d_logits=None)), (ALIGNMENT, dict(loss=0x30001))])
def test_cross_entropy(status, change):
    assert call("sdl_cross_entropy", **change) == status


@pytest.mark.parametrize("status,change", CROSS_ENTROPY + [(INVALID, dict(lse=None)), (INVALID, dict(d_logits=None))])
def test_cross_entropy_backward(status, change):
    assert call("sdl_cross_entropy_backward", **change) == status


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=None)), (INVALID, dict(x=view(0))), (INVALID, dict(out=None)), (INVALID, dict(out=view(0x40000, token=0))), (INVALID, dict(out=view(0x40000, batch=0))),
    (INVALID, dict(dtype=2)), (INVALID, dict(out_dtype=7)), (INVALID, dict(steps=0)), (INVALID, dict(coefficients=None)), (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=NAN)),
    (INVALID, dict(eps=INF)), (INVALID, dict(scale=NAN)), (INVALID, dict(scale=-INF)), (INVALID, dict(workspace=None)), (INVALID, dict(workspace_bytes=1000)),
    (UNSUPPORTED, dict(rows=65537)), (UNSUPPORTED, dict(cols=1 << 31)), (UNSUPPORTED, dict(batch=65536)), (UNSUPPORTED, dict(batch=65535, rows=8192, cols=8192)),
    (ALIGNMENT, dict(x=view(0x10001))), (ALIGNMENT, dict(out=view(0x40001))), (ALIGNMENT, dict(workspace=0x80008)), (ALIGNMENT, dict(dtype=0, x=view(0x10002))),
    (INVALID, dict(out=view(token=1 << 9))), (INVALID, dict(out=view(batch=1 << 19))), (INVALID, dict(out=view(), out_dtype=0)),
    (OK, dict(batch=0)), (OK, dict(rows=0, x=None, out=None)), (OK, dict(cols=0))])
def test_orthogonalize(status, change):
    assert call("sdl_orthogonalize", **change) == status


@pytest.mark.parametrize("steps", [
    [(3.0, 0.0, 0.0)], [(-2.5, 0.0, 0.0)], [(NAN, 0.0, 0.0)], [(1.0, INF, 0.0)], [(1.0, 0.0, -INF)], [(1e30, -1e30, 0.0)], [(1.5, 0.0, 0.0)] * 2, [(1.5, -0.5, 0.0), (1.9, -0.5, 2.0)],
    [(8.0, -8.0, 0.0)], [(3.4445, -4.7750, 3.5)]])
def test_coefficients_that_lift_a_singular_value_beyond_two(steps):
    flat = [x for s in steps for x in s]
    assert call("sdl_orthogonalize", coefficients=numbers(*flat), steps=len(steps)) == INVALID


def test_coefficients_that_are_known_not_to():
    """Without matrices nothing is launched, and the coefficients are looked at all the same."""
    for steps in (sdl.ORTHOGONALIZE_QUINTIC, sdl.ORTHOGONALIZE_CUBIC * 3, [(2.0, 0.0, 0.0)], [(0.0, 0.0, 0.0)], [(2.0, -1.5, 0.5)] * 10, [(1.0, 1e-9, -1e-9)]):
        assert call("sdl_orthogonalize", batch=0, coefficients=numbers(*[x for s in steps for x in s]), steps=len(steps)) == OK
    assert call("sdl_orthogonalize", batch=0, coefficients=numbers(3.0, 0.0, 0.0)) == INVALID


def test_workspace_sizes_of_what_is_refused_are_nothing():
    assert sdl.sdl_embedding_workspace_bytes(0, 64) == 0 and sdl.sdl_embedding_workspace_bytes(1 << 29, 64) == 0 and sdl.sdl_embedding_workspace_bytes(10, 65537) == 0
    assert sdl.sdl_embedding_workspace_bytes(10, 64) >= 80
    f = sdl.sdl_orthogonalize_workspace_bytes
    assert f(1, 100, 200, 1) > 0 and f(0, 100, 200, 1) == 0 and f(1, 0, 200, 1) == 0 and f(1, 100, 0, 1) == 0 and f(1, 100, 200, 2) == 0 and f(1, 65537, 1, 1) == 0
    assert f(65536, 1, 1, 0) == 0 and f(1, 100, 200, 0) == f(1, 200, 100, 0)
    assert f(4, 2048, 2048, 0) > f(4, 2048, 2048, 1) > 4 * 2048 * 2048 * 4


class Device(torch.Tensor):
    """A host tensor that says it is on the device, for the checks that come before any address is used."""
    is_cuda = True


def on_device(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


def ids(*shape, dtype=torch.int64):
    return on_device(*shape, dtype=dtype)


class Default:
    """The binding's calls on the default stream, which they need not ask a device for."""

    def __getattr__(self, name):
        return functools.partial(getattr(sdl, name), stream=0)


def test_the_binding_refuses_what_does_not_belong_together():
    on = Default()
    table, t, out = on_device(10, 8), ids(2, 3), on_device(2, 3, 8)
    space, rows = on_device(1 << 20), on_device(2, 3)
    logits, loss = on_device(2, 3, 8), on_device(2, 3)
    m = on_device(2, 4, 6)
    bad = [
        lambda: on.sdl_embedding(on_device(10, 9), t, out),
        lambda: on.sdl_embedding(on_device(2, 10, 8), t, out),
        lambda: on.sdl_embedding(table, ids(2, 4), out),
        lambda: on.sdl_embedding(table, ids(2, 3, dtype=torch.int16), out),
        lambda: on.sdl_embedding(table, None, out),
        lambda: on.sdl_embedding(table, ids(3, 2).t(), out),
        lambda: on.sdl_embedding(table, t, on_device(1, 2, 3, 8)),
        lambda: on.sdl_embedding(table.double(), t, out),
        lambda: on.sdl_embedding(torch.zeros(10, 8), t, out),
        lambda: on.sdl_embedding(table, torch.zeros(2, 3, dtype=torch.int64), out),
        lambda: on.sdl_embedding_backward(out, t, on_device(10, 9), space),
        lambda: on.sdl_embedding_backward(out, ids(5), table, space),
        lambda: on.sdl_embedding_backward(out, t, table.t(), space),
        lambda: on.sdl_cross_entropy(logits, ids(2, 2), loss),
        lambda: on.sdl_cross_entropy(logits, t, on_device(2, 2)),
        lambda: on.sdl_cross_entropy(logits, t, loss, lse=on_device(2, 3, dtype=torch.float64)),
        lambda: on.sdl_cross_entropy(logits, t, loss, d_logits=on_device(2, 3, 9)),
        lambda: on.sdl_cross_entropy(logits, t, loss, d_logits=on_device(2, 3, 8, dtype=torch.bfloat16)),
        lambda: on.sdl_cross_entropy(logits, t, loss, d_loss=on_device(6)[::2]),
        lambda: on.sdl_cross_entropy(logits.transpose(1, 2), t, loss),
        lambda: on.sdl_cross_entropy_backward(logits, t, on_device(2, 2), logits),
        lambda: on.sdl_orthogonalize(m, on_device(2, 6, 4), space),
        lambda: on.sdl_orthogonalize(m[0], m, space),
        lambda: on.sdl_orthogonalize(on_device(5), on_device(5), space),
        lambda: on.sdl_orthogonalize(m.transpose(1, 2), m.transpose(1, 2), space),
        lambda: on.sdl_orthogonalize(m, m, space, [(1.0, 2.0)]),
        lambda: on.sdl_orthogonalize(m, m, space, [(1.0, 0.0, 0.0)] * 65),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", k)
    for f in (lambda: on.sdl_orthogonalize(m, m, space, [(3.0, 0.0, 0.0)]), lambda: on.sdl_orthogonalize(m, m, None), lambda: on.sdl_embedding_backward(out, t, table, None),
              lambda: on.sdl_cross_entropy(logits, t, loss, smoothing=2.0), lambda: on.sdl_cross_entropy(logits, t, None)):
        with pytest.raises(sdl.SdlError) as err:
            f()
        assert err.value.status == INVALID
    with pytest.raises(TypeError):
        on.sdl_orthogonalize(m, m, space, 5)
