"""What the operators of the inner step refuse, before anything is launched (CPU only: no refused call touches an address), and the
host-side table of rotary frequencies."""
import ctypes
import math

import pytest
import torch

import paper_2501_18512_amd as sdl

INVALID, UNSUPPORTED, ALIGNMENT, OK = -1, -2, -3, 0
INF, NAN = math.inf, math.nan


def view(data=0x10000, batch=1 << 20, token=1 << 10, head=128):
    return sdl._View(data, batch, token, head)


def call(name, **change):
    """The C entry point with arguments that would be launched, but for `change`."""
    shape = dict(batch=2, tokens=3, heads=4, width=64)
    attention = dict(batch=2, queries=3, keys=5, heads=4, kv_heads=2, width=64, dtype=1, scale=0.1, causal=1, q_len=None, k_len=None)
    good = {
        "sdl_layer_norm": dict(x=view(), **shape, dtype=1, weight=0x20000, bias=0x30000, param_dtype=1, eps=1e-5, y=view(0x40000), mean=0x50000, rstd=0x60000),
        "sdl_layer_norm_backward": dict(dy=view(), x=view(0x20000), **shape, dtype=1, weight=0x30000, param_dtype=1, mean=0x40000, rstd=0x50000,
                                        dx=view(0x60000), dweight=0x70000, dbias=0x80000, workspace=0x90000, workspace_bytes=1 << 24),
        "sdl_rotary": dict(x=view(), **shape, dtype=1, rot=32, layout=0, positions=0x20000, first=0, frequencies=0x30000, scale=1.0, inverse=0, out=view(0x40000)),
        "sdl_attention": dict(q=view(), k=view(0x20000), v=view(0x30000), **attention, out=view(0x40000), lse=0x50000, workspace=0x60000, workspace_bytes=1 << 30),
        "sdl_attention_backward": dict(d_out=view(), q=view(0x20000), k=view(0x30000), v=view(0x40000), out=view(0x50000), lse=0x60000, **attention,
                                       dq=view(0x70000), dk=view(0x80000), dv=view(0x90000), workspace=0xa0000, workspace_bytes=1 << 30),
    }[name]
    if name == "sdl_attention_backward":        # lse stands in front of the shape
        assert list(good)[:6] == ["d_out", "q", "k", "v", "out", "lse"]
    assert set(change) <= set(good)
    return getattr(sdl._lib, name)(*{**good, **change}.values(), None)


NORM = [
    (INVALID, dict(x=None)), (INVALID, dict(x=view(0))), (INVALID, dict(width=0)), (INVALID, dict(dtype=2)), (INVALID, dict(dtype=-1)),
    (INVALID, dict(param_dtype=3)), (UNSUPPORTED, dict(width=16385)), (UNSUPPORTED, dict(batch=1 << 16, tokens=1 << 15)),
    (UNSUPPORTED, dict(batch=1 << 31, tokens=1 << 31, heads=1 << 31)), (ALIGNMENT, dict(x=view(0x10001))), (ALIGNMENT, dict(weight=0x20001)),
    (ALIGNMENT, dict(mean=0x50002)), (ALIGNMENT, dict(rstd=0x60001)), (ALIGNMENT, dict(dtype=0, x=view(0x10002))),
]
ATTENTION = [
    (INVALID, dict(q=None)), (INVALID, dict(k=None)), (INVALID, dict(v=view(0))), (INVALID, dict(out=view(0))), (INVALID, dict(dtype=2)),
    (INVALID, dict(width=0)), (INVALID, dict(heads=3)), (INVALID, dict(kv_heads=0)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)),
    (INVALID, dict(scale=NAN)), (INVALID, dict(scale=INF)), (INVALID, dict(scale=7e-31)), (UNSUPPORTED, dict(width=129)), (UNSUPPORTED, dict(keys=(1 << 30) + 1)),
    (UNSUPPORTED, dict(queries=1 << 31, heads=1 << 30, kv_heads=1)), (UNSUPPORTED, dict(batch=1 << 30, queries=1)), (ALIGNMENT, dict(q=view(0x10001))),
    (ALIGNMENT, dict(v=view(0x10001))), (ALIGNMENT, dict(q_len=0x10002)), (ALIGNMENT, dict(k_len=0x10001)), (ALIGNMENT, dict(lse=0x10002)),
]


@pytest.mark.parametrize("status,change", NORM + [
    (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=NAN)), (INVALID, dict(eps=INF)), (INVALID, dict(y=None)), (INVALID, dict(y=view(0x40000, token=0))),
    (INVALID, dict(y=view(0x40000, batch=0))), (INVALID, dict(y=view(0x40000, head=0))), (ALIGNMENT, dict(bias=0x30001)),
    (ALIGNMENT, dict(y=view(0x40001))), (OK, dict(batch=0)), (OK, dict(tokens=0, x=None, y=None)), (OK, dict(heads=0))])
def test_layer_norm(status, change):
    assert call("sdl_layer_norm", **change) == status


@pytest.mark.parametrize("status,change", NORM + [
    (INVALID, dict(dy=view(0))), (INVALID, dict(dx=None)), (INVALID, dict(mean=None)), (INVALID, dict(rstd=None)), (INVALID, dict(workspace=None)),
    (INVALID, dict(workspace_bytes=1)), (INVALID, dict(dx=view(0x40000, token=0))), (ALIGNMENT, dict(dx=view(0x40001))),
    (ALIGNMENT, dict(dweight=0x10001)), (ALIGNMENT, dict(dbias=0x10001)), (ALIGNMENT, dict(workspace=0x10002)),
    (OK, dict(batch=0, dweight=None, dbias=None))])
def test_layer_norm_backward(status, change):
    assert call("sdl_layer_norm_backward", **change) == status


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=None)), (INVALID, dict(out=view(0))), (INVALID, dict(dtype=5)), (INVALID, dict(layout=2)), (INVALID, dict(rot=31)),
    (INVALID, dict(rot=66)), (INVALID, dict(width=0, rot=0)), (INVALID, dict(scale=NAN)), (INVALID, dict(frequencies=None)),
    (INVALID, dict(out=view(0x40000, token=0))), (INVALID, dict(out=view(0x10000, token=512))), (UNSUPPORTED, dict(width=1025)),
    (UNSUPPORTED, dict(batch=1 << 16, tokens=1 << 16)), (ALIGNMENT, dict(x=view(0x10001))), (ALIGNMENT, dict(out=view(0x10003))),
    (ALIGNMENT, dict(positions=0x10002)), (ALIGNMENT, dict(frequencies=0x10004)), (OK, dict(tokens=0)), (OK, dict(rot=0, frequencies=None, out=view()))])
def test_rotary(status, change):
    assert call("sdl_rotary", **change) == status


@pytest.mark.parametrize("status,change", ATTENTION + [
    (INVALID, dict(out=view(0x40000, token=0))), (ALIGNMENT, dict(workspace=0x10002)), (OK, dict(batch=0)), (OK, dict(queries=0)),
    (OK, dict(heads=0)), (OK, dict(heads=0, kv_heads=0))])
def test_attention(status, change):
    assert call("sdl_attention", **change) == status


def test_attention_that_splits_its_keys_needs_its_workspace():
    few = dict(batch=1, queries=1, keys=4096, heads=1, kv_heads=1)
    need = sdl.sdl_attention_workspace_bytes(1, 1, 4096, 1, 1, 64, sdl.DTYPE_BF16)
    assert need > 0
    assert call("sdl_attention", **few, workspace=None) == INVALID
    assert call("sdl_attention", **few, workspace_bytes=need - 1) == INVALID


@pytest.mark.parametrize("status,change", ATTENTION + [
    (INVALID, dict(d_out=None)), (INVALID, dict(lse=None)), (INVALID, dict(workspace=None)), (INVALID, dict(workspace_bytes=1)),
    (INVALID, dict(dq=view(0))), (INVALID, dict(dk=None)), (INVALID, dict(dv=view(0))), (INVALID, dict(dq=view(0x40000, head=0))),
    (INVALID, dict(dk=view(0x40000, token=0))), (ALIGNMENT, dict(dk=view(0x40001))), (ALIGNMENT, dict(workspace=0x10001)), (OK, dict(batch=0)),
    (OK, dict(queries=0, keys=0))])
def test_attention_backward(status, change):
    assert call("sdl_attention_backward", **change) == status


def test_workspace_sizes_of_what_is_refused_are_nothing():
    assert sdl.sdl_layer_norm_workspace_bytes(16385) == 0
    for f in (sdl.sdl_attention_workspace_bytes, sdl.sdl_attention_backward_workspace_bytes):
        assert f(1, 1, 1 << 20, 2, 2, 64, 1) > 0
        assert f(1, 1, 1 << 20, 3, 2, 64, 1) == 0 and f(1, 1, 1 << 20, 2, 0, 64, 1) == 0 and f(1, 1, 1 << 20, 2, 2, 0, 1) == 0
        assert f(1, 1, 1 << 20, 2, 2, 129, 1) == 0 and f(0, 0, 0, 0, 1, 64, 1) == 0 and f(1, 1, 1 << 20, 2, 2, 64, 2) == 0


class Device(torch.Tensor):
    """A host tensor that says it is on the device, for the checks that come before any address is used."""
    is_cuda = True


def on_device(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


def test_the_binding_refuses_what_is_no_such_tensor():
    x, d = torch.zeros(2, 3, 4, 8), on_device(2, 3, 4, 8)
    for call in (lambda: sdl.sdl_layer_norm(x, None, None, 1e-5, d), lambda: sdl.sdl_layer_norm(d, None, None, 1e-5, x),
                 lambda: sdl.sdl_layer_norm(d, torch.zeros(8), None, 1e-5, d), lambda: sdl.sdl_attention(x, x, x, x),
                 lambda: sdl.sdl_rotary(d, None, torch.zeros(4, dtype=torch.float64), d)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="attention takes"):
        sdl.sdl_attention(d, d[..., :4], d, d)
    with pytest.raises(ValueError, match="attention takes"):
        sdl.sdl_attention(d[0], d[0], d[0], d[0])
    with pytest.raises(ValueError, match="float32 and bfloat16"):
        sdl.sdl_layer_norm(on_device(3, 8, dtype=torch.float16), None, None, 1e-5, on_device(3, 8, dtype=torch.float16))
    with pytest.raises(ValueError, match="float32 and bfloat16"):
        sdl.alloc_attention(d.half(), d)
    for shape in ((), (1, 1, 1, 1, 1)):
        with pytest.raises(ValueError, match="one to four"):
            sdl.sdl_layer_norm(on_device(*shape) if shape else torch.tensor(1.0).as_subclass(Device), None, None, 1e-5, d)
    with pytest.raises(AttributeError):
        sdl.sdl_layer_norm(7, None, None, 1e-5, d)
    with pytest.raises(TypeError):
        sdl.sdl_layer_norm(d, None, None, "small", d)
    with pytest.raises(TypeError):
        sdl._operators.sdl_layer_norm(d)


def test_the_binding_refuses_other_shapes_types_and_strides():
    x, bf = on_device(2, 3, 4, 8), torch.bfloat16
    for y, what in ((on_device(2, 3, 4, 9), "shape"), (on_device(2, 3, 32), "shape"), (on_device(2, 3, 4, 8, dtype=bf), "type"),
                    (on_device(2, 3, 8, 4).transpose(2, 3), "neighbours")):
        with pytest.raises(ValueError, match=what):
            sdl.sdl_layer_norm(x, None, None, 1e-5, y)
    for w, b in ((on_device(7), None), (on_device(8), on_device(8, dtype=bf)), (None, on_device(4, 2, 2)[..., 0])):
        with pytest.raises(ValueError, match="8 elements|contiguous"):
            sdl.sdl_layer_norm(x, w, b, 1e-5, x)
    for change in (dict(mean=on_device(23)), dict(rstd=on_device(24, dtype=bf))):
        with pytest.raises(ValueError, match="24 elements"):
            sdl.sdl_layer_norm(x, None, None, 1e-5, x, **change)
    f = on_device(4, dtype=torch.float64)
    for positions, freq in ((on_device(6), f), (on_device(5, dtype=torch.int32), f), (None, on_device(4))):
        with pytest.raises(ValueError, match="elements of"):
            sdl.sdl_rotary(x, positions, freq, x)
    lens = on_device(2, dtype=torch.int32)
    for args, change in (((x, x, x[:, :2], x), {}), ((x, x.bfloat16(), x, x), {}), ((x, x, x, x[:1]), {}), ((x, x, x, x), dict(q_len=lens[:1])),
                         ((x, x, x, x), dict(k_len=on_device(2))), ((x, x, x, x), dict(lse=on_device(23)))):
        with pytest.raises(ValueError):
            sdl.sdl_attention(*args, **change)
    with pytest.raises(ValueError):
        sdl.sdl_attention_backward(x, x, x, x, x, on_device(24), x, x[:, :2], x, None)


def test_what_arrives_at_the_library():
    """Shapes, addresses and strides of tensors of one to four dimensions, as the C functions get them."""
    seen = {}

    def note(name):
        def f(*args):       # the views lie on the caller's stack
            seen[name] = [(a[0].data, a[0].stride_batch, a[0].stride_token, a[0].stride_head) if isinstance(a, ctypes.POINTER(sdl._View)) else a
                          for a in args]
            return 0
        return ctypes.CFUNCTYPE(ctypes.c_int, *getattr(sdl._lib, name).argtypes)(f)
    names = [n for n in dir(sdl._operators) if n.startswith("sdl_")]
    kept = {n: note(n) for n in names}
    types, hooks = (torch.float32, torch.bfloat16, torch.int32, torch.float64), (sdl._stream, torch.cuda.is_initialized, sdl._get_device, sdl._raw_stream)
    real = {n: ctypes.cast(getattr(sdl._lib, n), ctypes.c_void_p).value for n in names}
    sdl._operators.setup({n: ctypes.cast(f, ctypes.c_void_p).value for n, f in kept.items()}, types, *hooks)
    try:
        big = on_device(2, 5, 9, 16)
        for x, shape, strides in ((big[:, 1:, 2:6, 3:11], (2, 4, 4, 8), (720, 144, 16)), (big[0, :, :, 2:8], (5, 9, 1, 6), (144, 16, 0)),
                                  (big[0, 0], (1, 9, 1, 16), (0, 16, 0)), (big[0, 0, 0], (1, 1, 1, 16), (0, 0, 0)),
                                  (big.transpose(1, 2), (2, 9, 5, 16), (720, 16, 144))):
            sdl.sdl_layer_norm(x, None, None, 1e-5, x, stream=7)
            a = seen["sdl_layer_norm"]
            assert a[0] == (x.data_ptr(), *strides) and tuple(a[1:5]) == shape and a[5] == sdl.DTYPE_FP32 and a[10] == a[0] and a[13] == 7
        q, k, lse = on_device(2, 3, 4, 8, dtype=torch.bfloat16), on_device(2, 6, 2, 8, dtype=torch.bfloat16), on_device(2, 4, 3)
        lens, work = on_device(2, dtype=torch.int32), on_device(100)
        sdl.sdl_attention(q, k, k, q, lse, work, causal=True, k_len=lens, stream=9)
        a = seen["sdl_attention"]
        assert tuple(a[3:9]) == (2, 3, 6, 4, 2, 8) and a[9] == sdl.DTYPE_BF16 and abs(a[10] - 8 ** -0.5) < 1e-7 and a[11] == 1 and a[12] is None
        assert a[13] == lens.data_ptr() and a[15] == lse.data_ptr() and a[16] == work.data_ptr() and a[17] == 400 and a[18] == 9
        sdl.sdl_attention_backward(q, q, k, k, q, lse, q, k, k, work, 0.5, q_len=lens, stream=9)
        a = seen["sdl_attention_backward"]
        assert a[5] == lse.data_ptr() and tuple(a[6:12]) == (2, 3, 6, 4, 2, 8) and a[13] == 0.5 and a[14] == 0 and a[15] == lens.data_ptr() and a[16] is None
        assert a[18][0] == k.data_ptr() and a[20] == work.data_ptr() and a[21] == 400
        f = on_device(4, dtype=torch.float64)
        sdl.sdl_rotary(q, None, f, q, sdl.ROTARY_INTERLEAVED, 1.5, True, 77, stream=9)
        a = seen["sdl_rotary"]
        assert tuple(a[1:6]) == (2, 3, 4, 8, sdl.DTYPE_BF16) and tuple(a[6:8]) == (8, 1) and a[8] is None and a[9] == 77 and a[10] == f.data_ptr() and a[11] == 1.5 and a[12] == 1
        w, m = on_device(8, dtype=torch.bfloat16), on_device(2, 3, 4)
        x = on_device(2, 3, 4, 8)
        sdl.sdl_layer_norm_backward(x, x, w, m, m, x, w, None, work, stream=9)
        a = seen["sdl_layer_norm_backward"]
        assert tuple(a[2:7]) == (2, 3, 4, 8, 0) and a[7] == w.data_ptr() and a[8] == 1 and a[9] == a[10] == m.data_ptr() and a[12] == w.data_ptr() and a[13] is None
        assert a[14] == work.data_ptr() and a[15] == 400
    finally:
        sdl._operators.setup(real, types, *hooks)


def test_frequencies():
    assert sdl.sdl_rotary_frequencies(8).tolist() == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-15)
    assert sdl.sdl_rotary_frequencies(4, 100.0, sdl.ROTARY_LINEAR, 4.0).tolist() == pytest.approx([0.25, 0.025], rel=1e-15)
    # trained on 2 pi 100 positions (rounded): pairs that turn 100, 10, 1 and 0.1 times; 10 and more stay, 1 and less are stretched 8 times
    length = 628
    f = sdl.sdl_rotary_frequencies(8, 1e4, sdl.ROTARY_PARTS, 8.0, 1.0, 10.0, length)
    turns = [length * w / (2 * math.pi) for w in (1.0, 0.1, 0.01, 0.001)]
    keep = [min(1.0, max(0.0, (n - 1.0) / 9.0)) for n in turns]
    assert keep[0] == 1.0 and keep[3] == 0.0 and 0.9 < keep[1] < 1.0
    assert f.tolist() == pytest.approx([w * (k + (1 - k) / 8.0) for w, k in zip((1.0, 0.1, 0.01, 0.001), keep)], rel=1e-12)


@pytest.mark.parametrize("args", [(0,), (7,), (1026,), (8, 0.0), (8, -1.0), (8, NAN), (8, INF), (8, 1e4, 3), (8, 1e4, -1), (8, 1e4, 1, 0.0),
                                  (8, 1e4, 1, NAN), (8, 1e4, 2, 8.0, 4.0, 4.0, 100), (8, 1e4, 2, 8.0, -1.0, 4.0, 100), (8, 1e4, 2, 8.0, 1.0, INF, 100),
                                  (8, 1e4, 2, 8.0, 1.0, 4.0, 0)])
def test_frequencies_that_are_refused(args):
    with pytest.raises(sdl.SdlError):
        sdl.sdl_rotary_frequencies(*args)


def test_frequencies_need_a_place():
    assert sdl._lib.sdl_rotary_frequencies(8, 1e4, 0, 1.0, 1.0, 4.0, 0, ctypes.c_void_p()) == INVALID
