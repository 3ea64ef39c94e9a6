"""Random calls of the extension module of csrc/sdl_operators.c: operators_fuzz.py <extension> <library of stand-ins>."""
import ctypes, importlib.util, random, sys
spec = importlib.util.spec_from_file_location("_operators", sys.argv[1])
m = importlib.util.module_from_spec(spec)
spec.loader.exec_module(m)
lib = ctypes.CDLL(sys.argv[2])
names = [n for n in dir(m) if n.startswith("sdl_")]
F32, BF16, I32, F64 = "float32", "bfloat16", "int32", "float64"
rng = random.Random(1)
device = lambda: rng.choice([0, 0, 0, 1, None])
m.setup({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names}, (F32, BF16, I32, F64), lambda s: 0 if s is None else s,
        lambda: rng.random() < 0.8, device, lambda d: rng.choice([5, 2 ** 64 - 1]) if d is not None else 1 // 0)

class Index:
    def __index__(self): return 3

class Tensor:
    is_cuda = True
    def __init__(self, shape, dtype, odd=False):
        self.dtype, self.shape = dtype, tuple(shape)
        step, strides = 1, []
        for n in reversed(self.shape):
            strides.insert(0, step)
            step *= n
        self.strides, self.at, self.n = tuple(strides), 64, step
        if odd:
            rng.choice([lambda: setattr(self, "shape", rng.choice([(), (1,) * 5, [2, 2], 5, None, (2 ** 32, 4), (-1, 4), ("x", 4), (Index(), 4), (2 ** 70,)])),
                        lambda: setattr(self, "strides", rng.choice([(), (1,) * 5, [2, 2], 5, None, (2 ** 63 - 1,) * 4, (-2 ** 63,) * 4, (2 ** 70,) * 4, ("x",) * 4])),
                        lambda: setattr(self, "dtype", rng.choice([F32, BF16, I32, F64, None, 5, object()])),
                        lambda: setattr(self, "at", rng.choice([0, -1, 2 ** 64 - 1, 2 ** 70, "x", None, 0.5])),
                        lambda: setattr(self, "n", rng.choice([0, -1, 2 ** 63 - 1, 2 ** 70, None])),
                        lambda: setattr(self, "is_cuda", rng.choice([False, 0, [], None])),
                        lambda: self.__dict__.__delitem__(rng.choice(["shape", "dtype"])),
                        lambda: setattr(self, "strides", (2,) * len(self.shape))])()
    def stride(self): return self.strides
    def data_ptr(self): return self.at
    def numel(self): return self.n
    def element_size(self): return rng.choice([1, 2, 4, -1, 2 ** 62]) if rng.random() < 0.1 else 4
    def is_contiguous(self): return rng.random() < 0.98

calls = refused = 0
for turn in range(6000):
    easy = turn % 2 == 0
    dims = rng.randint(1, 4)
    B, L, H, W, G, K = (rng.randint(1, 4) for _ in range(6))
    x = (B, L, H, W)[4 - dims:] if dims != 3 else (B, L, W)
    if dims == 2: x = (L, W)
    rows = 1
    for n in x[:-1]: rows *= n
    b, t = ({4: (B, L), 3: (B, L), 2: (1, L), 1: (1, 1)})[dims]
    T, P = rng.choice([F32, BF16]), rng.choice([F32, BF16])
    def tensor(shape, dtype, none=False):
        if none and rng.random() < 0.3: return None
        if not easy and rng.random() < 0.1: return rng.choice([None, 5, "x", object()])
        return Tensor(shape, dtype, not easy and rng.random() < 0.15)
    number = lambda v: v if easy or rng.random() < 0.9 else rng.choice([None, "x", 2 ** 70, 10 ** 400, -1, float("nan"), Index()])
    stream = rng.choice([None, 0, 5])
    q, kv = (B, L, H, W), (B, K, G, W)
    lens = lambda: tensor((B,), I32, True)
    todo = {
        "sdl_layer_norm": lambda: [tensor(x, T), tensor((W,), P, True), tensor((W,), P, True), number(1e-5), tensor(x, T), tensor((rows,), F32, True),
                                   tensor((rows,), F32, True), stream],
        "sdl_layer_norm_backward": lambda: [tensor(x, T), tensor(x, T), tensor((W,), P, True), tensor((rows,), F32), tensor((rows,), F32), tensor(x, T),
                                            tensor((W,), P, True), tensor((W,), P, True), tensor((64,), F32, True), stream],
        "sdl_rotary": lambda: [tensor(x, T), tensor((b, t), I32, True), tensor((W // 2,), F64), tensor(x, T), number(0), number(1.0), number(False), number(0), stream],
        "sdl_attention": lambda: [tensor(q, T), tensor(kv, T), tensor(kv, T), tensor(q, T), tensor((B, H, L), F32, True), tensor((64,), F32, True), number(0.5),
                                  number(True), lens(), lens(), stream],
        "sdl_attention_backward": lambda: [tensor(q, T), tensor(q, T), tensor(kv, T), tensor(kv, T), tensor(q, T), tensor((B, H, L), F32), tensor(q, T),
                                           tensor(kv, T), tensor(kv, T), tensor((64,), F32), number(0.5), number(True), lens(), lens(), stream],
    }
    assert sorted(todo) == names
    for name, make in todo.items():
        args = make()
        if not easy and rng.random() < 0.02: args.pop()
        try:
            assert getattr(m, name)(*args) in (0, 1)
            calls += 1
        except (TypeError, AttributeError, ValueError, OverflowError, ZeroDivisionError):
            refused += 1
print("calls", calls, "refused", refused)
