"""Random calls of the extension module of csrc/sdl_training.c: training_fuzz.py <extension> <library of stand-ins>."""
import ctypes, importlib.util, random, sys
spec = importlib.util.spec_from_file_location("_training", sys.argv[1])
mod = importlib.util.module_from_spec(spec)
spec.loader.exec_module(mod)
lib = ctypes.CDLL(sys.argv[2])
names = [n for n in dir(mod) if n.startswith("sdl_")]
F32, BF16, I32, I64 = "float32", "bfloat16", "int32", "int64"
rng = random.Random(1)
device = lambda: rng.choice([0, 0, 0, 1, None])
mod.setup({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names}, (F32, BF16, I32, I64), lambda s: 0 if s is None else s,
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
                        lambda: setattr(self, "dtype", rng.choice([F32, BF16, I32, I64, "float64", None, 5, object()])),
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
class Changing(list):
    """A list that loses its members while they are read."""
    def __init__(self, *a):
        super().__init__(*a)
        outer = self
        class Number:
            def __float__(self):
                outer.clear()
                return 0.5
        if self: self[0] = (Number(), 0.0, 0.0)

for turn in range(6000):
    easy = turn % 2 == 0
    dims = rng.randint(1, 3)
    B, L, W, V = (rng.randint(1, 4) for _ in range(4))
    x = (B, L, W)[3 - dims:]
    places = x[:-1] or (1,)
    T, P, I = rng.choice([F32, BF16]), rng.choice([F32, BF16]), rng.choice([I32, I64])
    def tensor(shape, dtype, none=False):
        if none and rng.random() < 0.3: return None
        if not easy and rng.random() < 0.1: return rng.choice([None, 5, "x", object()])
        return Tensor(shape, dtype, not easy and rng.random() < 0.15)
    number = lambda v: v if easy or rng.random() < 0.9 else rng.choice([None, "x", 2 ** 70, 10 ** 400, -1, float("nan"), Index()])
    triples = [(1.5, -0.5, 0.0)] * rng.choice([0, 1, 5, 64])
    coefficients = triples if easy or rng.random() < 0.7 else rng.choice([None, 5, [(1.0, 2.0)], [(1.0, 2.0, "x")], [None], triples + [5], [(1.0, 2.0, 3.0)] * 65, iter(triples), "abc",
                                                                          ["abc"], Changing(triples), (Index(),), [[1, 2, 3]]])
    stream = rng.choice([None, 0, 5])
    m = (B, L, W)[rng.randint(0, 1):]
    todo = {
        "sdl_embedding": lambda: [tensor((V, W), P), tensor(places, I), tensor(x, T), number(1.0), stream],
        "sdl_embedding_backward": lambda: [tensor(x, T), tensor(places, I), tensor((V, W), P), tensor((64,), F32, True), number(1.0), stream],
        "sdl_cross_entropy": lambda: [tensor(x, T), tensor(places, I), tensor(places, F32, True), tensor(places, F32, True), tensor(x, T, True), tensor(places, F32, True),
                                      number(0.1), number(1e-4), stream],
        "sdl_cross_entropy_backward": lambda: [tensor(x, T), tensor(places, I), tensor(places, F32), tensor(x, T), tensor(places, F32, True), number(0.1), number(0.0), stream],
        "sdl_orthogonalize": lambda: [tensor(m, T), tensor(m, P), tensor((64,), F32, True), coefficients, number(1e-7), number(1.0), stream],
    }
    assert sorted(todo) == names
    for name, make in todo.items():
        args = make()
        if not easy and rng.random() < 0.02: args.pop()
        try:
            assert getattr(mod, name)(*args) in (0, 1)
            calls += 1
        except (TypeError, AttributeError, ValueError, OverflowError, ZeroDivisionError):
            refused += 1
print("calls", calls, "refused", refused)
