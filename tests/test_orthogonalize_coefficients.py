"""Which polynomials sdl_orthogonalize takes, against the largest value of each as it is found by looking at many points (CPU only: nothing is launched)."""
import random

import torch

from test_training_refusals import INVALID, OK, call, numbers


def reach(steps):
    """The largest |p(s)| of the last polynomial where s is as far as the ones before it have gone; infinity once one has gone beyond 2."""
    h = 1.0
    for a, b, c in steps:
        s = torch.linspace(0.0, h, 20001, dtype=torch.float64)
        h = float((a * s + b * s ** 3 + c * s ** 5).abs().max())
        if h > 2.001:
            return h
    return h


def taken(steps):
    # as the call gets them, in fp32
    steps = [tuple(float(torch.tensor(x)) for x in s) for s in steps]
    return reach(steps), call("sdl_orthogonalize", batch=0, coefficients=numbers(*[x for s in steps for x in s]), steps=len(steps))


def test_a_last_coefficient_that_is_next_to_nothing():
    """8 s - 8 s^3 is 3.08 at its largest, and so it is with 1e-20 s^5 beside it; the zeros of its derivative lie nowhere else then."""
    for c in (0.0, 1e-6, -1e-6, 1e-12, -1e-12, 1e-15, 1e-16, -1e-16, 1e-17, 1e-20, -1e-20, 1e-30, 1e-45):
        for sign in (1.0, -1.0):
            most, status = taken([(sign * 8.0, sign * -8.0, c)])
            assert most > 3.0 and status == INVALID, (sign, c)
            most, status = taken([(sign * 5.0, sign * -5.0, c)])
            assert most < 1.95 and status == OK, (sign, c)
            # the step after it starts where this one ends: at 1.92 and not at 0
            most, status = taken([(sign * 5.0, sign * -5.0, c), (1.5, 0.0, 0.0)])
            assert most > 2.8 and status == INVALID, (sign, c)


def test_a_first_coefficient_that_is_next_to_nothing():
    for a in (0.0, 1e-12, -1e-12, 1e-17, -1e-17, 1e-30):
        most, status = taken([(a, 20.0, -20.0)])            # s^3 - s^5 is 0.186 at its largest
        assert most > 3.5 and status == INVALID, a
        most, status = taken([(a, 10.0, -10.0)])
        assert most < 1.9 and status == OK, a


def test_coefficients_of_all_sizes():
    rng = random.Random(1)
    seen = {OK: 0, INVALID: 0}
    for turn in range(3000):
        size = lambda: rng.choice([-1.0, 1.0]) * (rng.uniform(0.0, 8.0) if rng.random() < 0.7 else 10.0 ** rng.uniform(-30.0, 1.0))  # noqa: E731
        steps = [(size(), size(), rng.choice([0.0, size()])) for _ in range(rng.randint(1, 2))]
        most, status = taken(steps)
        if abs(most - 2.0) < 2e-3:      # as near as looking tells
            continue
        assert status == (OK if most <= 2.0 else INVALID), (steps, most)
        seen[status] += 1
    assert min(seen.values()) > 300, seen
