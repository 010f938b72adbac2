"""Clipping reads the gradients a second time while it writes its results: what it writes may share memory with nothing that it reads, but a result with its own
gradient, in place.  Refused in host code: nothing here touches a device."""
import ctypes
import itertools
import random

import pytest

from test_layer_refusals import lib, refused  # noqa: F401

P = ctypes.c_void_p
NORM, WS = P(1 << 30), P(1 << 31)


def clip(lib, grads, outs, sizes, dtype=0, norm=NORM):
    n = len(sizes)
    arr = lambda a: None if a is None else (ctypes.c_void_p * n)(*a)
    return lib.tma_grad_clip(n, arr(grads), arr(outs), (ctypes.c_int64 * n)(*sizes), dtype, 1.0, norm, WS, 1 << 30, None)


CASES = {
    "a permuted list": ([4096, 8192], [8192, 4096], [100, 100]),
    "a result on the next gradient": ([4096, 8192], [16384, 4096], [100, 100]),
    "shifted by one value": ([4096], [4100], [100]),
    "shifted back": ([4100], [4096], [100]),
    "the last value on the first of another": ([4096, 8192], [1 << 20, 4096 + 396], [100, 100]),
    "in place and on another": ([4096, 4096 + 400, 1 << 20], [4096, 1 << 21, 4096 + 400], [100, 100, 100]),
    "a gradient given twice, one in place": ([4096, 4096], [4096, 8192], [100, 100]),
    "a flat buffer shifted against the gradients'": ([4096 + 400 * k for k in range(300)], [4096 + 400 * k + 200 for k in range(300)], [100] * 300),
    "gradients in one result's middle": ([4096, 1 << 20], [8192, 4096 - 2000], [100, 1000]),
}


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("case", CASES.values(), ids=CASES)
def test_results_on_gradients(lib, case, dtype):
    grads, outs, sizes = case
    refused(lib, clip(lib, grads, outs, [s * (2 if dtype else 1) for s in sizes], dtype), -1, b"overlap")


@pytest.mark.parametrize("at", [4096, 4096 + 396, 1 << 20, (1 << 20) + 396])
def test_the_norm_on_what_is_read_or_written(lib, at):
    refused(lib, clip(lib, [4096], [1 << 20], [100], norm=P(at)), -1, b"norm_out")
    if at < 1 << 20:
        refused(lib, clip(lib, [4096], None, [100], norm=P(at)), -1, b"norm_out")


def apart(grads, outs, sizes, size):
    """By comparing everything with everything."""
    span = lambda p, s: range(p, p + s * size)
    meet = lambda a, b: len(a) and len(b) and a.start < b.stop and b.start < a.stop
    for i, j in itertools.product(range(len(sizes)), repeat=2):
        if i != j and meet(span(outs[i], sizes[i]), span(outs[j], sizes[j])):
            return False
        if (i != j or outs[i] != grads[j]) and meet(span(outs[i], sizes[i]), span(grads[j], sizes[j])):
            return False
    return True


def test_lists_drawn_at_random(lib):
    """Every list that has an overlap is refused.  (One that has none would be launched: those are not called here.)"""
    rng, refusals = random.Random(3), 0
    for _ in range(3000):
        n = rng.randint(1, 6)
        sizes = [rng.choice([0, 1, 2, 3, 5]) for _ in range(n)]
        grads = [4096 + 4 * rng.randint(0, 40) for _ in range(n)]
        outs = [g if rng.random() < 0.4 else 4096 + 4 * rng.randint(0, 40) for g in grads]
        if not apart(grads, outs, sizes, 4):
            refused(lib, clip(lib, grads, outs, sizes), -1, b"overlap")
            refusals += 1
    assert refusals > 500
