"""Whether two tensors with strides have an element in common, against sets of their elements."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("overlap") / "overlap_host.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-o", so, os.path.join(HERE, "emulation", "overlap_host.cpp")])
    lib = ctypes.CDLL(so)
    return lambda a, b: bool(lib.overlap_meet((ctypes.c_int64 * 8)(*a), (ctypes.c_int64 * 8)(*b)))


def _elements(t):
    at, *size = t[:4]
    s, D = t[4:7], t[7]
    return {at + sum(i * k for i, k in zip(x, s)) + e for x in itertools.product(*map(range, size)) for e in range(D)}


def _tensor(rng):
    """Slices, parts and permutations of buffers, and strides of no order at all."""
    size = [rng.randint(0 if rng.random() < 0.05 else 1, 4) for _ in range(3)]
    D = rng.randint(1, 5)
    if rng.random() < 0.3:
        s = [rng.randint(0, 30) for _ in range(3)]
    else:
        order, s, step = rng.sample(range(3), 3), [0] * 3, D
        for i in order:
            step += rng.choice([0, 0, 1, 4])
            s[i] = step
            step *= size[i] + rng.choice([0, 0, 1])
            if step == 0:
                step = D
        if rng.random() < 0.2:
            s[rng.randrange(3)] = 0
    return [rng.randint(0, 60), *size, *s, D]


def test_against_sets(meet):
    rng, seen = random.Random(5), [0, 0]
    for _ in range(20000):
        a = _tensor(rng)
        b = _tensor(rng)
        if rng.random() < 0.5:  # another slice of the same buffer
            b[4:7] = a[4:7]
        want = bool(_elements(a) & _elements(b))
        assert meet(a, b) == want == meet(b, a), (a, b)
        seen[want] += 1
    assert min(seen) > 3000


def test_slices_of_a_fused_projection(meet):
    B, L, H, D = 64, 4096, 8, 128
    s = [L * 3 * H * D, 3 * H * D, D]
    q, k = [0, B, L, H, *s, D], [H * D, B, L, H, *s, D]
    assert not meet(q, k) and meet(q, [D, *k[1:]]) and meet(k, [2 * H * D - 1, *k[1:]]) and not meet(k, [2 * H * D, *k[1:]])
    cache = [0, B, L, H, H * L * D, D, L * D, D]  # heads before tokens
    assert meet(cache, [5 * L * D, *cache[1:]]) and not meet([0, B, L // 2, *cache[3:]], [L // 2 * D, B, L // 2, *cache[3:]])
