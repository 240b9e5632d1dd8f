"""What an entry point works out about the buckets asks for no memory, so that nothing is thrown through it; and is exact."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("attn") / "attention_alloc_host.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-fsanitize=bounds", "-fno-sanitize-recover=all", "-Wl,-Bsymbolic", "-o", so,
                           os.path.join(HERE, "emulation", "attention_alloc_host.cpp")])
    return ctypes.CDLL(so)


@pytest.mark.parametrize("side,distance", [(2, 2), (8, 64), (16, 128), (32, 1024), (5, 81), (64, 512), (128, 1024), (256, 1024), (256, 129), (255, 1023)])
def test_borders_without_memory(lib, side, distance):
    e, want, n = side // 2, 0, side // 2
    m = side - e
    for k in range(1, m):
        while n ** m * e ** k < distance ** k * e ** m:
            n += 1
        want += n
    assert lib.attention_borders(side, distance) == want
