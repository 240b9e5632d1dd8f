"""The borders of the relative position buckets, as the library's host code works them out, against exact arithmetic."""
import ctypes
import os
import subprocess

import pytest

from oracle import operators as O

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("attn") / "attention_host.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", so,
                           os.path.join(HERE, "emulation", "attention_host.cpp")])
    return ctypes.CDLL(so)


@pytest.mark.parametrize("side,distance", [(2, 2), (2, 3), (3, 16), (4, 16), (8, 64), (16, 128), (16, 250), (32, 128), (32, 1024),
                                           (5, 81), (6, 24), (7, 1024), (64, 512), (128, 65), (128, 1000), (256, 1024)])
def test_buckets(lib, side, distance):
    far = lib.attention_far(side, distance)
    assert 0 < far <= distance
    for n in list(range(0, min(distance, 200))) + [distance - 1, distance, distance + 1, 1024, 5000]:
        assert lib.attention_bucket(side, distance, n) == O.bucket(-n, side, distance, False), n
    assert lib.attention_bucket(side, distance, far) == side - 1 == lib.attention_bucket(side, distance, 1 << 20)
    assert lib.attention_bucket(side, distance, far - 1) < side - 1
