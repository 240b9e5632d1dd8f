"""Calls of more workgroups than a launch may have are refused before anything is launched (no GPU)."""
import ctypes

import pytest

import paper_2103_03936_amd as pf

P, Z = ctypes.c_void_p, ctypes.c_size_t
FAKE = [P((i + 1) << 50) for i in range(12)]  # far apart; never dereferenced


def _desc(B, Lq, Lk, heads, causal=0, D=8):
    return ctypes.byref(pf.pf_attention_desc(B, Lq, Lk, heads, heads, D, causal, 0, 0, 0, pf.PF_BF16, 1.0))


@pytest.mark.parametrize("case", [(1 << 20, 40, 40, 16), (1 << 24, 33, 0, 1), (1 << 25, 1, 1, 1), (1 << 18, 8200, 20, 1), (1 << 23, 300, 4, 1, 1)], ids=str)
def test_forward(case):
    d = _desc(*case)
    q, k, v, o, lse, ws = FAKE[:6]
    assert pf.lib.pf_attention_fwd(d, q, k, v, None, None, None, None, o, lse, ws, Z(1 << 45), None) == 3


@pytest.mark.parametrize("case", [(1 << 20, 40, 40, 16), (1 << 22, 2, 500, 1, 1), (1 << 23, 2, 200, 1), (1 << 24, 0, 2, 1), (1 << 24, 2, 2, 1, 0, 128)], ids=str)
def test_backward(case):
    d = _desc(*case)
    assert pf.lib.pf_attention_bwd(d, *FAKE[:3], None, None, None, None, *FAKE[3:9], None, 0, FAKE[9], Z(1 << 45), None) == 3
