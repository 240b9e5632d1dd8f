"""A plan for states of one width is not taken by a step for the other (no GPU)."""
import ctypes

import pytest

import paper_2103_03936_amd as pf

P, Z = ctypes.c_void_p, ctypes.c_size_t


@pytest.mark.parametrize("counts", [(5000,), (1, 4096, 4097), (0,), (1 << 20,) * 40])
def test_widths(counts):
    n = len(counts)
    rec = (pf.pf_adamw_tensor * n)(*(pf.pf_adamw_tensor(256, 512, 768, 1024, 1280, 1536, None, c, 0.0) for c in counts))
    desc = {bits: pf.pf_adamw_desc(n, bits, 0.9, 0.99, 1e-8) for bits in (32, 8)}
    size = {bits: pf.lib.pf_adamw_plan_bytes(ctypes.byref(d), rec) for bits, d in desc.items()}
    host = ctypes.create_string_buffer(max(size.values()))
    for bits, other in ((32, 8), (8, 32)):
        assert pf.lib.pf_adamw_plan_fill(ctypes.byref(desc[bits]), rec, host, Z(size[bits])) == 0
        assert pf.lib.pf_adamw_plan_fill(ctypes.byref(desc[bits]), rec, host, Z(size[bits] - 1)) == 4
        assert pf.lib.pf_adamw_step(ctypes.byref(desc[other]), P(256), Z(size[bits]), P(256), None, P(256), None) == 4
