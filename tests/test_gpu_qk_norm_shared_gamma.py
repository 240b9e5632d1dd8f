"""Queries and keys with one weight for their norms: both gradients go into one tensor."""
import numpy as np
import pytest
import torch

from operator_bounds import E, assert_within
from test_gpu_qk_norm import _inputs
from parity import to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", [("bf16", 3, 37, 8, 2, 64, 64, "halves", "rms", True), ("f32", 1, 3000, 2, 1, 16, 16, "pairs", "rms", True),
                               ("f32", 1, 1, 1, 1, 256, 0, "halves", "rms", True)], ids=str)
def test_one_gradient_for_both(c):
    import paper_2103_03936_amd as pf
    dtype, rot, style = c[0], c[6], c[7]
    d, _ = _inputs(c, 13, 0)
    g = {k: to_gpu(v, "f32" if k[0] == "g" else dtype) for k, v in d.items()}
    call = lambda **kw: pf.pf_qk_norm_rotate_bwd(g["Q"], g["K"], g["dQ"], g["dK"], g["gq"], g["gq"], rot_dim=rot, style=style, **kw)  # noqa: E731
    dQ, dK, dq, dk = call()
    for start in (0.0, 1.0):
        both = torch.full_like(dq, start)
        got = call(grads=(both, both))
        assert got[2] is both and got[3] is both and torch.equal(got[0], dQ) and torch.equal(got[1], dK)
        x, y = dq.double().cpu().numpy(), dk.double().cpu().numpy()  # (each rounded once; their sum once, and once more with what was there)
        assert_within(both, start + x + y, E * (np.abs(x) + np.abs(y) + np.abs(x + y) + np.abs(start + x + y)) * 1.001, "dgamma")
        assert all(torch.equal(a, b) for a, b in zip(call(grads=(torch.full_like(dq, start),) * 2), got))
