"""Numbers that an int does not hold are refused, not taken modulo 2^32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_too_large():
    import paper_2103_03936_amd as pf
    q, t = torch.zeros(1, 2, 2, 16, device="cuda"), torch.zeros(8, 2, device="cuda")
    for wrap in (1 << 32, -(1 << 32), 1 << 40):
        with pytest.raises(OverflowError):
            pf.pf_qk_norm_rotate_fwd(q, None, rot_dim=wrap + 8)
        with pytest.raises(OverflowError):
            pf.pf_attention_fwd(q, q, q, t, max_distance=wrap + 128)
    pf.pf_qk_norm_rotate_fwd(q, None, rot_dim=8)
    pf.pf_attention_fwd(q, q, q, t, max_distance=128)
