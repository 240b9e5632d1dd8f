"""Keys and values off the alignment that the kernels load with, beside queries that are on it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["K", "V", "KV"])
def test_misaligned_keys_and_values(which):
    import paper_2103_03936_amd as pf
    q = torch.zeros(2, 4, 4, 8, device="cuda")
    k = torch.zeros(2, 6, 2, 16, device="cuda")
    off, on = k[..., 1:9], k[..., 8:]
    K, V = (off if "K" in which else on), (off if "V" in which else on)
    pf.pf_attention_fwd(q, on, on)
    with pytest.raises(pf.PfError):
        pf.pf_attention_fwd(q, K, V)
    O_, lse = pf.pf_attention_fwd(q, on, on)
    with pytest.raises(pf.PfError):
        pf.pf_attention_bwd(q, K, V, O_, lse, O_)
    narrow = torch.zeros(2, 6, 2 * 10, device="cuda").as_strided((2, 6, 2, 8), (120, 20, 10, 1))  # heads 40 bytes apart
    with pytest.raises(pf.PfError):
        pf.pf_attention_fwd(q, *(narrow if c in which else on for c in "KV"))
