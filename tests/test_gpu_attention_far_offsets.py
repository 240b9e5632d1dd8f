"""A cache so large that the second sequence's keys lie more than 2^32 elements behind the first one's."""
import pytest
import torch

from test_gpu_attention import _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", [(2, 1, 600, 4, 2, 64, True, 32, 128, "append"), (2, 70, 90, 2, 1, 64, False, 32, 128, "pad")], ids=str)
def test_strides_past_32_bits(c):
    import paper_2103_03936_amd as pf
    d, g, _, kw = _case(c, "bf16", 97)
    (B, Lk, hk, D), far = g["K"].shape, (1 << 32) + 64
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("two tensors of 8.6 GB")
    K, V = (torch.empty(far + Lk * hk * D, dtype=torch.bfloat16, device="cuda").as_strided((B, Lk, hk, D), (far, hk * D, D, 1)) for _ in range(2))
    K.copy_(g["K"])
    V.copy_(g["V"])
    want = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    got = pf.pf_attention_fwd(g["Q"], K, V, g["table"], **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x, y in zip(pf.pf_attention_bwd(g["Q"], K, V, *got, g["dO"], g["table"], **kw),
                    pf.pf_attention_bwd(g["Q"], g["K"], g["V"], *want, g["dO"], g["table"], **kw)):
        assert torch.equal(x, y)
    # rotated keys go there, too
    out = pf.pf_qk_norm_rotate_fwd(g["K"], None)[0]
    assert torch.equal(pf.pf_qk_norm_rotate_fwd(g["K"], None, out=(K, None))[0], out)
