"""Queries that stand before the first key see nothing under a causal mask: what Q and dO hold there does not matter."""
import pytest
import torch

from test_gpu_attention import _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("buckets", [0, 16])
@pytest.mark.parametrize("c", [(2, 70, 90, 2, 1, 64, [-5, -33]), (2, 150, 130, 2, 2, 128, [-100, -64]), (3, 40, 300, 2, 2, 32, [-40, -1, 3]),
                               (70, 140, 70, 8, 4, 64, [-3 * b for b in range(70)]), (2, 3, 600, 2, 1, 64, [-2, 0])], ids=str)
def test_rows_that_see_nothing_take_no_part(c, buckets, dtype):
    import paper_2103_03936_amd as pf
    start = c[-1]
    _, g, _, kw = _case((*c[:-1], True, buckets, 64, None), dtype, 95)
    kw["q_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")

    def run():
        O_, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
        return (O_, lse, *pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], **kw),
                *pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], need_dtable=False, **kw))

    clean = run()
    for b, s in enumerate(start):
        g["Q"][b, :max(0, -s)] = float("nan")
        g["dO"][b, :max(0, -s)] = float("nan")
    for name, x, y in zip("O lse dQ dK dV dtable dQ dK dV".split(), run(), clean):
        assert (x is None and y is None) or (torch.equal(x, y) and not x.isnan().any()), name
    for b, s in enumerate(start):
        assert not clean[0][b, :max(0, -s)].any() and not clean[2][b, :max(0, -s)].any()
