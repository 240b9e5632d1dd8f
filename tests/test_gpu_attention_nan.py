"""A NaN among what a query uses is in that query's results, however its keys were split between workgroups."""
import numpy as np
import pytest
import torch

from test_gpu_attention import _case

pytestmark = pytest.mark.gpu


def _same_but(got, clean, rows, heads, scores=True):
    """Results O, and lse if the scores are what has the NaN, of `rows` = [(sequence, query)] in `heads` are NaN, all others as
    they were."""
    (O_, lse), (O0, lse0) = got, clean
    other = torch.ones(lse.shape, dtype=torch.bool, device="cuda")
    for b, i in rows:
        for h in heads:
            assert O_[b, i, h].isnan().all() and (lse[b, h, i].isnan() if scores else lse[b, h, i] == lse0[b, h, i]), (b, i, h)
            other[b, h, i] = False
    assert torch.equal(O_.transpose(1, 2)[other], O0.transpose(1, 2)[other]) and torch.equal(lse[other], lse0[other])


# B, Lq, Lk, heads_q, heads_kv, D: several parts of 256 keys or more, all of them whole blocks of 32
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("c", [(2, 1, 512, 2, 1, 64), (1, 1, 4096, 4, 2, 128), (2, 3, 1024, 2, 2, 40), (1, 64, 4096, 1, 1, 64)], ids=str)
def test_nan_query_over_several_parts(c, buckets, causal, dtype):
    import paper_2103_03936_amd as pf
    B, Lq, Lk = c[:3]
    _, g, _, kw = _case((*c, causal, buckets, 128, None), dtype, 91)
    if causal:
        kw["q_start"] = torch.full((B,), Lk - Lq, dtype=torch.int32, device="cuda")
    clean = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    assert not clean[0].isnan().any()
    g["Q"][B - 1, Lq - 1, 0, 5] = float("nan")
    got = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    _same_but(got, clean, [(B - 1, Lq - 1)], [0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["K", "V"])
@pytest.mark.parametrize("part", [0, 1, 3])
def test_a_part_of_nothing_but_nan(part, what, dtype):
    """1024 keys are four parts of 256: one whose keys, or values, are all NaN is not taken for an empty one."""
    import paper_2103_03936_amd as pf
    _, g, _, kw = _case((2, 1, 1024, 4, 2, 64, False, 32, 128, None), dtype, 93)
    clean = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    g[what][1, 256 * part:256 * (part + 1), 1] = float("nan")  # the second key head: query heads 2 and 3
    _same_but(pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw), clean, [(1, 0)], [2, 3],
              scores=what == "K")
    # behind the sequence's keys it does not matter
    kw["kv_len"] = torch.tensor([1024, 256 * part], dtype=torch.int32, device="cuda")
    got = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    want = pf.pf_attention_fwd(g["Q"], torch.nan_to_num(g["K"]), torch.nan_to_num(g["V"]), g["table"], **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0].isnan().any()
