"""Attention whose two lengths differ much, in training; lengths and positions out of their range; calls of two threads at once."""
import threading

import numpy as np
import pytest
import torch

from operator_bounds import assert_within, attention_bounds
from oracle import operators as O
from test_gpu_attention import _case, test_against_definition as against_definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(1, 4096, 77, 4, 2, 64, False, 32, 128, None), (2, 16, 4096, 4, 1, 128, False, 32, 128, "pad"),
                               (1, 2100, 2100, 2, 1, 64, True, 32, 128, None), (1, 4096, 5, 1, 1, 40, False, 0, 0, None),
                               (1, 1500, 3000, 1, 1, 96, True, 16, 64, "append")], ids=str)
def test_long_and_short(c, dtype):
    against_definition(c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq", [1, 70])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_and_positions_are_taken_as_within_their_range(causal, Lq, dtype):
    import paper_2103_03936_amd as pf
    B, Lk = 6, 600
    d, g, _, kw = _case((B, Lq, Lk, 2, 1, 64, causal, 16, 64, None), dtype, 99)
    big = 2 ** 31 - 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    wild = dict(q_len=i32([-1, big, Lq, -big, big, Lq]), kv_len=i32([big, -7, Lk, big, Lk + 1, Lk]), q_start=i32([0, 5, big, 3, -big - 1, 590]))
    tame = dict(q_len=i32([0, Lq, Lq, 0, Lq, Lq]), kv_len=i32([Lk, 0, Lk, Lk, Lk, Lk]), q_start=i32([0, 5, 1 << 30, 3, -(1 << 30), 590]))
    out = []
    for lens in (wild, tame):
        O_, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw, **lens)
        out.append((O_, lse, *pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], **kw, **lens)))
    for x, y in zip(*out):
        assert torch.equal(x, y) and not x.isnan().any()
    near = {k: v.cpu().numpy() for k, v in tame.items()}
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), d["table"].astype(np.float64), causal=causal, max_distance=64,
                    bidirectional=not causal, **near)
    dO = d["dO"].astype(np.float64)
    bounds = attention_bounds(o, dO, dtype)
    for name, x, y, b in zip("O lse dQ dK dV dtable".split(), out[0], (o.O, o.lse, *o.backward(dO)), bounds):
        assert_within(x, y, b, name)


def test_two_threads_at_once():
    """Each on a stream of its own, with other biases and sizes: what a thread keeps of its last call is its own."""
    import paper_2103_03936_amd as pf
    work = [_case(c, "bf16", 55)[1::2] for c in [(2, 70, 70, 4, 2, 64, True, 32, 128, None), (1, 900, 900, 4, 2, 64, False, 16, 100, None)]]
    got = [[], []]

    def run(i):
        g, kw = work[i]
        Qo, Ko = pf.pf_qk_norm_rotate_fwd(g["Q"], g["K"], theta=(10000.0, 500.0)[i])
        O_, lse = pf.pf_attention_fwd(Qo, Ko, g["V"], g["table"], **kw)
        return (O_, lse, *pf.pf_attention_bwd(Qo, Ko, g["V"], O_, lse, g["dO"], g["table"], **kw))

    want = [run(0), run(1)]
    torch.cuda.synchronize()

    def thread(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got[i].append(run(i))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(got[i]) == 20
        for result in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(result, want[i]))
