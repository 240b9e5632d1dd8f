"""Tables that mix biases of very different sizes, as masks do, over random shapes: levels that are far apart have the results
and gradients of levels 300 apart, whose exponentials are as good as none either."""
import numpy as np
import pytest
import torch

from operator_bounds import assert_within, attention_bounds
from oracle import operators as O
from parity import to_gpu
from test_gpu_attention import _case

pytestmark = pytest.mark.gpu

REAL = [0.0, -1e4, -1e9, float(np.finfo(np.float32).min), 1e6, -np.inf]
LIKE = [0.0, -300.0, -600.0, -900.0, 300.0, -np.inf]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed", range(16))
def test_levels(seed, dtype):
    import paper_2103_03936_amd as pf
    rng = np.random.default_rng(seed)
    hk = int(rng.choice([1, 2, 4]))
    hq, causal = hk * int(rng.choice([1, 2, 5])), bool(rng.integers(2))
    B, D = int(rng.choice([1, 3, 40])), int(rng.choice([8, 32, 40, 64, 96, 128]))
    kind = str(rng.choice(["pad", "append", "before", "none"])) if causal else str(rng.choice(["pad", "none"]))
    Lq, Lk = int(rng.integers(1, 140)), int(rng.integers(1, 300))
    if kind == "append" or seed % 5 == 0:
        Lq = int(rng.integers(1, 6))
        Lk = max(Lk, Lq) + (500 if seed % 5 == 0 else 0)
    nb, dist = int(rng.choice([4, 16, 32])), int(rng.choice([20, 100]))
    d, g, _, kw = _case((B, Lq, Lk, hq, hk, D, causal, nb, dist, None if kind == "none" else kind), dtype, 200 + seed)
    lens = {k: kw[k].cpu().numpy() for k in ("q_start", "q_len", "kv_len") if k in kw}
    level = rng.choice(6, (nb, hq), p=rng.dirichlet([1] * 6)).astype(int)
    # (beside a bias of 1e6 float32 has no digits of a small one that comes with it: levels alone there)
    small = np.where(np.isin(level, [0]), rng.standard_normal((nb, hq)), 0.0).astype(np.float32)
    real, like = np.float32(REAL)[level] + small, np.float32(LIKE)[level] + small
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), like.astype(np.float64), causal=causal, max_distance=dist,
                    bidirectional=not causal, **lens)
    dO = d["dO"].astype(np.float64)
    bounds, want = attention_bounds(o, dO, dtype), o.backward(dO)
    table = to_gpu(real)
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], table, **kw)
    assert_within(got, o.O, bounds[0], "O")
    assert np.array_equal(lse.cpu().numpy() == -np.inf, o.lse == -np.inf)
    back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], table, **kw)
    for name, x, y, b in zip("dQ dK dV dtable".split(), back, want, bounds[2:]):
        assert_within(x, y, b, name)
    for x, y in zip(back, pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], table, **kw)):
        assert torch.equal(x, y)
    # captured and replayed with another table: whether a row is large is decided anew
    graph = torch.cuda.CUDAGraph()
    plain = torch.zeros_like(table)
    held = plain.clone()
    with torch.cuda.graph(graph):
        O2, lse2 = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], held, **kw)
        back2 = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O2, lse2, g["dO"], held, **kw)
    for t in (table, plain, table):
        held.copy_(t)
        a = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], t, **kw)
        b = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], *a, g["dO"], t, **kw)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((O2, lse2, *back2), (*a, *b)):
            assert torch.equal(x, y)
