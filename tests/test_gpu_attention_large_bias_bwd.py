"""Biases of any finite size, backward, and scores of any size: P is normalised by the row's own sum where lse has lost it."""
import numpy as np
import pytest

from operator_bounds import E, assert_within, attention_bounds
from oracle import operators as O
from parity import to_gpu
from test_gpu_attention import _case
from test_gpu_attention_large_bias import LOWEST, SHAPES

pytestmark = pytest.mark.gpu


def _check(c, dtype, real, like):
    """real: the table that the kernels get; like: one with the same softmax and gradients, of a size that double and
    float hold easily."""
    import paper_2103_03936_amd as pf
    B, Lq, Lk, hq, hk, D, causal, kind = c
    d, g, _, kw = _case((B, Lq, Lk, hq, hk, D, causal, real.shape[0], 16, kind), dtype, 23)
    lens = {k: kw[k].cpu().numpy() for k in ("q_start", "q_len", "kv_len") if k in kw}
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), like.astype(np.float64), causal=causal, max_distance=16,
                    bidirectional=not causal, **lens)
    dO = d["dO"].astype(np.float64)
    bounds, want = attention_bounds(o, dO, dtype), o.backward(dO)
    table = to_gpu(real)
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], table, **kw)
    back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], table, **kw)
    for name, y, z, b in zip(("dQ", "dK", "dV", "dtable"), back, want, bounds[2:]):
        assert_within(y, z, b, name)
    plain = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], table, need_dtable=False, **kw)
    for name, y, z, b in zip(("dQ", "dK", "dV"), plain, want, bounds[2:]):
        assert_within(y, z, b, name + " without dtable")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-1e8, -1e9, 1e9, -1e20, LOWEST])
@pytest.mark.parametrize("c", SHAPES, ids=str)
def test_all_keys_share_it(c, low, dtype):
    nb = 8 if c[6] else 16
    real = np.full((nb, c[3]), low, dtype=np.float32)
    _check(c, dtype, real, np.zeros_like(real))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-1e8, -1e9, LOWEST])
@pytest.mark.parametrize("c", [SHAPES[0], SHAPES[1], (4, 90, 90, 2, 1, 64, True, "pad")], ids=str)
def test_rows_that_see_only_low_buckets(c, low, dtype):
    """Buckets 0 .. 3 (distances 0 .. 3) are low: the first four queries see nothing else, the others do not see those
    keys beside the further ones.  Then buckets 2 and 3 lower still."""
    rng = np.random.default_rng(3)
    real = rng.standard_normal((8, c[3])).astype(np.float32)
    like = real.copy()
    real[:4], like[:4] = low, -300.0
    _check(c, dtype, real, like)
    if low != LOWEST:
        real[2:4], like[2:4] = 2 * low, -600.0
        _check(c, dtype, real, like)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_high_bucket(dtype):
    """Where one bucket is far above the others its keys share the row between them."""
    rng = np.random.default_rng(4)
    real = rng.standard_normal((16, 2)).astype(np.float32)
    like = real.copy()
    real[9], like[9] = 1e9, 300.0  # the next key
    real[15], like[15] = 1e9, 300.0  # all far ones behind
    _check((2, 100, 100, 2, 2, 64, False, "pad"), dtype, real, like)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(1, 100, 100, 2, 2, 64, True, None), (2, 130, 200, 4, 2, 128, False, "pad"),
                               (9, 300, 300, 32, 8, 64, False, "pad"), (65, 140, 135, 8, 4, 40, False, "pad")], ids=str)
def test_large_scores(c, dtype):
    """Scores of some thousands without a bias.  Queries and keys are small whole numbers, so that float holds every product
    whatever the order of its sum; each query's P sums to 1, so that its part of dV sums to its dO."""
    import paper_2103_03936_amd as pf
    B, Lq, Lk, hq, hk, D, causal, kind = c
    d, g, _, kw = _case((B, Lq, Lk, hq, hk, D, causal, 0, 0, kind), dtype, 29)
    d["Q"], d["K"] = np.rint(4 * d["Q"]), np.rint(4 * d["K"])
    g["Q"], g["K"] = to_gpu(d["Q"], dtype), to_gpu(d["K"], dtype)
    lens = {k: kw[k].cpu().numpy() for k in ("q_start", "q_len", "kv_len") if k in kw}
    kw = dict(causal=causal, scale=16.0, **{k: kw[k] for k in lens})
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), causal=causal, scale=16.0, **lens)
    assert np.abs(o.lse[np.isfinite(o.lse)]).max() > 2000
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], **kw)
    dO = d["dO"].astype(np.float64)
    back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], **kw)
    bounds, want = attention_bounds(o, dO, dtype), o.backward(dO)
    for name, x, y, b in zip(("O", "dQ", "dK", "dV"), (got, *back[:3]), (o.O, *want[:3]), (bounds[0], *bounds[2:5])):
        assert_within(x, y, b, name)
    # P: nk exponentials of 2 steps each and their sum, once rounded to the type; dV: a sum over the queries that is rounded once
    nq, nk, half = lens.get("q_len", np.full(B, Lq)), lens.get("kv_len", np.full(B, Lk)), 2.0 ** -8 if dtype == "bf16" else 0.0
    dV = back[2].double().cpu().numpy()
    for b in range(B):
        if nq[b] == 0 or nk[b] == 0:
            continue
        at = dO[b, :nq[b]].reshape(nq[b], hk, hq // hk, D)
        slack = (half + (nq[b] * hq // hk + nk[b] + 100) * E) * np.abs(at).sum((0, 2)) + 1.01 * half * np.abs(dV[b]).sum(0)
        assert (np.abs(dV[b].sum(0) - at.sum((0, 2))) <= slack).all(), b
