"""Biases of any finite size, forward.  A bias that a whole row shares does not change its softmax: a row whose keys all have a
bias of -1e9, or of the type's lowest value, has the results that it has without it."""
import numpy as np
import pytest
import torch

from operator_bounds import E, assert_within, attention_bounds
from oracle import operators as O
from parity import to_gpu
from test_gpu_attention import _case

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)
SHAPES = [  # B, Lq, Lk, heads_q, heads_kv, D, causal, lengths
    (1, 100, 100, 2, 2, 64, True, None),
    (2, 300, 300, 4, 2, 128, True, "pad"),
    (2, 70, 205, 3, 1, 96, False, "pad"),
    (1, 205, 70, 2, 2, 40, False, None),
    (2, 1, 700, 8, 2, 128, True, "append"),     # decoding, several parts
    (3, 40, 100, 2, 1, 64, True, "append"),
    (1, 64, 2048, 1, 1, 64, False, None),       # more rows than one product takes, several parts
    (9, 300, 300, 32, 8, 64, False, "pad"),     # no two waves share queries
    (65, 140, 135, 8, 4, 40, False, "pad"),     # waves with keys of their own
]


def _check(c, dtype, real, like):
    """real: the table that the kernels get; like: one with the same softmax and gradients, of a size that double and
    float hold easily."""
    import paper_2103_03936_amd as pf
    B, Lq, Lk, hq, hk, D, causal, kind = c
    d, g, _, kw = _case((B, Lq, Lk, hq, hk, D, causal, real.shape[0], 16, kind), dtype, 23)
    lens = {k: kw[k].cpu().numpy() for k in ("q_start", "q_len", "kv_len") if k in kw}
    opts = dict(causal=causal, max_distance=16, bidirectional=not causal, **lens)
    x = [d[k].astype(np.float64) for k in "QKV"]
    o = O.Attention(*x, like.astype(np.float64), **opts)
    bounds = attention_bounds(o, None, dtype)
    table = to_gpu(real)
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], table, **kw)
    assert_within(got, o.O, bounds[0], "O")
    top = np.abs(real).max()
    if top < 2e38:  # (the bias is held times log2(e), and not beyond the type's largest value)
        want_lse = O.Attention(*x, real.astype(np.float64), **opts).lse
        assert_within(lse, want_lse, bounds[1] + 8 * E * np.where(np.isfinite(want_lse), np.abs(want_lse), 0), "lse")


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
