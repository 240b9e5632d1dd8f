"""Norms of queries and keys with the rotation against their definition in double, and how the calls are made."""
import numpy as np
import pytest
import torch

from operator_bounds import assert_within, qk_bounds, turn_bound
from oracle import operators as O
from parity import to_gpu
from workloads import Stream

pytestmark = pytest.mark.gpu

CASES = [
    # dtype, B, L, heads_q, heads_k, D, rot, style, norm, gamma
    ("f32", 1, 1, 1, 1, 8, 8, "halves", "rms", True),
    ("bf16", 1, 1, 1, 0, 8, 4, "pairs", "rms", True),
    ("bf16", 64, 1, 8, 8, 64, 64, "halves", "rms", True),       # a decoding step
    ("bf16", 3, 37, 8, 8, 64, 64, "halves", "rms", True),
    ("bf16", 2, 19, 8, 2, 128, 128, "pairs", "rms", True),
    ("bf16", 2, 50, 6, 2, 80, 40, "halves", "rms", True),       # 20 pairs and 20 unturned: four to a lane
    ("f32", 2, 50, 6, 2, 80, 40, "pairs", "rms", True),
    ("f32", 2, 33, 5, 1, 96, 48, "halves", "rms", False),
    ("bf16", 2, 33, 3, 3, 200, 100, "halves", "none", False),
    ("f32", 2, 9, 4, 4, 256, 256, "halves", "none", False),
    ("bf16", 1, 40, 9, 3, 256, 36, "pairs", "rms", True),       # 18 pairs: two to a lane, all 64 lanes
    ("f32", 1, 7, 2, 1, 248, 4, "halves", "rms", True),
    ("bf16", 2, 11, 4, 2, 32, 0, "halves", "rms", True),        # no rotation
    ("f32", 1, 3000, 2, 1, 16, 16, "pairs", "rms", True),       # more tokens than workgroups
]


def _inputs(c, seed, far):
    dtype, B, L, hq, hk, D, rot, style, norm, gamma = c
    s = Stream(seed, dtype)
    f = Stream(seed + 1)
    pos = (s.integers((B, 1), far) + np.arange(L)[None]).astype(np.int32) if far else None
    d = dict(Q=s.normal((B, L, hq, D)), K=s.normal((B, L, max(hk, 1), D), 3.0), dQ=s.normal((B, L, hq, D)),
             dK=s.normal((B, L, max(hk, 1), D)), gq=1 + f.normal((D,), 0.2) if gamma else None,
             gk=1 + f.normal((D,), 0.2) if gamma else None)
    return d, pos


def _check(c, d, pos, out, back):
    dtype, B, L, hq, hk, D, rot, style, norm, gamma = c
    p = np.broadcast_to(np.arange(L), (B, L)) if pos is None else pos
    kw = dict(norm=norm, rot_dim=rot, style=style)
    for i, (x, dy, g) in enumerate(((d["Q"], d["dQ"], d["gq"]), (d["K"], d["dK"], d["gk"]))[:1 + (hk > 0)]):
        x, dy, g = x.astype(np.float64), dy.astype(np.float64), None if g is None else g.astype(np.float64)
        y = O.qk_norm_rotate_fwd(x, g, p, **kw)
        dx, dg = O.qk_norm_rotate_bwd(x, dy, g, p, **kw)
        if norm == "rms":
            by, bx, bg = qk_bounds(x, dy, g, p, dtype, D)
        else:
            by, bx = turn_bound(x, p, dtype), turn_bound(dy, p, dtype)
        assert_within(out[i], y, by, "QK"[i] + "o")
        assert_within(back[i], dx, bx, "dQ dK".split()[i])
        if norm == "rms" and g is not None:
            assert_within(back[2 + i], dg, bg, "dgamma")


@pytest.mark.parametrize("far", [0, 2 ** 30])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_against_definition(c, far):
    import paper_2103_03936_amd as pf
    dtype, B, L, hq, hk, D, rot, style, norm, gamma = c
    d, pos = _inputs(c, 11, far)
    g = {k: to_gpu(v, "f32" if k[0] == "g" else dtype) for k, v in d.items()}
    kw = dict(positions=None if pos is None else torch.from_numpy(pos).cuda(), norm=norm, rot_dim=rot, style=style)
    K, dK = (g["K"], g["dK"]) if hk else (None, None)
    out = pf.pf_qk_norm_rotate_fwd(g["Q"], K, g["gq"], g["gk"], **kw)
    back = pf.pf_qk_norm_rotate_bwd(g["Q"], K, g["dQ"], dK, g["gq"], g["gk"], **kw)
    again = pf.pf_qk_norm_rotate_bwd(g["Q"], K, g["dQ"], dK, g["gq"], g["gk"], **kw)
    if not hk:
        assert out[1] is None and back[1] is None and back[3] is None
    _check(c, d, pos, out, back)
    for x, y in zip(back, again):
        assert x is None or torch.equal(x, y)


def test_slices_of_one_buffer_and_of_a_cache():
    """Q and K as slices of a fused projection, Ko into a cache, gradients into a fused gradient: the values around stay."""
    import paper_2103_03936_amd as pf
    c = ("bf16", 3, 5, 4, 2, 64, 64, "halves", "rms", True)
    d, pos = _inputs(c, 21, 1000)
    g = {k: to_gpu(v, "f32" if k[0] == "g" else "bf16") for k, v in d.items()}
    kw = dict(positions=torch.from_numpy(pos).cuda())
    want = pf.pf_qk_norm_rotate_fwd(g["Q"], g["K"], g["gq"], g["gk"], **kw)
    wback = pf.pf_qk_norm_rotate_bwd(g["Q"], g["K"], g["dQ"], g["dK"], g["gq"], g["gk"], **kw)
    fused = torch.full((3, 5, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    fused[:, :, :4], fused[:, :, 4:6] = g["Q"], g["K"]
    cache = torch.full((3, 20, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    Qo = torch.empty_like(g["Q"])
    Q, K = fused[:, :, :4], fused[:, :, 4:6]
    got = pf.pf_qk_norm_rotate_fwd(Q, K, g["gq"], g["gk"], out=(Qo, cache[:, 6:11]), **kw)
    assert got[0] is Qo and torch.equal(Qo, want[0]) and torch.equal(cache[:, 6:11], want[1])
    assert (cache[:, :6] == 9).all() and (cache[:, 11:] == 9).all()
    dfused = torch.full((3, 5, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    dg = (torch.ones(64, device="cuda"), torch.zeros(64, device="cuda"))
    back = pf.pf_qk_norm_rotate_bwd(Q, K, g["dQ"], g["dK"], g["gq"], g["gk"], grads=dg, out=(dfused[:, :, :4], dfused[:, :, 4:6]), **kw)
    assert torch.equal(dfused[:, :, :4], wback[0]) and torch.equal(dfused[:, :, 4:6], wback[1]) and (dfused[:, :, 6:] == 3).all()
    assert back[2] is dg[0] and torch.equal(dg[0], 1 + wback[2]) and torch.equal(dg[1], wback[3])
    # in place
    pf.pf_qk_norm_rotate_fwd(Q, K, g["gq"], g["gk"], out=(Q, K), **kw)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and (fused[:, :, 6:] == 7).all()
    # transposed storage: heads before tokens
    Qt = g["Q"].transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(pf.pf_qk_norm_rotate_fwd(Qt, None, g["gq"], **kw)[0], want[0])


def test_empty_batch_and_refusals():
    import paper_2103_03936_amd as pf
    x = torch.zeros(0, 4, 2, 16, device="cuda")
    gamma = torch.ones(16, device="cuda")
    assert pf.pf_qk_norm_rotate_fwd(x, x, gamma, gamma)[0].shape == x.shape
    back = pf.pf_qk_norm_rotate_bwd(x, x, x, x, gamma, gamma)
    assert not back[2].any() and not back[3].any()
    y = torch.zeros(2, 4, 2, 16, device="cuda")
    for bad in (lambda: pf.pf_qk_norm_rotate_fwd(y.half(), None), lambda: pf.pf_qk_norm_rotate_fwd(y[..., ::2], None),
                lambda: pf.pf_qk_norm_rotate_fwd(y[..., :12], None), lambda: pf.pf_qk_norm_rotate_fwd(y, None, gamma.bfloat16()),
                lambda: pf.pf_qk_norm_rotate_fwd(y, y.bfloat16()), lambda: pf.pf_qk_norm_rotate_fwd(y[:1, :1, :1].expand(2, 4, 2, 16), None),
                lambda: pf.pf_qk_norm_rotate_fwd(y, None, out=(y[:1].expand(2, 4, 2, 16), None)),
                lambda: pf.pf_qk_norm_rotate_fwd(y, None, positions=torch.zeros(2, 4, device="cuda", dtype=torch.int64)),
                lambda: pf.pf_qk_norm_rotate_fwd(torch.zeros(2, 4, 2, 20, device="cuda")[..., 4:], None, rot_dim=6)):
        with pytest.raises(pf.PfError):
            bad()
    for bad in (lambda: pf.pf_qk_norm_rotate_fwd(y, None, gamma[:8]), lambda: pf.pf_qk_norm_rotate_fwd(y, y[:1]),
                lambda: pf.pf_qk_norm_rotate_fwd(y, None, out=(y,)), lambda: pf.pf_qk_norm_rotate_bwd(y, None, y[:, :2], None)):
        with pytest.raises(ValueError):
            bad()
