"""Attention with the bucketed relative position bias against its definition in double: sizes and masks where it can go
wrong, strides, empty rows, what lies behind the lengths, decoding, repeated and captured calls."""
import numpy as np
import pytest
import torch

from operator_bounds import assert_within, attention_bounds
from oracle import operators as O
from parity import to_gpu
from workloads import Stream

pytestmark = pytest.mark.gpu

CASES = [
    # B, Lq, Lk, heads_q, heads_kv, D, causal, buckets, max_distance, lengths
    (1, 1, 1, 1, 1, 8, False, 8, 16, None),
    (2, 128, 128, 2, 2, 64, False, 32, 128, "pad"),       # an encoder layer, padded
    (1, 129, 129, 2, 1, 64, True, 32, 128, None),         # one row past a tile, shared key head
    (1, 300, 300, 4, 2, 128, True, 16, 64, "pad"),
    (2, 333, 333, 1, 1, 32, False, 8, 20, "pad"),         # far on both sides within a tile
    (1, 70, 205, 3, 1, 96, False, 64, 250, "pad"),        # cross attention: more keys than queries
    (1, 205, 70, 2, 2, 80, False, 32, 128, None),         # more queries than keys
    (2, 65, 65, 2, 2, 40, True, 0, 0, None),              # no bias
    (1, 260, 260, 2, 1, 72, False, 0, 0, "pad"),
    (3, 40, 100, 2, 1, 64, True, 32, 128, "append"),      # a chunk of new tokens at the end of a cache
    (2, 1, 700, 8, 2, 128, True, 32, 128, "append"),      # decoding
    (3, 3, 1000, 4, 4, 64, True, 16, 128, "append"),
    (2, 1, 513, 6, 2, 96, False, 32, 40, "pad"),
    (1, 8, 90, 4, 1, 32, True, 0, 0, "append"),           # 32 rows of one key head
    (1, 9, 90, 4, 1, 32, True, 0, 0, "append"),           # 36
    (1, 2, 3000, 1, 1, 64, False, 256, 1024, None),       # the most buckets, far
    (1, 300, 1500, 1, 1, 32, False, 256, 1024, None),
    (1, 200, 1300, 1, 1, 128, False, 256, 1024, None),    # more than 64 KB of LDS for the table's gradient
    (2, 50, 60, 2, 1, 64, True, 8, 16, "before"),         # queries before the first key: rows that see nothing
]


def _lens(kind, B, Lq, Lk, rng):
    i32 = lambda x: np.asarray(x, dtype=np.int32)  # noqa: E731
    if kind is None:
        return {}
    if kind == "pad":  # one sequence is empty if there are several
        nk = i32([Lk - rng.integers(0, Lk) for _ in range(B)])
        nk[-1] = 0 if B > 1 else nk[-1]
        nq = nk if Lq == Lk else i32([Lq - rng.integers(0, Lq) for _ in range(B)])
        return dict(q_len=nq, kv_len=nk)
    if kind == "append":
        nk = i32([rng.integers(Lq, Lk + 1) for _ in range(B)])
        return dict(q_start=nk - Lq, kv_len=nk)
    return dict(q_start=i32([-30 - 5 * b for b in range(B)]))


def _case(c, dtype, seed):
    B, Lq, Lk, hq, hk, D, causal, nb, dist, kind = c
    s, f = Stream(seed, dtype), Stream(seed + 1)
    d = dict(Q=s.normal((B, Lq, hq, D)), K=s.normal((B, Lk, hk, D)), V=s.normal((B, Lk, hk, D)), dO=s.normal((B, Lq, hq, D)),
             table=f.normal((nb, hq)) if nb else None)
    lens = _lens(kind, B, Lq, Lk, np.random.default_rng(seed))
    kw = dict(causal=causal, max_distance=dist, bidirectional=not causal)
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), None if d["table"] is None else d["table"].astype(np.float64), **kw, **lens)
    g = {k: to_gpu(v, "f32" if k == "table" else dtype) for k, v in d.items()}
    return d, g, o, dict(kw, **{k: torch.from_numpy(v).cuda() for k, v in lens.items()})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_against_definition(c, dtype):
    import paper_2103_03936_amd as pf
    d, g, o, kw = _case(c, dtype, 31)
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    dO = d["dO"].astype(np.float64)
    bounds = attention_bounds(o, dO, dtype)
    assert_within(got, o.O, bounds[0], "O")
    assert_within(lse, o.lse, bounds[1], "lse")
    back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], g["table"], **kw)
    for name, x, y, b in zip(("dQ", "dK", "dV", "dtable"), back, o.backward(dO), bounds[2:]):
        if y is None:
            assert x is None
        else:
            assert_within(x, y, b, name)
    # without the table's gradient dQ, dK, dV hold the same bounds; each call repeats bit for bit
    plain = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], g["table"], need_dtable=False, **kw)
    assert plain[3] is None
    for name, x, y, b in zip(("dQ", "dK", "dV"), plain, o.backward(dO), bounds[2:]):
        assert_within(x, y, b, name + " without dtable")
    for x, y in zip(back, pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], g["table"], **kw)):
        assert x is None or torch.equal(x, y)
    only = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], save_lse=False, **kw)
    assert only[1] is None and torch.equal(only[0], got)


@pytest.mark.parametrize("c", [CASES[1], CASES[3], CASES[9], CASES[10]], ids=str)
def test_what_lies_behind_the_lengths_does_not_matter(c):
    import paper_2103_03936_amd as pf
    d, g, o, kw = _case(c, "bf16", 41)
    want = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    wback = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], *want, g["dO"], g["table"], **kw)
    for b in range(c[0]):
        nk = int(kw["kv_len"][b])
        g["K"][b, nk:], g["V"][b, nk:] = float("nan"), float("inf")
        if "q_len" in kw:
            nq = int(kw["q_len"][b])
            g["Q"][b, nq:], g["dO"][b, nq:] = float("nan"), float("nan")
    got = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], *got, g["dO"], g["table"], **kw)
    for x, y in zip(got + back, want + wback):
        assert torch.equal(x, y)
    for b in range(c[0]):  # gradients of what takes no part are zero
        assert not back[1][b, int(kw["kv_len"][b]):].any() and not back[2][b, int(kw["kv_len"][b]):].any()
        if "q_len" in kw:
            assert not back[0][b, int(kw["q_len"][b]):].any() and not got[0][b, int(kw["q_len"][b]):].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Slices of a fused projection, a part of a cache, heads before tokens, and one key shared by a batch."""
    import paper_2103_03936_amd as pf
    c = (2, 45, 45, 4, 4, 64, True, 16, 32, None)
    d, g, o, kw = _case(c, dtype, 51)
    want = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    wback = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], *want, g["dO"], g["table"], **kw)
    fused = torch.stack((g["Q"], g["K"], g["V"]), 2).contiguous()  # [B, L, 3, H, D]
    cache = torch.full((2, 60, 4, 64), float("nan"), dtype=g["K"].dtype, device="cuda")
    cache[:, :45] = g["V"]
    for Q, K, V in ((fused[:, :, 0], fused[:, :, 1], fused[:, :, 2]), (g["Q"], g["K"], cache[:, :45]),
                    (g["Q"].transpose(1, 2).contiguous().transpose(1, 2), g["K"], g["V"])):
        got = pf.pf_attention_fwd(Q, K, V, g["table"], **kw)
        for x, y in zip(got + pf.pf_attention_bwd(Q, K, V, *got, g["dO"], g["table"], **kw), want + wback):
            assert torch.equal(x, y)
    one = g["K"][:1].expand(2, 45, 4, 64)
    assert torch.equal(pf.pf_attention_fwd(g["Q"], one, g["V"], g["table"], **kw)[0],
                       pf.pf_attention_fwd(g["Q"], one.contiguous(), g["V"], g["table"], **kw)[0])
    q1 = g["Q"][:, 44:].contiguous()
    at = torch.full((2,), 44, dtype=torch.int32, device="cuda")
    a = pf.pf_attention_fwd(fused[:, 44:, 0], fused[:, :, 1], cache[:, :45], g["table"], q_start=at, **kw)
    b = pf.pf_attention_fwd(q1, g["K"], g["V"], g["table"], q_start=at, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_gradients_into_given_tensors():
    import paper_2103_03936_amd as pf
    c = (2, 33, 33, 2, 2, 64, False, 8, 20, "pad")
    d, g, o, kw = _case(c, "f32", 61)
    O_, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    want = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], **kw)
    dY = torch.full((3, 2, 33, 2, 64), 5.0, device="cuda")
    dt = torch.ones(8, 2, device="cuda")
    got = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], grads=dt, out=(dY[0], dY[1], dY[2]), **kw)
    for i in range(3):
        assert torch.equal(dY[i], want[i])
    assert got[3] is dt and torch.equal(dt, 1 + want[3])


def test_scores_of_any_size():
    """Large scores, a bias of the type's lowest value and of minus infinity, a scale of nothing, negative scales."""
    import paper_2103_03936_amd as pf
    c = (1, 100, 100, 2, 2, 64, True, 8, 16, None)
    for dtype in ("f32", "bf16"):
        d, g, _, kw = _case(c, dtype, 71)
        for scale, low in ((10.0, None), (0.0, None), (-0.125, None), (0.125, torch.finfo(torch.float32).min)):
            table = d["table"].copy()
            if low is not None:
                table[0, 0] = low
            o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), table.astype(np.float64), causal=True, max_distance=16,
                            bidirectional=False, scale=scale)
            got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], to_gpu(table), scale=scale, **kw)
            bO, bL = attention_bounds(o, None, dtype)
            if low is None:
                assert_within(got, o.O, bO, f"O scale {scale}")
                assert_within(lse, o.lse, bL, f"lse scale {scale}")
            else:  # row 0 sees itself alone, at the lowest bias; the others see no key of that bias
                seen = slice(1, None)
                assert torch.isfinite(got.float()).all()
                assert np.allclose(got[0, 0, 0].double().cpu().numpy(), o.O[0, 0, 0], rtol=2 ** -7)
                clean = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), np.where(np.abs(table) > 1e30, -1e4, table).astype(np.float64),
                                    causal=True, max_distance=16, bidirectional=False, scale=scale)
                assert_within(got[:, seen], clean.O[:, seen], attention_bounds(clean, None, dtype)[0][:, seen], "O low bias")
        table[0, 0] = -np.inf  # a query's own key is not seen at all then: row 0 sees nothing
        got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], to_gpu(table), scale=0.125, **kw)
        assert not got[0, 0, 0].any() and lse[0, 0, 0] == -float("inf")
        assert_within(got[:, seen], clean.O[:, seen], attention_bounds(clean, None, dtype)[0][:, seen], "O bias -inf")
        back = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], to_gpu(table), scale=0.125, **kw)
        assert all(torch.isfinite(x.float()).all() for x in back) and not back[0][0, 0, 0].any() and back[3][0, 0] == 0


def test_empty_calls():
    import paper_2103_03936_amd as pf
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    t = z(8, 2)
    O_, lse = pf.pf_attention_fwd(z(2, 0, 2, 16), z(2, 5, 2, 16), z(2, 5, 2, 16), t)
    assert O_.shape == (2, 0, 2, 16)
    back = pf.pf_attention_bwd(z(2, 0, 2, 16), z(2, 5, 2, 16), z(2, 5, 2, 16), O_, lse, O_, t)
    assert not back[1].any() and not back[2].any() and not back[3].any()
    q = torch.ones(2, 3, 2, 16, device="cuda")
    for Lq in (3, 40):
        q = torch.ones(2, Lq, 2, 16, device="cuda")
        O_, lse = pf.pf_attention_fwd(q, z(2, 0, 2, 16), z(2, 0, 2, 16), t)
        assert not O_.any() and (lse == -float("inf")).all()
        back = pf.pf_attention_bwd(q, z(2, 0, 2, 16), z(2, 0, 2, 16), O_, lse, q, t)
        assert not back[0].any() and not back[3].any()
    O_, lse = pf.pf_attention_fwd(z(0, 3, 2, 16), z(0, 5, 2, 16), z(0, 5, 2, 16), t)
    assert not pf.pf_attention_bwd(z(0, 3, 2, 16), z(0, 5, 2, 16), z(0, 5, 2, 16), O_, lse, O_, t)[3].any()


def test_refusals():
    import paper_2103_03936_amd as pf
    q = torch.zeros(2, 4, 4, 16, device="cuda")
    k = torch.zeros(2, 6, 2, 16, device="cuda")
    t = torch.zeros(8, 4, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    O_, lse = pf.pf_attention_fwd(q, k, k, t)
    for bad in (lambda: pf.pf_attention_fwd(q, k.bfloat16(), k, t), lambda: pf.pf_attention_fwd(q, k, k, t.bfloat16()),
                lambda: pf.pf_attention_fwd(q.half(), k.half(), k.half()), lambda: pf.pf_attention_fwd(q, k, k, t, kv_len=n.long()),
                lambda: pf.pf_attention_fwd(q[..., ::2], k[..., ::2], k[..., ::2]), lambda: pf.pf_attention_fwd(q, k, k, t[:, :1].expand(8, 4)),
                lambda: pf.pf_attention_fwd(q, k, k, torch.zeros(7, 4, device="cuda")), lambda: pf.pf_attention_fwd(q, k, k, t, max_distance=2),
                lambda: pf.pf_attention_fwd(q, k, k, t, max_distance=2000), lambda: pf.pf_attention_fwd(q, k, k, t, scale=float("nan")),
                lambda: pf.pf_attention_fwd(torch.zeros(1, 1, 1, 136, device="cuda"), *[torch.zeros(1, 1, 1, 136, device="cuda")] * 2),
                lambda: pf.pf_attention_fwd(q, k[:, :, :, 1:9], k[:, :, :, 1:9]) if False else pf.pf_attention_fwd(q[..., 2:10], k[..., 2:10], k[..., 2:10]),
                lambda: pf.pf_attention_fwd(q, k.cpu(), k, t), lambda: pf.pf_attention_fwd(q[:, :, :3], k, k)):
        with pytest.raises(pf.PfError):
            bad()
    for bad in (lambda: pf.pf_attention_fwd(q, k, k[:, :5], t), lambda: pf.pf_attention_fwd(q, k, k, t[:, :2].contiguous()),
                lambda: pf.pf_attention_fwd(q, k, k, t, kv_len=n[:1]), lambda: pf.pf_attention_fwd(q, k, k, t[:0]),
                lambda: pf.pf_attention_bwd(q, k, k, O_, lse[:, :2], O_, t), lambda: pf.pf_attention_bwd(q, k, k, O_, lse, O_[:1], t)):
        with pytest.raises(ValueError):
            bad()


def test_another_stream_and_graph_replay():
    """Calls on a side stream, and forward and backward captured and replayed with new inputs, eager calls in between."""
    import paper_2103_03936_amd as pf
    cases = [(2, 70, 70, 4, 2, 64, True, 32, 128, None), (2, 1, 900, 4, 2, 64, True, 32, 128, "append")]
    for c in cases:
        def run(g, kw):
            O_, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
            return (O_, lse, *pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O_, lse, g["dO"], g["table"], **kw))

        _, static, _, skw = _case(c, "bf16", 80)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            first = run(static, skw)
        side.synchronize()
        for x, y in zip(first, run(static, skw)):
            assert torch.equal(x, y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run(static, skw)
        for rep in range(1, 4):
            _, fresh, _, kw = _case(c, "bf16", 80 + rep)
            eager = run(fresh, kw)
            for k in static:
                static[k].copy_(fresh[k])
            for k in ("q_start", "kv_len"):
                if k in kw:
                    skw[k].copy_(kw[k])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(outs, eager):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(9, 300, 300, 32, 8, 64, False, 32, 128, "pad"), (11, 260, 260, 24, 8, 128, True, 32, 128, None),
                               (65, 140, 135, 8, 4, 40, False, 16, 64, "pad"), (130, 60, 90, 4, 4, 64, True, 32, 128, "append")], ids=str)
def test_many_tiles(c, dtype):
    """More tiles of queries than fit the card at once: no two waves share queries; causal tiles are taken in pairs.  Then more
    tiles of 128 keys than fit it: the waves of dK and dV have keys of their own."""
    test_against_definition(c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq", [1, 150])
def test_nan_stays_in_what_uses_it(Lq, dtype):
    """A NaN in a query reaches that query's results and none else; NaN in keys and values that no query sees reaches none."""
    import paper_2103_03936_amd as pf
    d, g, _, kw = _case((2, Lq, 200, 2, 1, 64, True, 32, 128, None), dtype, 77)
    start = np.asarray([20, 5], dtype=np.int32)
    kw["q_start"] = torch.from_numpy(start).cuda()
    o = O.Attention(*(d[k].astype(np.float64) for k in "QKV"), d["table"].astype(np.float64), causal=True, max_distance=128,
                    bidirectional=False, q_start=start)
    for b in range(2):
        g["K"][b, start[b] + Lq:] = float("nan")
        g["V"][b, start[b] + Lq:] = float("nan")
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    assert_within(got, o.O, attention_bounds(o, d["dO"].astype(np.float64), dtype)[0], "O")
    last = (1, Lq - 1, 1), (1, 1, Lq - 1)
    g["Q"][1, Lq - 1, 1, 3] = float("nan")
    O2, lse2 = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    assert O2[last[0]].isnan().all() and lse2[last[1]].isnan()
    dQ = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], O2, lse2, g["dO"], g["table"], **kw)[0]
    O2[last[0]], lse2[last[1]] = got[last[0]], lse[last[1]]
    assert torch.equal(O2, got) and torch.equal(lse2, lse)
    assert dQ[last[0]].isnan().all()
    dQ[last[0]] = 0
    assert not dQ.isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(3, 70, 1, 4, 2, 64, False, 32, 128, None), (5, 1, 1, 2, 2, 32, True, 16, 64, None),
                               (200, 70, 1, 8, 4, 64, False, 32, 128, None)], ids=str)
def test_one_key(c, dtype):
    """The softmax of one score is 1 whatever the score: no gradient, not even rounding's."""
    import paper_2103_03936_amd as pf
    d, g, o, kw = _case(c, dtype, 19)
    got, lse = pf.pf_attention_fwd(g["Q"], g["K"], g["V"], g["table"], **kw)
    assert torch.equal(got, g["V"].repeat_interleave(c[3] // c[4], 2).expand_as(got))
    dQ, dK, dV, dtable = pf.pf_attention_bwd(g["Q"], g["K"], g["V"], got, lse, g["dO"], g["table"], **kw)
    for x in (dQ, dK, dtable):
        assert not x.any()
    dO = d["dO"].astype(np.float64)
    assert_within(dV, o.backward(dO)[2], attention_bounds(o, dO, dtype)[4], "dV")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [(1, 100, 900, 4, 1, 64, True, 32, 128, "append"), (2, 45, 1300, 3, 1, 128, False, 16, 64, "pad"),
                               (1, 130, 1500, 2, 2, 40, True, 0, 0, "append"), (1, 33, 500, 1, 1, 32, True, 32, 128, None),
                               (2, 70, 700, 2, 2, 96, True, 8, 16, "before"), (1, 12, 2000, 6, 2, 64, False, 32, 128, "pad")], ids=str)
def test_few_queries_many_keys(c, dtype):
    """More rows than one product takes and keys split between workgroups: tiles that pass from one head to the next, and do not."""
    test_against_definition(c, dtype)
