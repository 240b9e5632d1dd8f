"""Refusals of the operators between a Transformer layer's projections and of the AdamW step: wrong arguments come back
as a status before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

import paper_2103_03936_amd as pf

P = ctypes.c_void_p
FAKE = P(256)  # never dereferenced: the calls below fail before any launch
Z = ctypes.c_size_t
BIG = Z(1 << 40)


def _qk(B=2, L=3, hq=4, hk=2, D=16, rot=16, norm=1, style=0, dtype=0, eps=1e-6, theta=1e4, **strides):
    d = pf.pf_qk_norm_desc(B, L, hq, hk, D, rot, norm, style, dtype, eps, theta)
    for k, v in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*v))
    return ctypes.byref(d)


def test_qk_norm_refusals():
    f = lambda d, Q=FAKE, K=FAKE, gq=None, pos=None, Qo=FAKE, Ko=FAKE: pf.lib.pf_qk_norm_rotate_fwd(  # noqa: E731
        d, Q, K, gq, None, pos, Qo, Ko, None)
    assert f(None) == 1
    for bad in (dict(hq=0), dict(hk=-1), dict(D=0), dict(B=-1), dict(L=-1), dict(rot=-4)):
        assert f(_qk(**bad)) == 2, bad
    for bad in (dict(dtype=5), dict(norm=2), dict(style=2), dict(D=12), dict(D=264), dict(rot=6), dict(rot=20), dict(theta=0.0),
                dict(theta=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(B=1 << 20, L=1 << 11),
                dict(q_stride=(48, 16, 6)), dict(k_stride=(-64, 16, 16)), dict(qo_stride=(2, 64, 16)), dict(dk_stride=(64, 64, 1)),
                dict(dtype=1, q_stride=(64, 4, 16))):
        assert f(_qk(**bad)) == 3, bad
    assert f(_qk(), Q=None) == 1 and f(_qk(), K=None) == 1 and f(_qk(), Qo=None) == 1 and f(_qk(), Ko=None) == 1
    assert f(_qk(), Q=P(264)) == 3 and f(_qk(), gq=P(258)) == 3 and f(_qk(), pos=P(257)) == 3 and f(_qk(), Ko=P(260)) == 3
    assert f(_qk(B=0), Q=None) == 0 and f(_qk(L=0), Q=None) == 0
    b = lambda d, ws=FAKE, n=BIG, Q=FAKE, dq=FAKE, dg=FAKE: pf.lib.pf_qk_norm_rotate_bwd(  # noqa: E731
        d, Q, FAKE, None, None, None, FAKE, FAKE, dq, FAKE, dg, None, 0, ws, n, None)
    need = pf.lib.pf_qk_norm_rotate_bwd_workspace_bytes(_qk())
    assert need > 0
    assert b(_qk(), ws=None) == 4 and b(_qk(), n=Z(need - 1)) == 4 and b(_qk(), ws=P(128)) == 3
    assert b(_qk(), Q=None) == 1 and b(_qk(), dq=None) == 1 and b(_qk(), dg=P(257)) == 3
    assert pf.lib.pf_qk_norm_rotate_bwd_workspace_bytes(_qk(norm=0)) == 0
    assert pf.lib.pf_qk_norm_rotate_bwd_workspace_bytes(_qk(D=12)) == 0


def _at(B=2, Lq=3, Lk=5, hq=4, hk=2, D=16, causal=0, buckets=8, dist=16, two=1, dtype=0, scale=1.0, **strides):
    d = pf.pf_attention_desc(B, Lq, Lk, hq, hk, D, causal, buckets, dist, two, dtype, scale)
    for k, v in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*v))
    return ctypes.byref(d)


def test_attention_refusals():
    f = lambda d, Q=FAKE, K=FAKE, t=FAKE, O=FAKE, lens=None, lse=None, ws=None, n=Z(0): pf.lib.pf_attention_fwd(  # noqa: E731, E741
        d, Q, K, FAKE, t, lens, None, None, O, lse, ws, n, None)
    assert f(None) == 1
    for bad in (dict(B=-1), dict(Lq=-1), dict(Lk=-1), dict(hq=0), dict(hk=0), dict(D=0), dict(hq=3, hk=2)):
        assert f(_at(**bad)) == 2, bad
    for bad in (dict(dtype=3), dict(D=12), dict(D=136), dict(buckets=3), dict(buckets=2), dict(buckets=-2), dict(buckets=258),
                dict(buckets=1, two=0), dict(dist=2), dict(dist=1025), dict(buckets=256, two=0, dist=128), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(Lq=1 << 30), dict(Lk=1 << 30), dict(B=1 << 30), dict(B=1 << 20, Lq=1 << 20),
                dict(q_stride=(48, 16, 6)), dict(k_stride=(64, -16, 16)), dict(dtype=1, v_stride=(64, 16, 4))):
        assert f(_at(**bad)) == 3, bad
    assert f(_at(), Q=None) == 1 and f(_at(), K=None) == 1 and f(_at(), t=None) == 1 and f(_at(), O=None) == 1
    assert f(_at(), Q=P(264)) == 3 and f(_at(), lens=P(257)) == 3 and f(_at(), lse=P(258)) == 3
    assert f(_at(B=0), Q=None) == 0 and f(_at(Lq=0), Q=None) == 0
    # few queries over many keys need room for their parts
    d = _at(B=1, Lq=1, Lk=4096)
    need = pf.lib.pf_attention_fwd_workspace_bytes(d)
    assert need > 0
    assert f(d) == 4 and f(d, ws=FAKE, n=Z(need - 1)) == 4 and f(d, ws=P(128), n=BIG) == 3
    assert pf.lib.pf_attention_fwd_workspace_bytes(_at(D=12)) == 0
    b = lambda d, O=FAKE, lse=FAKE, dO=FAKE, dK=FAKE, dt=FAKE, t=FAKE, ws=FAKE, n=BIG: pf.lib.pf_attention_bwd(  # noqa: E731, E741
        d, FAKE, FAKE, FAKE, t, None, None, None, O, lse, dO, FAKE, dK, FAKE, dt, 0, ws, n, None)
    need = pf.lib.pf_attention_bwd_workspace_bytes(_at())
    assert need > 0
    assert b(_at(), ws=None) == 4 and b(_at(), n=Z(need - 1)) == 4 and b(_at(), ws=P(320)) == 3
    assert b(_at(), O=None) == 1 and b(_at(), lse=None) == 1 and b(_at(), dO=None) == 1 and b(_at(), dK=None) == 1 and b(_at(), t=None) == 1
    assert b(_at(), dt=P(257)) == 3 and b(_at(), dO=P(264)) == 3 and b(_at(D=20)) == 3


def test_attention_outputs_are_not_inputs():
    q, k, v, o, lse, g, dq, dk, dv, ws = (P(256 * (i + 1)) for i in range(10))
    d = _at()
    for out in (q, k, v):
        assert pf.lib.pf_attention_fwd(d, q, k, v, FAKE, None, None, None, out, None, None, Z(0), None) == 3
    good = [dq, dk, dv]
    for i in range(3):
        for other in [q, k, v, o, g] + good[:i]:
            outs = good[:i] + [other] + good[i + 1:]
            assert pf.lib.pf_attention_bwd(d, q, k, v, FAKE, None, None, None, o, lse, g, *outs, None, 0, ws, BIG, None) == 3


def _adamw(n=1, bits=32, b1=0.9, b2=0.99, eps=1e-8):
    return pf.pf_adamw_desc(n, bits, b1, b2, eps)


def _tensor(**kw):
    t = dict(param=256, grad=512, m=768, v=1024, m_scale=None, v_scale=None, copy=None, count=5000, weight_decay=0.0)
    t.update(kw)
    return (pf.pf_adamw_tensor * 1)(pf.pf_adamw_tensor(*(t[k] for k, _ in pf.pf_adamw_tensor._fields_)))


def test_adamw_refusals():
    size, fill, step = pf.lib.pf_adamw_plan_bytes, pf.lib.pf_adamw_plan_fill, pf.lib.pf_adamw_step
    host = ctypes.create_string_buffer(1 << 16)

    def status(d, t):
        assert size(ctypes.byref(d), t) == 0
        return fill(ctypes.byref(d), t, host, Z(len(host)))

    assert fill(None, _tensor(), host, Z(len(host))) == 1
    assert status(_adamw(), None) == 1
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None)):
        assert status(_adamw(), _tensor(**bad)) == 1, bad
    assert status(_adamw(bits=8), _tensor()) == 1  # no scales
    assert status(_adamw(n=-1), _tensor()) == 2 and status(_adamw(), _tensor(count=-1)) == 2
    assert status(_adamw(), _tensor(count=1 << 62)) == 2
    for d in (_adamw(bits=16), _adamw(b1=1.0), _adamw(b2=-0.1), _adamw(eps=-1.0), _adamw(b1=float("nan"))):
        assert status(d, _tensor()) == 3
    for bad in (dict(param=258), dict(grad=513), dict(m=770), dict(copy=257)):
        assert status(_adamw(), _tensor(**bad)) == 3, bad
    good, t = _adamw(), _tensor()
    need = size(ctypes.byref(good), t)
    assert need > 0 and fill(ctypes.byref(good), t, host, Z(need - 1)) == 4 and fill(ctypes.byref(good), t, None, Z(need)) == 4
    assert fill(ctypes.byref(good), t, host, Z(need)) == 0
    # a tensor without values is left out
    assert size(ctypes.byref(good), _tensor(count=0, param=None)) < need
    d = ctypes.byref(good)
    assert step(None, FAKE, Z(need), FAKE, None, FAKE, None) == 1
    assert step(d, FAKE, Z(need), None, None, FAKE, None) == 1 and step(d, FAKE, Z(need), FAKE, None, None, None) == 1
    assert step(d, None, Z(need), FAKE, None, FAKE, None) == 4 and step(d, FAKE, Z(100), FAKE, None, FAKE, None) == 4
    assert step(d, FAKE, Z(need - 4), FAKE, None, FAKE, None) == 4
    assert step(d, P(128), Z(need), FAKE, None, FAKE, None) == 3 and step(d, FAKE, Z(need), P(258), None, FAKE, None) == 3
    assert step(d, FAKE, Z(need), FAKE, None, P(260), None) == 3
    assert step(ctypes.byref(_adamw(bits=4)), FAKE, Z(need), FAKE, None, FAKE, None) == 3


def test_python_refuses_cpu_tensors_and_bad_options():
    x = torch.zeros(1, 2, 4, 16)
    with pytest.raises(pf.PfError):
        pf.pf_qk_norm_rotate_fwd(x, None)
    with pytest.raises(pf.PfError):
        pf.pf_attention_fwd(x, x, x)
    with pytest.raises(KeyError):
        pf.pf_qk_norm_rotate_fwd(x, None, norm="layer")
    with pytest.raises(KeyError):
        pf.pf_qk_norm_rotate_fwd(x, None, style="both")
    with pytest.raises(ValueError):
        pf.pf_qk_norm_rotate_fwd(x[0], None)
    with pytest.raises(TypeError):
        pf.pf_attention_fwd(x, None, x)
    w = torch.zeros(8)
    with pytest.raises(pf.PfError):
        pf.AdamW([w], [w])
    with pytest.raises(pf.PfError):
        pf.AdamW([w], [w], state_bits=16)
    with pytest.raises(ValueError):
        pf.AdamW([w], [w, w])
    with pytest.raises(ValueError):
        pf.AdamW([w], [w], betas=(1.0, 0.9))
    with pytest.raises(ValueError):
        pf.AdamW([], [])
