"""Outputs that overlap inputs or each other are refused before anything is launched (no GPU)."""
import ctypes

import pytest

import paper_2103_03936_amd as pf

P, Z = ctypes.c_void_p, ctypes.c_size_t
BIG = Z(1 << 40)
B, L, HQ, HK, D = 2, 5, 4, 2, 16
NQ, NK = B * L * HQ * D * 4, B * L * HK * D * 4  # bytes, float32
AT = 1 << 20


def _places(*sizes):
    """Addresses of tensors that do not meet, 256-byte aligned."""
    at, out = AT, []
    for n in sizes:
        out.append(at)
        at += (n + 511) // 256 * 256
    return out


def _qk(**strides):
    d = pf.pf_qk_norm_desc(B, L, HQ, HK, D, D, 1, 0, 0, 1e-6, 1e4)
    for k, v in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*v))
    return ctypes.byref(d)


@pytest.mark.parametrize("which,where", [(w, x) for w in "Qo Ko".split() for x in ("other", "inside", "end", "output")])
def test_norm_forward(which, where):
    q, k, qo, ko = _places(NQ, NK, NQ, NK)
    own, other, mine, size = (q, k, "qo", NQ) if which == "Qo" else (k, q, "ko", NK)
    bad = {"other": other, "inside": own + 16, "end": own + size - 16, "output": (ko if which == "Qo" else qo) + 16}[where]
    outs = dict(qo=qo, ko=ko)
    outs[mine] = bad
    assert pf.lib.pf_qk_norm_rotate_fwd(_qk(), P(q), P(k), None, None, None, P(outs["qo"]), P(outs["ko"]), None) == 3


def test_norm_forward_in_place_at_other_strides():
    q, k, qo, ko = _places(4 * NQ, NK, NQ, NK)
    apart = (L * HQ * D * 2, HQ * D * 2, D * 2)
    assert pf.lib.pf_qk_norm_rotate_fwd(_qk(qo_stride=apart), P(q), P(k), None, None, None, P(q), P(ko), None) == 3
    # slices of one buffer that do not meet are told from those that do
    fused = dict(q_stride=(L * 8 * D, 8 * D, D), k_stride=(L * 8 * D, 8 * D, D), qo_stride=(L * 8 * D, 8 * D, D))
    assert pf.lib.pf_qk_norm_rotate_fwd(_qk(**fused), P(q), P(q + 4 * HQ * D), None, None, None, P(q + 4 * D), P(ko), None) == 3


@pytest.mark.parametrize("bad", [("dq", "k"), ("dq", "dko"), ("dk", "q"), ("dk", "dqo"), ("dk", "dq"), ("gq", "q"), ("gk", "dq"), ("gq", "gk+")], ids=str)
def test_norm_backward(bad):
    names = "q k dqo dko dq dk gq gk ws".split()
    at = dict(zip(names, _places(NQ, NK, NQ, NK, NQ, NK, 4 * D, 4 * D, 1 << 16)))
    at[bad[0]] = at[bad[1].rstrip("+")] + (4 if bad[1][-1] == "+" else 16)
    p = {k: P(v) for k, v in at.items()}
    assert pf.lib.pf_qk_norm_rotate_bwd(_qk(), p["q"], p["k"], None, None, None, p["dqo"], p["dko"], p["dq"], p["dk"], p["gq"], p["gk"], 0, p["ws"],
                                        BIG, None) == 3


def _attention(**strides):
    d = pf.pf_attention_desc(B, L, L, HQ, HK, D, 0, 8, 16, 1, 0, 1.0)
    for k, v in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*v))
    return ctypes.byref(d)


SIZES = dict(q=NQ, k=NK, v=NK, t=8 * HQ * 4, o=NQ, lse=B * L * HQ * 4, g=NQ, dq=NQ, dk=NK, dv=NK, dt=8 * HQ * 4)


@pytest.mark.parametrize("bad", [(x, y) for x, y in [("o", "q"), ("o", "k"), ("o", "v"), ("o", "t"), ("lse", "q"), ("lse", "o")]], ids=str)
@pytest.mark.parametrize("end", [False, True])
def test_attention_forward(bad, end):
    at = dict(zip(SIZES, _places(*SIZES.values())))
    at[bad[0]] = at[bad[1]] + (SIZES[bad[1]] - 16 if end else 16)
    p = {k: P(v) for k, v in at.items()}
    assert pf.lib.pf_attention_fwd(_attention(), p["q"], p["k"], p["v"], p["t"], None, None, None, p["o"], p["lse"], None, Z(0), None) == 3


@pytest.mark.parametrize("bad", [(x, y) for x in ("dq", "dk", "dv", "dt") for y in SIZES if x != y and not (x == "dt" and y[0] == "d")], ids=str)
def test_attention_backward(bad):
    at = dict(zip(SIZES, _places(*SIZES.values())))
    at[bad[0]] = at[bad[1]] + (SIZES[bad[1]] - 16)
    p = {k: P(v) for k, v in at.items()}
    ws = P(1 << 30)
    assert pf.lib.pf_attention_bwd(_attention(), p["q"], p["k"], p["v"], p["t"], None, None, None, p["o"], p["lse"], p["g"], p["dq"], p["dk"], p["dv"],
                                   p["dt"], 0, ws, BIG, None) == 3


def test_attention_keys_with_room_behind_each_sequence():
    """An output that reaches into a sequence's keys is refused wherever that is."""
    at = dict(zip(SIZES, _places(*SIZES.values())))
    k = 1 << 24
    d = _attention(k_stride=(1 << 18, HK * D, D))
    p = {n: P(v) for n, v in at.items()}
    call = lambda dq: pf.lib.pf_attention_bwd(d, p["q"], P(k), p["v"], p["t"], None, None, None, p["o"], p["lse"], p["g"], P(dq), p["dk"],  # noqa: E731
                                              p["dv"], None, 0, P(1 << 30), BIG, None)
    assert call(k + (1 << 20) + 16) == 3 and call(k + 4 * L * HK * D - 16) == 3
