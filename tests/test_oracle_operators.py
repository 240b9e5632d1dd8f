"""The double-precision definitions of oracle/operators.py pinned without them: gradients against differences, the
attention against a direct loop, the buckets against hand-counted ones."""
import numpy as np
import pytest

from oracle import operators as O


def _difference(f, x, dy, at, h=1e-6):
    up, down = x.copy(), x.copy()
    up[at] += h
    down[at] -= h
    return ((f(up) - f(down)) * dy).sum() / (2 * h)


@pytest.mark.parametrize("style,rot,norm", [("halves", 8, "rms"), ("pairs", 4, "rms"), ("pairs", 8, "none"), ("halves", 0, "rms")])
def test_qk_norm_rotate_gradients(style, rot, norm):
    rng = np.random.default_rng(1)
    x, dy, gamma = rng.standard_normal((2, 3, 2, 8)), rng.standard_normal((2, 3, 2, 8)), rng.uniform(0.5, 1.5, 8)
    pos = rng.integers(0, 50, (2, 3))
    kw = dict(norm=norm, rot_dim=rot, style=style, eps=1e-3)
    dx, dg = O.qk_norm_rotate_bwd(x, dy, gamma, pos, **kw)
    for at in [(0, 0, 0, 0), (1, 2, 1, 7), (0, 1, 1, 3)]:
        assert abs(_difference(lambda z: O.qk_norm_rotate_fwd(z, gamma, pos, **kw), x, dy, at) - dx[at]) < 1e-7
    if norm == "rms":
        for j in (0, 5):
            assert abs(_difference(lambda z: O.qk_norm_rotate_fwd(x, z, pos, **kw), gamma, dy, (j,)) - dg[j]) < 1e-7


def test_rotation_keeps_products_of_equal_distance():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((1, 1, 1, 16)), rng.standard_normal((1, 1, 1, 16))
    at = lambda x, p, s: O.qk_norm_rotate_fwd(x, None, np.array([[p]]), norm="none", style=s)  # noqa: E731
    for style in ("halves", "pairs"):
        a = (at(q, 3, style) * at(k, 11, style)).sum()
        b = (at(q, 1003, style) * at(k, 1011, style)).sum()
        assert abs(a - b) < 1e-9
        assert np.allclose(at(q, 0, style), q)


def test_buckets_by_hand():
    # 8 buckets up to distance 16, one side: 0 1 2 3, then borders at 4, 4 sqrt 2, 8, 8 sqrt 2
    got = [O.bucket(-n, 8, 16, False) for n in range(20)]
    assert got == [0, 1, 2, 3, 4, 4, 5, 5, 6, 6, 6, 6, 7, 7, 7, 7, 7, 7, 7, 7]
    assert O.bucket(5, 8, 16, False) == 0
    assert [O.bucket(n, 16, 16, True) for n in (-4, 0, 1, 4, 100)] == [4, 0, 9, 12, 15]


@pytest.mark.parametrize("causal", [False, True])
def test_attention_by_loop_and_differences(causal):
    rng = np.random.default_rng(3)
    Q, K, V = rng.standard_normal((2, 3, 4, 8)), rng.standard_normal((2, 5, 2, 8)), rng.standard_normal((2, 5, 2, 8))
    table, dO = rng.standard_normal((4, 4)), rng.standard_normal((2, 3, 4, 8))
    kw = dict(causal=causal, max_distance=4, bidirectional=not causal, q_start=[1, -1], q_len=[3, 2], kv_len=[5, 4])
    a = O.Attention(Q, K, V, table, **kw)
    for b, i, h in [(0, 0, 0), (0, 2, 3), (1, 0, 1), (1, 1, 2), (1, 2, 0)]:
        p, w, total = i + (1, -1)[b], np.zeros(8), 0.0
        for j in range((5, 4)[b]):
            if (causal and j > p) or i >= (3, 2)[b]:
                continue
            e = np.exp(Q[b, i, h] @ K[b, j, h // 2] / np.sqrt(8) + table[O.bucket(j - p, 4, 4, not causal), h])
            w, total = w + e * V[b, j, h // 2], total + e
        if total:
            assert np.allclose(a.O[b, i, h], w / total) and np.isclose(a.lse[b, h, i], np.log(total))
        else:
            assert not a.O[b, i, h].any() and a.lse[b, h, i] == -np.inf
    grads = a.backward(dO)
    for x, name, d in ((Q, 0, grads[0]), (K, 1, grads[1]), (V, 2, grads[2]), (table, 3, grads[3])):
        for flat in (0, x.size // 2, x.size - 1):
            at = np.unravel_index(flat, x.shape)
            args = [Q, K, V, table]
            f = lambda z: O.Attention(*[z if k == name else y for k, y in enumerate(args)], **kw).O  # noqa: B023, E731
            assert abs(_difference(f, x, dO, at) - d[at]) < 1e-7


def test_adamw_by_hand():
    p, m, v = O.adamw(1.0, 0.5, 0.0, 0.0, 1, 0.1, 0.9, 0.99, 0.0, 0.01)
    assert np.isclose(m, 0.05) and np.isclose(v, 0.0025)
    assert np.isclose(p, 0.999 - 0.1)  # the first step has the gradient's sign


def test_e4m3_scale_and_step():
    assert O.e4m3_scale(448.0) == 1.0 and O.e4m3_scale(449.0) == 2.0 and O.e4m3_scale(224.0) == 0.5
    assert O.e4m3_scale(0.0) == 2.0 ** -126
    assert O.e4m3_step(np.array([448.0, 1.0, 2.0 ** -7]))[0] == 32 and O.e4m3_step(np.array([1.0]))[0] == 0.125
    assert O.e4m3_step(np.array([2.0 ** -7]))[0] == 2.0 ** -9
