"""Plain double-precision definitions of what a Transformer layer has between its factorized projections and of the
optimizer's step -- TEST INFRASTRUCTURE, like the rest of this package: numpy loops and products written from the
formulas in include/pufferfish.h, sharing no code with the GPU library.
"""
import numpy as np


# ------------------------------------------------------------------ norms and rotation

def _turn(u, positions, rot_dim, theta, style, back=False):
    """u[B, L, H, D] with its first rot_dim values turned (or turned back)."""
    y = u.copy()
    for i in range(rot_dim // 2):
        a = positions.astype(np.float64) * float(theta) ** (-2.0 * i / rot_dim)  # [B, L]
        c, s = np.cos(a)[:, :, None], np.sin(a)[:, :, None] * (-1.0 if back else 1.0)
        p, q = (i, i + rot_dim // 2) if style == "halves" else (2 * i, 2 * i + 1)
        y[..., p] = u[..., p] * c - u[..., q] * s
        y[..., q] = u[..., p] * s + u[..., q] * c
    return y


def qk_norm_rotate_fwd(x, gamma, positions, norm="rms", eps=1e-6, rot_dim=None, theta=10000.0, style="halves"):
    """One of the two tensors, x[B, L, H, D]."""
    u = x
    if norm == "rms":
        u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if gamma is None else gamma)
    return _turn(u, positions, x.shape[-1] if rot_dim is None else rot_dim, theta, style)


def qk_norm_rotate_bwd(x, dy, gamma, positions, norm="rms", eps=1e-6, rot_dim=None, theta=10000.0, style="halves"):
    """(dx, dgamma)."""
    D = x.shape[-1]
    du = _turn(dy, positions, D if rot_dim is None else rot_dim, theta, style, back=True)
    if norm != "rms":
        return du, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    g = np.ones(D) if gamma is None else gamma
    # du_k/dx_j = g_k (r [j = k] - x_k x_j r^3 / D)
    w = du * g
    dx = r * w - x * r ** 3 * (w * x).sum(-1, keepdims=True) / D
    return dx, (du * x * r).sum((0, 1, 2))


# ------------------------------------------------------------------ attention

def bucket(dist, buckets, max_distance, bidirectional):
    """Bucket of the distance key - query, in exact arithmetic."""
    side, first = buckets, 0
    if bidirectional:
        side = buckets // 2
        first = side if dist > 0 else 0
    elif dist > 0:
        return 0
    n, e = abs(dist), side // 2
    if n < e:
        return first + n
    m, k = side - e, 0
    # floor(m log(n/e) / log(D/e)): the most k with (D/e)^k <= (n/e)^m, in whole numbers
    left, right = e ** m * max_distance, n ** m * e  # (D/e)^(k + 1) e^(m + k + 1), (n/e)^m e^(m + k + 1)
    while k < m - 1 and left <= right:
        k, left, right = k + 1, left * max_distance, right * e
    return first + e + k


class Attention:
    """All arrays of one call; see pf_attention_fwd.  O, lse; backward(dO) -> dQ, dK, dV, dtable."""

    def __init__(self, Q, K, V, table=None, causal=False, scale=None, max_distance=128, bidirectional=True, q_start=None,
                 q_len=None, kv_len=None):
        B, Lq, H, D = Q.shape
        Lk, Hk = K.shape[1:3]
        self.Q, self.K, self.V, self.table = Q, K, V, table
        self.scale = scale = D ** -0.5 if scale is None else scale
        self.G = H // Hk
        self.O, self.lse = np.zeros_like(Q), np.full((B, H, Lq), -np.inf)
        self.parts = {}
        for b in range(B):
            nq = Lq if q_len is None else min(max(int(q_len[b]), 0), Lq)
            nk = Lk if kv_len is None else min(max(int(kv_len[b]), 0), Lk)
            if nq == 0 or nk == 0:
                continue
            pos = (0 if q_start is None else int(q_start[b])) + np.arange(nq)
            rel = np.arange(nk)[None] - pos[:, None]
            seen = rel <= 0 if causal else np.ones_like(rel, dtype=bool)
            u = None
            if table is not None:
                kinds, place = np.unique(rel, return_inverse=True)
                kinds = [bucket(int(np.clip(x, -2 * max_distance, 2 * max_distance)), table.shape[0], max_distance, bidirectional)
                         for x in kinds]
                u = np.array(kinds)[place.reshape(rel.shape)]
            for h in range(H):
                S = scale * Q[b, :nq, h] @ K[b, :nk, h // self.G].T
                if u is not None:
                    S = S + table[u, h]
                S = np.where(seen, S, -np.inf)
                top = S.max(1, keepdims=True)
                E = np.exp(S - np.where(np.isfinite(top), top, 0.0))
                total = E.sum(1, keepdims=True)
                P = E / np.where(total > 0, total, 1.0)
                with np.errstate(divide="ignore"):
                    self.lse[b, h, :nq] = (top + np.log(total))[:, 0]
                self.O[b, :nq, h] = P @ V[b, :nk, h // self.G]
                self.parts[b, h] = (nq, nk, u, S, P)

    def backward(self, dO):
        dQ, dK, dV = np.zeros_like(self.Q), np.zeros_like(self.K), np.zeros_like(self.V)
        dT = None if self.table is None else np.zeros_like(self.table)
        for (b, h), (nq, nk, u, _, P) in self.parts.items():
            k = h // self.G
            g = dO[b, :nq, h]
            dP = g @ self.V[b, :nk, k].T
            dS = P * (dP - (P * dP).sum(1, keepdims=True))
            dV[b, :nk, k] += P.T @ g
            dQ[b, :nq, h] = self.scale * dS @ self.K[b, :nk, k]
            dK[b, :nk, k] += self.scale * dS.T @ self.Q[b, :nq, h]
            if dT is not None:
                np.add.at(dT[:, h], u, dS)
        return dQ, dK, dV, dT


# ------------------------------------------------------------------ AdamW

def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay):
    """Step number t: (p, m, v)."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * weight_decay)
    return p - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps), m, v


def e4m3_scale(top):
    """The smallest power of two from 2^-126 on with top / scale <= 448."""
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def e4m3_step(x):
    """The distance between neighbouring 8-bit values around |x| <= 448."""
    x = np.abs(x)
    e = np.floor(np.log2(np.where(x > 0, x, 1.0)))
    return 2.0 ** (np.maximum(e, -6) - 3)
