"""How far the GPU operators may be from the double-precision definitions, value by value, by arithmetic.

Every sum of n products in float32 is within (n + 1) E of the sum of the products' magnitudes, E = 2^-24 (half a step of
float32, relative); an output rounded to bf16 is off by half a step, 2^-8 relative; P and dS are rounded once, to the
inputs' type, before they are multiplied.  The bounds below are worst cases of that, not estimates."""
import numpy as np

E = 2.0 ** -24
HALF = {"f32": E, "bf16": 2.0 ** -8}
TINY = 1e-30


def assert_within(got, want, bound, name):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert (np.isfinite(got) == np.isfinite(want)).all(), f"{name}: not finite in other places"
    fine = np.isfinite(want)
    assert (got[~fine] == want[~fine]).all(), f"{name}: other infinities"
    over = np.where(fine, np.abs(np.where(fine, got - np.where(fine, want, 0), 0)) - (bound + TINY), -1)
    worst = np.unravel_index(np.argmax(over), over.shape) if over.size else ()
    assert over.size == 0 or over[worst] <= 0, f"{name}{list(worst)}: {got[worst]} for {want[worst]}, allowed {np.broadcast_to(bound, want.shape)[worst]}"


def _turn(positions):
    """How far sine and cosine may be off: the angle's fraction in float32 (2 pi times half a step of 1/2 at the most), the
    functions to 2 steps; in double the position's own digits."""
    return 8 * E + np.abs(positions.astype(np.float64)).max(initial=0) * 2.0 ** -50


def turn_bound(x, positions, dtype):
    """A rotation alone: two values mix."""
    return (HALF[dtype] + 3 * E + _turn(positions)) * 2 * np.abs(x).max(-1, keepdims=True)


def qk_bounds(x, dy, gamma, positions, dtype, D):
    """(output, dx, dgamma)."""
    # rstd: D squares summed, halved by the root, a root and a division
    turn = _turn(positions)
    k = (D / 2 + 12) * E
    g = np.ones(D) if gamma is None else np.abs(gamma)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-30)
    top = np.abs(x * r * g).max(-1, keepdims=True)  # (a turned value mixes two)
    y = HALF[dtype] * 2 * top + (k + turn) * 2 * top
    dtop = np.abs(dy).max(-1, keepdims=True)
    w = 2 * dtop * g.max()
    h = np.abs(x) * r
    mean = (w * h).mean(-1, keepdims=True)
    dx = (HALF[dtype] + (2 * D + 40) * E + 2 * turn) * r * (w + h * mean)
    rows = x.shape[0] * x.shape[1] * x.shape[2]
    dg = ((rows + D + 40) * E + 2 * turn) * (2 * dtop * h).sum((0, 1, 2))
    return y, dx, dg


def attention_bounds(a, dO, dtype):
    """Of an oracle.operators.Attention: (O, lse, dQ, dK, dV, dtable)."""
    u, D = HALF[dtype] if dtype == "bf16" else 0.0, a.Q.shape[-1]
    bO, bL = np.zeros_like(a.O), np.zeros_like(a.lse)
    bQ, bK, bV = np.zeros_like(a.Q), np.zeros_like(a.K), np.zeros_like(a.V)
    bT = np.zeros_like(a.table) if a.table is not None else None
    out = HALF[dtype]
    absQ, absK, absV = np.abs(a.Q), np.abs(a.K), np.abs(a.V)
    for (b, h), (nq, nk, bk, S, P) in a.parts.items():
        k = h // a.G
        q, kk, v = absQ[b, :nq, h], absK[b, :nk, k], absV[b, :nk, k]
        finite = np.where(np.isfinite(S), np.abs(S), 0.0)
        top = finite.max(1, keepdims=True)
        # the score, its scaling by a rounded scale and log2(e), the bias, the maximum taken off it
        eS = (D + 6) * E * abs(a.scale) * (q @ kk.T) + 6 * E * (finite + top + 1)
        n = nk + 40
        eLse = (P * eS).sum(1, keepdims=True) * 1.01 + n * E + 4 * E * (top + 1 + np.log(nk + 1.0))
        bL[b, h, :nq] = eLse[:, 0]
        eP = P * (1.01 * (eS + eLse) + 6 * E)
        PV = P @ v
        eO = eP @ v + u * PV + (n + 2) * E * PV
        bO[b, :nq, h] = eO + out * (np.abs(a.O[b, :nq, h]) + eO)
        if dO is None:
            continue
        g = np.abs(dO[b, :nq, h])
        signed = dO[b, :nq, h] @ a.V[b, :nk, k].T
        dP, edP = np.abs(signed), (D + 2) * E * (g @ v.T)
        delta = np.abs((P * signed).sum(1, keepdims=True))
        # delta from O, rounded (without a table gradient), or from P dP
        rounded = (g * bO[b, :nq, h]).sum(1, keepdims=True) + D * E * (g * PV).sum(1, keepdims=True)
        summed = (eP * dP + P * edP).sum(1, keepdims=True) + n * E * (P * dP).sum(1, keepdims=True)
        dS = np.abs(P * (signed - (P * signed).sum(1, keepdims=True)))

        def of(eDelta):
            return P * (edP + eDelta + 4 * E * (dP + delta)) + eP * (dP + delta)

        e = of(np.maximum(rounded, summed))
        full = e * (1 + u) + u * dS
        m = nq * a.G + 40
        bV[b, :nk, k] += (eP * (1 + u) + u * P + m * E * P).T @ g
        bQ[b, :nq, h] = abs(a.scale) * (full + n * E * dS) @ kk
        bK[b, :nk, k] += abs(a.scale) * (full + m * E * dS).T @ q
        if bT is not None:
            np.add.at(bT[:, h], bk, of(summed) + (nq + nk + 100) * E * dS)
    if dO is None:
        return bO, bL
    Q, K, V, T = a.backward(dO)
    return (bO, bL, bQ + out * (np.abs(Q) + bQ), bK + out * (np.abs(K) + bK), bV + out * (np.abs(V) + bV),
            None if bT is None else bT + E * np.abs(T))
