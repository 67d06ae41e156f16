"""Plain forms of rotary positions and of attention over a paged cache, in 64 bits or more, with the error bounds their tests use.
Not a test module."""
import numpy as np

import plain64

U = 2.0 ** -24        # an fp32 rounding is off by at most this, relative to the value


def rope(x, pos, freq, layout, scale=1.0, back=False):
    """x [rows, heads, dh], pos [rows], freq [rot / 2] -> turned rows and how far fp32 arithmetic may be off them (before the rounding
    to the array's type).  Angles in 80 bits: a product with a position of 2^31 has 33 bits behind the point left."""
    rot = 2 * len(freq)
    angle = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freq, np.longdouble)
    c, s = (np.asarray(f(angle), np.float64)[:, None] * scale for f in (np.cos, np.sin))
    if back:
        s = -s
    y, bound = np.array(x, np.float64), np.zeros(x.shape)
    a = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
    b = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    # sine and cosine: the remainder's conversion and product with 2 pi / 2^32 (3 roundings of at most pi / 4), two roundings of the
    # series, one of the product with the scale; then two roundings of the products: below 8 roundings of (|a| + |b|) |scale|
    size = 8 * U * abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    bound[..., a], bound[..., b] = size, size
    return y, bound


def attend(Q, q_pos, scale, K, V, k_pos):
    """Q [T, H, dh], K, V [n, Hkv, dh]: plain64.attend with each KV head serving H / Hkv query heads."""
    g = Q.shape[1] // K.shape[1]
    return plain64.attend(Q, q_pos, scale, np.repeat(K, g, 1), np.repeat(V, g, 1), k_pos)


def attend_bounds(Q, q_pos, scale, K, V, k_pos, O, lse, half, weight_half):
    """How far O and the log-sum-exp may be off.  A logit: dh products added in any order, each addition off by at most 2^-23 of what it
    adds up (accumulators may cut), and the product with the scale.  A weight: the error of its exponent, and the exponential's own
    (2^-21 covers ex2.approx).  Weights rounded on the way: weight_half.  Sums of n terms, joined from parts; one rounding of O (half)."""
    g = Q.shape[1] // K.shape[1]
    K, V, u, dh = np.repeat(K, g, 1), np.repeat(V, g, 1), 2.0 ** -23, Q.shape[2]
    tO, tL = half * np.abs(O), np.zeros_like(lse)
    see = k_pos[None, :] <= q_pos[:, None]
    for t in range(Q.shape[0]):
        k = see[t]
        n = int(k.sum())
        if n == 0:
            continue
        x = np.einsum("hd,khd->hk", Q[t], K[k]) * scale
        size = abs(scale) * np.einsum("hd,khd->hk", np.abs(Q[t]), np.abs(K[k]))
        spread = np.abs(x).max(1) + np.abs(lse[t])
        ex = ((dh + 8) * u * size).max(1) + 4 * u * spread + 2.0 ** -21
        p = np.exp(x - lse[t][:, None])
        A = np.einsum("hk,khd->hd", p, np.abs(V[k]))
        tO[t] += (1 + half) * (2 * ex + weight_half + 2 * (n + 16) * u)[:, None] * A
        tL[t] = ex + (n + 16) * u + 4 * u * np.abs(lse[t])
    return tO, tL
