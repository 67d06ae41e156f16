"""Plain forms in 64 bits (numpy) of attention over [nuggets ; local tokens], of its gradient and of the 4-bit cache format,
with the error bounds their tests use.  Not a test module."""
import numpy as np

GROUP = 32
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # a rounding is off by at most this, relative to the value


def bf16_floor(x):
    """Largest bf16 number <= x, for float64 x that are float32 numbers."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.int64)
    cut = b & 0xffff0000
    cut = np.where((cut != b) & (b >> 31 == 1), cut + 0x10000, cut)
    return cut.astype(np.uint32).view(np.float32).astype(np.float64)


def quantise(x):
    """x [..., dh] -> codes (whole numbers), s, m per group, from the format's definition by search over bf16 numbers."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    bad = ~np.isfinite(g).all(-1)
    gf = np.where(bad[..., None], 0.0, g)
    m = bf16_floor(gf.min(-1))
    span = gf.max(-1) - m
    # candidates around span / 15: the least bf16 number s with 15 s >= span
    bits = (np.asarray(span / 15.0, np.float32).view(np.uint32) >> 16).astype(np.int64)
    s = np.full(span.shape, np.inf)
    for d in (2, 1, 0, -1, -2):
        c = (np.maximum(bits + d, 0) << 16).astype(np.uint32).view(np.float32).astype(np.float64)
        s = np.where(15.0 * c >= span, np.minimum(s, c), s)
    with np.errstate(over="ignore"):
        bad |= ~(span.astype(np.float32) <= np.finfo(np.float32).max) | ~np.isfinite(m)
    # x - m as t + e exactly (two-sum), since a feature may lie closer to a border than 64 bits show in the difference alone
    mm, ss = m[..., None], s[..., None]
    with np.errstate(all="ignore"):
        t = gf - mm
        z = t - gf
        e = (gf - (t - z)) + (-mm - z)
        c = np.where(ss > 0, np.floor(t / ss), 0.0)
        c = np.where(bad[..., None], 0.0, c)
        border = (c + 0.5) * ss
        above = (t > border) | ((t == border) & ((e > 0) | ((e == 0) & (c % 2 == 1))))
        c = np.where((ss > 0) & ~bad[..., None], c + above, 0.0).astype(np.int64)
    return c.reshape(x.shape), np.where(bad, np.nan, s), np.where(bad, 0.0, m)


def pack(c, s, m):
    """codes [rows, H, dh], s, m [rows, H, groups] -> bytes [rows, H, dh / 2], words [rows, H, groups]."""
    codes = (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    hi = lambda v: (np.asarray(v, np.float32).view(np.uint32) >> 16).astype(np.uint32)  # noqa: E731
    return codes, (np.where(np.isnan(s), np.uint32(0x7fc0), hi(s)) | (hi(m) << 16)).astype(np.uint32).view(np.int32)


def values(codes, words):
    """float64 values that packed rows stand for."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],)).astype(np.float64)
    w = words.view(np.uint32)
    s = (w << 16).view(np.float32).astype(np.float64)
    m = (w & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)
    g = c.reshape(c.shape[:-1] + (c.shape[-1] // GROUP, GROUP))
    with np.errstate(invalid="ignore"):
        return (m[..., None] + g * s[..., None]).reshape(c.shape)


def attend(Q, q_pos, scale, K, V, k_pos):
    """Q [T, H, dh], K, V [n, H, dh] -> O [T, H, dh], lse [T, H]; a key is visible where its position is not behind the query's."""
    T, H, dh = Q.shape
    O, lse = np.zeros((T, H, V.shape[2])), np.full((T, H), -np.inf)
    see = k_pos[None, :] <= q_pos[:, None]
    for t in range(T):
        k = see[t]
        if not k.any():
            continue
        x = np.einsum("hd,khd->hk", Q[t], K[k]) * scale
        top = x.max(1, keepdims=True)
        p = np.exp(x - top)
        tot = p.sum(1, keepdims=True)
        lse[t] = (np.log(tot) + top)[:, 0]
        O[t] = np.einsum("hk,khd->hd", p / tot, V[k])
    return O, lse


def attend_backward(Q, q_pos, scale, K, V, k_pos, O, lse, dO):
    """dQ, dK, dV and dlogit [n] (sum over heads and queries of the gradient at the softmax's argument)."""
    see = (k_pos[None, :] <= q_pos[:, None])[None]                      # [1, T, n]
    x = np.einsum("thd,khd->htk", Q, K) * scale
    with np.errstate(over="ignore", invalid="ignore"):
        P = np.where(see, np.exp(x - lse.T[:, :, None]), 0.0)
    D = np.einsum("thd,thd->ht", dO, O)[:, :, None]
    dS = P * (np.einsum("thd,khd->htk", dO, V) - D)
    return (np.einsum("htk,khd->thd", dS, K) * scale, np.einsum("htk,thd->khd", dS, Q) * scale, np.einsum("htk,thd->khd", P, dO),
            dS.sum((0, 1)), P, dS)


def logit_bound(Q, K, scale, dh, low=None):
    """How far an fp32 logit may be from the exact one: dh products added in any order (and, over a 4-bit cache, the part
    q . m beside them), each operation off by at most 2^-24 of what it adds up."""
    if Q.shape[0] == 0 or K.shape[0] == 0:
        return 0.0
    a = np.abs(K) if low is None else np.abs(K) + 2.0 * np.abs(low)
    size = abs(scale) * max(float(np.max(np.abs(Q[:, h]) @ a[:, h].T)) for h in range(Q.shape[1]))
    return (dh + 16) * 2.0 ** -24 * size


def backward_with_bounds(Q, q_pos, scale, K, V, k_pos, O, lse, dO, half, weight_half=0.0):
    """attend_backward and how far each result may be off.  fp32 operations, each off by at most 2^-24 of what it adds up (2^-23
    allowed, for accumulators that cut); results rounded once (half); P and dS rounded on the way where weight_half > 0."""
    dQ, dK, dV, dx, P, dS = attend_backward(Q, q_pos, scale, K, V, k_pos, O, lse, dO)
    T, n, dh, u = Q.shape[0], K.shape[0], Q.shape[2], 2.0 ** -23
    if T == 0 or n == 0:
        return (dQ, dK, dV, dx), (np.zeros_like(dQ), np.zeros_like(dK), np.zeros_like(dV), np.zeros_like(dx))
    eins = np.einsum
    size_x = abs(scale) * eins("thd,khd->htk", np.abs(Q), np.abs(K))
    fin = np.where(np.isfinite(lse), np.abs(lse), 0.0).T[:, :, None]
    ex = (dh + 8) * u * size_x + 4 * u * (size_x + fin) + 2.0 ** -21                 # relative error of P
    dP = eins("thd,khd->htk", dO, V) - eins("thd,thd->ht", dO, O)[:, :, None]
    ed = (dh + 8) * u * (eins("thd,khd->htk", np.abs(dO), np.abs(V)) + eins("thd,thd->ht", np.abs(dO), np.abs(O))[:, :, None])
    eP = P * (ex + weight_half)
    eS = P * (ex * np.abs(dP) + (1.0 + ex) * ed)
    eSr = eS + weight_half * (np.abs(dS) + eS)                                       # as the products see it
    aS, sc = np.abs(dS), abs(scale)
    tQ = half * np.abs(dQ) + sc * ((1 + half) * eins("htk,khd->thd", eSr, np.abs(K)) + (n + 8) * u * eins("htk,khd->thd", aS, np.abs(K)))
    tK = half * np.abs(dK) + sc * ((1 + half) * eins("htk,thd->khd", eSr, np.abs(Q)) + (T + 8) * u * eins("htk,thd->khd", aS, np.abs(Q)))
    tV = half * np.abs(dV) + (1 + half) * eins("htk,thd->khd", eP, np.abs(dO)) + (T + 8) * u * eins("htk,thd->khd", P, np.abs(dO))
    tx = eS.sum((0, 1)) + (T * Q.shape[1] + 8) * u * aS.sum((0, 1))
    return (dQ, dK, dV, dx), (tQ, tK, tV, tx)
