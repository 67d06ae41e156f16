"""The plain 64-bit forms the GPU tests compare with: the 4-bit format against its definition by enumeration, the gradient
against differences."""
import numpy as np
import plain64


def test_format_by_enumeration():
    rs = np.random.RandomState(0)
    x = np.float32(rs.standard_normal((40, 2, 64)) * 10.0 ** rs.randint(-3, 4, (40, 1, 1))).astype(np.float64)
    x[0] = 0.25
    x[1, 0, :32] = np.arange(32) * 0.5
    c, s, m = plain64.quantise(x)
    assert c.min() >= 0 and c.max() <= 15
    g, cg = x.reshape(40, 2, 2, 32), c.reshape(40, 2, 2, 32)
    ok = lambda v: np.array_equal(np.float32(v).view(np.uint32) & 0xffff, np.zeros(v.shape, np.uint32))  # noqa: E731
    assert ok(s) and ok(m)
    lo, hi = g.min(-1), g.max(-1)
    up = (np.float32(m).view(np.int32) + np.where(m < 0, -0x10000, 0x10000)).astype(np.int32).view(np.float32).astype(np.float64)
    assert np.all(m <= lo) and np.all((up > lo) | (m == 0))
    less = np.where(s > 0, (np.float32(s).view(np.int32) - 0x10000).view(np.float32), -1.0)
    assert np.all(15.0 * s >= hi - m) and np.all(15.0 * less < hi - m)
    # each code is the nearest of the sixteen values, the even one of two equally near
    for code in range(16):
        here, mine = np.abs(m[..., None] + code * s[..., None] - g), np.abs(m[..., None] + cg * s[..., None] - g)
        eps = 1e-12 * s[..., None]
        assert np.all((mine <= here + eps))
        tie = (np.abs(mine - here) <= eps) & (cg != code) & (s[..., None] > 0)
        assert np.all(cg[tie] % 2 == 0)
    codes, words = plain64.pack(c, s, m)
    assert np.array_equal(plain64.values(codes, words), (m[..., None] + cg * s[..., None]).reshape(x.shape))


def test_gradient_by_differences():
    rs = np.random.RandomState(1)
    T, n, H, dh = 4, 7, 2, 8
    Q, K, V, dO = (rs.standard_normal(s) for s in ((T, H, dh), (n, H, dh), (n, H, dh), (T, H, dh)))
    q_pos, k_pos, scale = np.array([-1, 2, 4, 9]), np.array([0, 1, 2, 3, 5, 8, 30]), 0.4
    loss = lambda q, k, v: float(np.sum(plain64.attend(q, q_pos, scale, k, v, k_pos)[0] * dO))  # noqa: E731
    O, lse = plain64.attend(Q, q_pos, scale, K, V, k_pos)
    assert np.isneginf(lse[0]).all() and np.all(O[0] == 0)
    dQ, dK, dV, dx, P, dS = plain64.attend_backward(Q, q_pos, scale, K, V, k_pos, O, lse, dO)
    e = 1e-6
    for X, dX, at in ((Q, dQ, 0), (K, dK, 1), (V, dV, 2)):
        for _ in range(40):
            i = tuple(rs.randint(0, s) for s in X.shape)
            a, b = X.copy(), X.copy()
            a[i] += e
            b[i] -= e
            args = [Q, K, V]
            hi = loss(*[a if k == at else t for k, t in enumerate(args)])
            lo = loss(*[b if k == at else t for k, t in enumerate(args)])
            assert abs((hi - lo) / (2 * e) - dX[i]) < 1e-7
    # a key's score enters every logit of that key (an extra feature of q that is 1 / scale, of k that is the score)
    Q1 = np.concatenate([Q, np.full((T, H, 1), 1.0 / scale)], -1)
    for j in range(n):
        def shifted(t):
            k1 = np.concatenate([K, np.zeros((n, H, 1))], -1)
            k1[j, :, -1] = t
            return float(np.sum(plain64.attend(Q1, q_pos, scale, k1, V, k_pos)[0] * dO))
        assert abs((shifted(e) - shifted(-e)) / (2 * e) - dx[j]) < 1e-7
    assert np.all(P[:, :, 6] == 0) and np.all(dK[6] == 0) and np.all(dQ[0] == 0)
