"""The 4-bit nugget cache on the GPU: append and expansion bit for bit against the format's definition in 64 bits, attention over
it against the plain form over the values the codes stand for."""
import numpy as np
import pytest
import torch

import plain64
from paper_2310_02409_b200 import api, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _cache(rows, H, dh, fill=0x5a):
    return (torch.full((rows, H, 2, dh // 2), fill, dtype=torch.uint8, device="cuda"),
            torch.full((rows, H, 2, dh // 32), 0x12345678, dtype=torch.int32, device="cuda"),
            torch.full((rows,), -7, dtype=torch.int32, device="cuda"))


def _hard_rows(H, dh, dtype):
    """Rows whose groups are what the format finds hard, in the storage type."""
    rs = np.random.RandomState(5)
    rows = []
    rows.append(np.zeros((H, dh)))                                            # s = 0
    rows.append(np.full((H, dh), -1.7))                                       # constant (fp32: not a bf16 number)
    rows.append(np.tile(np.arange(32) * 0.5 - 8.0, H * dh // 32))             # many values exactly on borders
    rows.append(np.tile(np.concatenate([[-1.5, 13.5], np.tile([1e-10, -1e-10, 0.0, 1e-30, -1e-30], 6)]), H * dh // 32))  # borders decided far below fp32
    rows.append(rs.standard_normal(H * dh) * 1e-40)                           # subnormal
    rows.append(rs.standard_normal(H * dh) * 1e37)
    rows.append(rs.standard_normal(H * dh) * 10.0 ** rs.randint(-30, 30, H * dh))
    rows.append(np.tile(np.concatenate([[0.0, 15.0], np.arange(30) / 2.0]), H * dh // 32))   # every half step
    rows.append(np.where(rs.randint(0, 200, H * dh) == 0, np.nan, rs.standard_normal(H * dh)))
    rows.append(np.where(rs.randint(0, 200, H * dh) == 0, np.inf, rs.standard_normal(H * dh)))
    rows.append(np.where(rs.randint(0, 200, H * dh) == 0, -np.inf, rs.standard_normal(H * dh)))
    rows.append(np.where(np.arange(H * dh) % 32 == 3, 3.3e38, -3.3e38) * (np.arange(H * dh) % 64 < 32))   # span overflows
    x = np.stack([np.asarray(r).reshape(H, dh) for r in rows])
    return torch.from_numpy(x).to(torch.float32).to(dtype)


@pytest.mark.parametrize("dtype,H,dh", [(BF, 32, 128), (F32, 4, 64), (BF, 3, 64), (F32, 5, 128), (BF, 1, 64), (F32, 1, 128)])
def test_gather_q4_is_the_format_bit_for_bit(dodo, dtype, H, dh):
    lens, ks, used = [40, 0, 300, 1, 64], [17, 0, 31, 1, 64], [3, 0, 0, 1, 2]
    seq_off, nug_off = inputs.offsets(lens), inputs.offsets(ks)
    cache_off = inputs.offsets([k + u + 2 for k, u in zip(ks, used)])
    N, rows = int(seq_off[-1]), int(cache_off[-1])
    K = inputs.randn((N, H, dh), "q4", H, dh, "K", dtype=dtype)
    V = inputs.randn((N, H, dh), "q4", H, dh, "V", std=3.0, dtype=dtype)
    hard = _hard_rows(H, dh, dtype)
    K[40:40 + len(hard)] = hard
    V[340:340 + 1] = hard[6:7]
    V[341:341 + len(hard)] = hard
    rs = np.random.RandomState(1)
    idx = [np.sort(rs.permutation(n)[:k]).astype(np.int32) for n, k in zip(lens, ks)]
    idx[2] = np.arange(31, dtype=np.int32)                    # the hard rows are selected
    idx = np.concatenate(idx)
    pos_base = np.array([5, 6, 700, 8, 9], np.int32)
    q4, sc, pos = _cache(rows, H, dh)
    before = [t.cpu().numpy().copy() for t in (q4, sc, pos)]
    clen = np.asarray(used, np.int32)
    dodo.gather_kv_q4(K.cuda(), V.cuda(), seq_off, _cuda(idx), nug_off, pos_base, q4, sc, pos, cache_off, clen)
    torch.cuda.synchronize()
    assert clen.tolist() == [k + u for k, u in zip(ks, used)]
    got = [t.cpu().numpy() for t in (q4, sc, pos)]
    want = [b.copy() for b in before]
    for b in range(5):
        rows_b = seq_off[b] + idx[nug_off[b]:nug_off[b + 1]]
        at = slice(int(cache_off[b]) + used[b], int(cache_off[b]) + used[b] + ks[b])
        for kv, X in enumerate((K, V)):
            c, w = plain64.pack(*plain64.quantise(X.float().numpy()[rows_b]))
            want[0][at, :, kv], want[1][at, :, kv] = c, w
        want[2][at] = pos_base[b] + idx[nug_off[b]:nug_off[b + 1]]
    for name, g, w in zip(("steps", "codes", "positions"), (got[1], got[0], got[2]), (want[1], want[0], want[2])):
        off = np.argwhere(g != w)
        assert len(off) == 0, (name, len(off), off[:4].tolist(), g[tuple(off[0])], w[tuple(off[0])])
    # what the codes stand for is at most half a step from the row
    c, s, m = plain64.quantise(K.float().numpy()[:40])
    v = plain64.values(*plain64.pack(c, s, m))
    assert np.all(np.abs(v - K.float().numpy()[:40]) <= np.repeat(s, 32, -1) * 0.5 * (1 + 1e-12))

    # expansion: one rounding to fp32, for bf16 one more; rows that are not in use stay
    Ke, Ve = torch.full((rows, H, dh), 9.0, dtype=dtype, device="cuda"), torch.full((rows, H, dh), -9.0, dtype=dtype, device="cuda")
    dodo.expand_kv_q4(q4, sc, cache_off, clen, Ke, Ve)
    torch.cuda.synchronize()
    live = np.zeros(rows, bool)
    for b in range(5):
        live[cache_off[b]:cache_off[b] + clen[b]] = True
    for kv, (E, fill) in enumerate(((Ke, 9.0), (Ve, -9.0))):
        with np.errstate(over="ignore", invalid="ignore"):
            ref = torch.from_numpy(plain64.values(got[0][:, :, kv], got[1][:, :, kv]).astype(np.float32)).to(dtype)
        assert torch.equal(torch.isnan(E.cpu()[live]), torch.isnan(ref[live]))
        assert torch.equal(torch.nan_to_num(E.cpu()[live].float()), torch.nan_to_num(ref[live].float()))
        assert bool((E.cpu()[~live].float() == fill).all())
    assert dodo.device_status() == 0


def test_gather_q4_appends_many_sequences_and_matches_gather(dodo):
    # 70 sequences: two launch groups; the cache equals quantising what dodo_gather_kv stores
    H, dh, B = 2, 64, 70
    rs = np.random.RandomState(3)
    lens = [int(x) for x in rs.randint(0, 40, B)]
    ks = [n // 3 for n in lens]
    seq_off, nug_off, cache_off = inputs.offsets(lens), inputs.offsets(ks), inputs.offsets([2 * k for k in ks])
    K, V = (inputs.randn((int(seq_off[-1]), H, dh), "q4many", n, dtype=BF).cuda() for n in "KV")
    idx = _cuda(np.concatenate([np.sort(rs.permutation(n)[:k]) for n, k in zip(lens, ks)]).astype(np.int32))
    rows = int(cache_off[-1])
    q4, sc, pos = _cache(rows, H, dh)
    cK, cV = torch.zeros((rows, H, dh), dtype=BF, device="cuda"), torch.zeros((rows, H, dh), dtype=BF, device="cuda")
    cpos = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    cl4, cl = np.zeros(B, np.int32), np.zeros(B, np.int32)
    for base in (0, 1000):
        pb = np.full(B, base, np.int32)
        dodo.gather_kv_q4(K, V, seq_off, idx, nug_off, pb, q4, sc, pos, cache_off, cl4)
        dodo.gather_kv(K, V, seq_off, idx, nug_off, pb, cK, cV, cpos, cache_off, cl)
    torch.cuda.synchronize()
    assert np.array_equal(cl4, cl) and torch.equal(pos, cpos)
    for kv, X in enumerate((cK, cV)):
        c, w = plain64.pack(*plain64.quantise(X.float().cpu().numpy()))
        assert np.array_equal(q4.cpu().numpy()[:, :, kv], c) and np.array_equal(sc.cpu().numpy()[:, :, kv], w)


def test_gather_q4_bad_index_is_reported_not_followed(libdodo):
    ctx = api.Dodo(0)
    H, dh = 2, 64
    K = torch.ones((10, H, dh), device="cuda")
    q4, sc, pos = _cache(4, H, dh)
    b4, bs = q4.clone(), sc.clone()
    clen = np.zeros(1, np.int32)
    ctx.gather_kv_q4(K, K, [0, 10], _cuda(np.array([0, -1, 10, 9], np.int32)), [0, 4], [0], q4, sc, pos, [0, 4], clen)
    torch.cuda.synchronize()
    assert ctx.device_status() == api.DEV_BAD_INDEX
    assert torch.equal(q4[1:3], b4[1:3]) and torch.equal(sc[1:3], bs[1:3]) and pos.tolist() == [0, -7, -7, 9]
    ctx.reset()
    assert ctx.device_status() == 0
    ctx.close()


# ---- attention --------------------------------------------------------------------------------------------------------
def _problem(tag, dtype, H, dh, tqs, clens, llens, inside=False, slack=2, kstd=1.0, vstd=2.0, scale=None):
    """A ragged batch over a 4-bit cache; row regions have slack rows that hold NaN groups, the local array NaN rows."""
    rs = np.random.RandomState(inputs.seed_for(tag) % 2 ** 32)
    B = len(tqs)
    p = dict(B=B, H=H, dh=dh, dtype=dtype, scale=dh ** -0.5 if scale is None else scale)
    p["q_off"], p["cache_off"] = inputs.offsets(tqs), inputs.offsets([c + slack for c in clens])
    p["clen"], p["llen"] = np.asarray(clens, np.int32), np.asarray(llens, np.int32)
    p["loc_off"] = inputs.offsets([n + slack for n in llens])[:-1].copy()
    rows, lrows = int(p["cache_off"][-1]), int(sum(n + slack for n in llens))
    span = [5 * c + 3 for c in clens]
    p["loc_pos0"] = np.asarray(span, np.int32)
    p["q_pos0"] = np.asarray([s // 2 - 2 if inside else s + n - t for s, n, t in zip(span, llens, tqs)], np.int32)
    cpos = np.full(rows, 0, np.int32)
    kv = [kstd * rs.standard_normal((rows, H, dh)), vstd * rs.standard_normal((rows, H, dh))]
    packed = [plain64.pack(*plain64.quantise(np.asarray(torch.from_numpy(x).float().to(dtype).float().numpy()))) for x in kv]
    codes, words = np.stack([packed[0][0], packed[1][0]], 2), np.stack([packed[0][1], packed[1][1]], 2)
    loc = [torch.from_numpy(rs.standard_normal((lrows, H, dh))).to(dtype) for _ in range(2)]
    live_l = np.zeros(lrows, bool)
    for b in range(B):
        c0 = int(p["cache_off"][b])
        cpos[c0:c0 + clens[b]] = np.sort(rs.permutation(span[b])[:clens[b]])
        words[c0 + clens[b]:int(p["cache_off"][b + 1])] = 0x7fc07fc0
        live_l[p["loc_off"][b]:p["loc_off"][b] + llens[b]] = True
    for t in loc:
        t[torch.from_numpy(~live_l)] = float("nan")
    p["codes"], p["words"], p["cpos"], p["loc"] = codes, words, cpos, loc
    p["Q"] = torch.from_numpy(rs.standard_normal((int(p["q_off"][-1]), H, dh))).to(dtype)
    return p


def _run_q4(dodo, p, workspace=None, lse=True, stream=None):
    d = dict(O=torch.full(p["Q"].shape, float("nan"), dtype=p["dtype"], device="cuda"),
             lse=torch.full(p["Q"].shape[:2], float("nan"), device="cuda") if lse else None)
    if workspace is None:
        workspace = torch.empty(dodo.attend_q4_workspace_bytes(p["H"], p["dh"], p["codes"].shape[0]), dtype=torch.uint8, device="cuda")
    dodo.attend_q4(p["Q"].cuda(), p["q_off"], p["q_pos0"], p["scale"], _cuda(p["codes"]), _cuda(p["words"]), _cuda(p["cpos"]),
                   p["cache_off"], p["clen"], p["loc"][0].cuda(), p["loc"][1].cuda(), p["loc_off"], p["llen"], p["loc_pos0"],
                   d["O"], d["lse"], workspace)
    torch.cuda.synchronize()
    return d["O"], d["lse"]


def _reference(p, rounded=False):
    """O, lse and the bounds on their errors, sequence by sequence."""
    K, V = plain64.values(p["codes"][:, :, 0], p["words"][:, :, 0]), plain64.values(p["codes"][:, :, 1], p["words"][:, :, 1])
    low = np.repeat((p["words"][:, :, 0].view(np.uint32) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64), 32, -1)
    Q, lK, lV = _f64(p["Q"]), _f64(p["loc"][0]), _f64(p["loc"][1])
    O, lse, tO, tL = np.zeros(Q.shape), np.zeros(Q.shape[:2]), np.zeros(Q.shape), np.zeros(Q.shape[:2])
    half = plain64.HALF["bf16" if p["dtype"] == BF else "f32"]
    for b in range(p["B"]):
        q, c = slice(int(p["q_off"][b]), int(p["q_off"][b + 1])), slice(int(p["cache_off"][b]), int(p["cache_off"][b]) + int(p["clen"][b]))
        l = slice(int(p["loc_off"][b]), int(p["loc_off"][b]) + int(p["llen"][b]))
        k, v = np.concatenate([K[c], lK[l]]), np.concatenate([V[c], lV[l]])
        kpos = np.concatenate([p["cpos"][c], p["loc_pos0"][b] + np.arange(p["llen"][b])])
        qpos = p["q_pos0"][b] + np.arange(q.stop - q.start)
        O[q], lse[q] = plain64.attend(Q[q], qpos, p["scale"], k, v, kpos)
        if not len(k) or q.stop == q.start:
            continue
        d = plain64.logit_bound(Q[q], k, p["scale"], p["dh"], np.concatenate([low[c], np.zeros_like(lK[l])]))
        extra = 0.0
        if rounded:     # keys and values rounded to bf16, weights rounded to bf16: each off by at most 2^-8 of itself
            d += 2.0 ** -8 * abs(p["scale"]) * max(float(np.max(np.abs(Q[q][:, h]) @ np.abs(k[:, h]).T)) for h in range(p["H"]))
            extra = 2.0 ** -8 + 2.0 ** -8
        w = 2.0 * d + extra + 2.0 ** -20 + len(k) * 2.0 ** -24     # relative error of a weight: its logit's, the exponential's, the sum's
        tO[q] = half * np.abs(O[q]) + w * np.max(np.abs(v))
        tL[q] = d + 2.0 ** -20 + len(k) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse[q]), lse[q], 0.0))
    return O, lse, tO, tL


def _check(p, O, lse, rounded=False):
    rO, rL, tO, tL = _reference(p, rounded)
    gO = _f64(O)
    assert np.all(np.isfinite(gO))
    assert np.all(np.abs(gO - rO) <= tO), float(np.max(np.abs(gO - rO) - tO))
    if lse is not None:
        gL = _f64(lse)
        empty = np.isneginf(rL)
        assert np.array_equal(np.isneginf(gL), empty)
        assert np.all(np.abs(gL[~empty] - rL[~empty]) <= tL[~empty])
        assert np.all(gO[empty] == 0.0)


SHAPES = [
    # dtype, H, dh, query tokens, cached rows, local rows
    (BF, 32, 128, [1] * 8, [205] * 8, [64] * 8),
    (BF, 2, 128, [1, 1, 1, 1, 1], [0, 1, 63, 129, 1000], [1, 0, 65, 7, 130]),
    (F32, 3, 64, [1, 1, 1], [700, 5, 0], [64, 1, 33]),
    (F32, 2, 128, [2, 1, 2], [33, 300, 64], [2, 9, 70]),
    (BF, 3, 64, [3, 4, 1, 0, 2], [257, 31, 8, 40, 0], [5, 4, 1, 3, 66]),
    (F32, 4, 64, [16], [52], [16]),
    (BF, 1, 128, [7], [4097], [100]),
    (BF, 40, 128, [1], [3277], [64]),
    (BF, 5, 64, [13, 31], [100, 900], [31, 40]),
    (BF, 2, 128, [2, 3, 0, 8, 1], [700, 16, 33, 205, 1], [2, 40, 7, 64, 130]),
    (BF, 3, 128, [9, 16, 5], [64, 1000, 0], [80, 16, 333]),
    (BF, 1, 128, [31], [2000], [31]),
    (BF, 2, 128, [17, 6], [0, 81], [17, 1000]),
    (BF, 2, 64, [2, 3, 0, 8, 1], [700, 16, 33, 205, 1], [2, 40, 7, 64, 130]),
    (BF, 3, 64, [9, 40, 5], [64, 1000, 0], [80, 40, 333]),
]


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attend_q4_against_plain(dodo, case, inside):
    dtype, H, dh, tqs, cl, ll = SHAPES[case]
    p = _problem(("q4a", case, inside), dtype, H, dh, tqs, cl, ll, inside)
    O, lse = _run_q4(dodo, p)
    _check(p, O, lse)
    O2, lse2 = _run_q4(dodo, p)                      # bit for bit the same again
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    O3, _ = _run_q4(dodo, p, lse=False)
    assert torch.equal(O, O3)
    assert dodo.device_status() == 0


def test_attend_q4_split_targets(libdodo):
    ctx = api.Dodo(0)
    p = _problem("q4split", BF, 3, 128, [1, 1, 2], [2000, 37, 500], [70, 0, 3])
    for target in (1, 7, 64, 4096):
        ctx.set_tuning(api.TUNE_ATTEND_TARGET_BLOCKS, target)
        _check(p, *_run_q4(ctx, p))
    ctx.close()


def test_attend_q4_masked_nan_rows_do_not_count(dodo):
    # cached rows ahead of the queries hold NaN, in the middle of the list and at its end
    p = _problem("q4nan", BF, 2, 128, [1, 2], [300, 90], [5, 2], inside=True)
    for b in range(2):
        c0, n = int(p["cache_off"][b]), int(p["clen"][b])
        hidden = c0 + np.flatnonzero(p["cpos"][c0:c0 + n] > p["q_pos0"][b] + 1)
        assert len(hidden) > 10
        p["words"][hidden] = np.array(0x7fc07fc0, np.uint32).view(np.int32)
    for t in p["loc"]:
        t.fill_(float("nan"))
    O, lse = _run_q4(dodo, p)
    q = dict(p)
    q["words"] = np.where(p["words"] == 0x7fc07fc0, 0, p["words"])
    q["loc"] = [torch.zeros_like(t) for t in p["loc"]]
    _check(q, O, lse)


@pytest.mark.parametrize("dtype,dh", [(F32, 64), (BF, 128), (BF, 64)])
def test_attend_q4_visible_nan_shows(dodo, dtype, dh):
    p = _problem("q4vis", dtype, 2, dh, [1], [40], [3])
    p["words"][7, 1, 0] = 0x7fc07fc0
    O, lse = _run_q4(dodo, p)
    assert bool(torch.isnan(O[0, 1]).all()) and bool(torch.isnan(lse[0, 1]))
    assert bool(torch.isfinite(O[0, 0]).all())
    # in a value: the group's features
    p = _problem("q4vis", dtype, 2, dh, [1], [40], [3])
    p["words"][39, 1, 1, 1] = 0x7fc07fc0
    O, lse = _run_q4(dodo, p)
    nan = torch.isnan(O[0, 1]).cpu()
    assert bool(nan[32:64].all()) and not bool(nan[:32].any()) and not bool(nan[64:].any()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 5), (BF, 128, 13), (BF, 64, 3), (BF, 64, 13), (F32, 64, 6)])
def test_attend_q4_partly_visible_nan_token(dodo, dtype, dh, tq):
    """A local token, and a nugget, that only the later queries see hold NaN and infinities: earlier queries' outputs are untouched."""
    p = _problem(("q4part", dh, tq), dtype, 2, dh, [tq], [50], [tq + 3], slack=0)
    clean, lc = _run_q4(dodo, p)
    for what, value in ((0, "nan"), (1, "nan"), (1, "inf")):
        q = dict(p, loc=[t.clone() for t in p["loc"]])
        q["loc"][what][tq + 3 - 2] = float(value)                # the last query but one's own token
        O, lse = _run_q4(dodo, q)
        assert torch.equal(O[:tq - 2], clean[:tq - 2]) and torch.equal(lse[:tq - 2], lc[:tq - 2])
        assert not bool(torch.isfinite(O[tq - 2:].float()).any())
        assert bool(torch.isfinite(lse[tq - 2:]).all()) == (what == 1)
    q = dict(p, words=p["words"].copy(), cpos=p["cpos"].copy())
    q["cpos"][49] = p["q_pos0"][0] + 2                           # a nugget that the first two queries do not see
    hidden, lh = _run_q4(dodo, q)
    q["words"][49] = 0x7fc07fc0
    O, lse = _run_q4(dodo, q)
    assert torch.equal(O[:2], hidden[:2]) and torch.equal(lse[:2], lh[:2])
    assert bool(torch.isnan(O[2:]).all()) and bool(torch.isnan(lse[2:]).all())


# the token kernel carries codes as bf16 numbers far below 1 and weights times steps far above: both ends of its range
@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 5), (BF, 64, 1), (BF, 64, 6), (F32, 64, 1)])
@pytest.mark.parametrize("kstd,vstd", [(1.0, 1e13), (1.0, 1e-15), (1.0, 1e-20), (1e12, 1.0), (1e-12, 1.0), (1e18, 1e-10)])
def test_attend_q4_range_of_values(dodo, dtype, dh, tq, kstd, vstd):
    p = _problem(("q4range", kstd, vstd, tq), dtype, 2, dh, [tq, tq], [300, 40], [1, 0], kstd=kstd, vstd=vstd)
    p["loc"][0].fill_(0.0)
    p["loc"][1].mul_(vstd)
    p["Q"] = (p["Q"].float() / kstd).to(dtype)
    _check(p, *_run_q4(dodo, p))


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 3), (BF, 64, 1), (F32, 128, 1)])
@pytest.mark.parametrize("rise", [0.3, 3.0, 90.0])
def test_attend_q4_rising_and_falling_logits(dodo, dtype, dh, tq, rise):
    """The running maximum climbs by less and by more than what moves the reference, from tile to tile and inside one."""
    p = _problem(("q4rise", rise), dtype, 2, dh, [tq, tq], [513, 130], [tq + 1, 0])
    K = plain64.values(p["codes"][:, :, 0], p["words"][:, :, 0])
    q = _f64(p["Q"])
    rows = np.arange(len(K))
    for b in range(2):      # key j along the query, so that its logit is about rise * j / 16, falling in the second sequence
        r = slice(int(p["cache_off"][b]), int(p["cache_off"][b + 1]))
        j = (rows[r] - r.start) * (1 if b == 0 else -1)
        unit = q[tq * b] / (np.sum(q[tq * b] ** 2, -1, keepdims=True) * p["scale"])
        K[r] = 0.05 * K[r] + (rise * j / 16.0)[:, None, None] * unit
    x = torch.from_numpy(K).float().to(dtype).float().numpy()
    p["codes"][:, :, 0], p["words"][:, :, 0] = plain64.pack(*plain64.quantise(x))
    _check(p, *_run_q4(dodo, p))


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 5), (BF, 128, 40), (BF, 64, 2), (F32, 128, 1)])
def test_attend_q4_negative_and_zero_scale(dodo, dtype, dh, tq):
    for scale in (-0.1, 0.0):
        p = _problem(("q4scale", scale, tq), dtype, 2, dh, [tq, tq], [300, 40], [tq, tq + 3], scale=scale)
        _check(p, *_run_q4(dodo, p))


@pytest.mark.parametrize("dtype,H,dh,tq", [(BF, 3, 128, 1), (BF, 3, 128, 10), (F32, 2, 64, 1)])
def test_attend_q4_many_sequences(dodo, dtype, H, dh, tq):
    # 70 sequences: two launch groups, some of them cut, whose partials share the workspace
    rs = np.random.RandomState(8)
    cl = rs.randint(0, 300, 70)
    cl[[3, 66]] = 3000, 5000
    p = _problem(("q4seqs", dh), dtype, H, dh, [int(x) for x in rs.randint(0, tq + 1, 70)], cl.tolist(), rs.randint(0, 40, 70).tolist())
    _check(p, *_run_q4(dodo, p))


def _at16(t):
    """The same tensor at an address that is a multiple of 16 and not of 32 or more."""
    k = 16 // t.element_size()
    buf = torch.empty(t.numel() + 2 * k, dtype=t.dtype, device="cuda")
    first = k if (buf.data_ptr() + 16) % 32 else 0
    out = buf[first:first + t.numel()].view(t.shape)
    out.copy_(t)
    assert out.data_ptr() % 32 == 16
    return out


@pytest.mark.parametrize("dtype,dh", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_q4_at_the_least_alignment(dodo, dtype, dh):
    H, n = 3, 90
    K, V, Q = (inputs.randn((n, H, dh), "q4align", k, dtype=dtype).cuda() for k in "KVQ")
    idx = torch.arange(0, n, 2, dtype=torch.int32, device="cuda")
    got = []
    for place in (lambda t: t, _at16):
        q4, sc, pos = (place(t) for t in _cache(45, H, dh, 0))
        clen = np.zeros(1, np.int32)
        dodo.gather_kv_q4(place(K), place(V), [0, n], idx, [0, 45], [0], q4, sc, pos, [0, 45], clen)
        out = [q4, sc, pos]
        eK, eV = place(torch.zeros((45, H, dh), dtype=dtype, device="cuda")), place(torch.zeros((45, H, dh), dtype=dtype, device="cuda"))
        dodo.expand_kv_q4(q4, sc, [0, 45], clen, eK, eV)
        out += [eK, eV]
        for tq in (1, 5, 40):
            ws = place(torch.empty(dodo.attend_q4_workspace_bytes(H, dh, 45), dtype=torch.uint8, device="cuda"))
            O, lse = place(torch.empty((tq, H, dh), dtype=dtype, device="cuda")), torch.empty((tq, H), device="cuda")
            dodo.attend_q4(place(Q[:tq].contiguous()), [0, tq], [n], dh ** -0.5, q4, sc, pos, [0, 45], clen, place(K), place(V), [0], [n], [n], O, lse, ws)
            out += [O, lse]
        torch.cuda.synchronize()
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_q4_rows_behind_two_to_the_31_elements(dodo):
    """The second sequence's region starts behind 2^31 codes: its rows, appended, expanded and attended, are those of a small cache."""
    H, dh, far, n = 128, 128, 270_000, 70
    assert far * H * dh > 2 ** 32 and far * H * 2 * dh // 2 > 2 ** 31
    K, V = (inputs.randn((n, H, dh), "q4far", k, dtype=BF).cuda() for k in "KV")
    Q = inputs.randn((1, H, dh), "q4far", "Q", dtype=BF).cuda()
    idx = torch.arange(n, dtype=torch.int32, device="cuda")
    got = []
    for base in (0, far):
        q4 = torch.empty((base + n, H, 2, dh // 2), dtype=torch.uint8, device="cuda")
        sc = torch.empty((base + n, H, 2, dh // 32), dtype=torch.int32, device="cuda")
        pos = torch.empty(base + n, dtype=torch.int32, device="cuda")
        off, clen = np.array([0, base, base + n], np.int32), np.zeros(2, np.int32)
        dodo.gather_kv_q4(K, V, [0, 0, n], idx, [0, 0, n], [0, 0], q4, sc, pos, off, clen)
        assert clen.tolist() == [0, n]
        out = [q4[base:].clone(), sc[base:].clone()]
        for tqs in ([0, 0, 1], [0, 0, 2]):
            q = Q.expand(tqs[2], H, dh).contiguous()
            O = torch.empty_like(q)
            dodo.attend_q4(q, tqs, [n, n], dh ** -0.5, q4, sc, pos, off, clen, None, None, None, None, None, O, None, None)
            out.append(O)
        eK, eV = (torch.empty((base + n, H, dh), dtype=BF, device="cuda") for _ in range(2))
        dodo.expand_kv_q4(q4, sc, off, clen, eK, eV)
        out += [eK[base:].clone(), eV[base:].clone()]
        torch.cuda.synchronize()
        got.append(out)
        del q4, sc, pos, eK, eV
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("tqs", [[130, 32, 1], [8, 1, 5]])
def test_attend_q4_query_block_on_tensor_cores(dodo, tqs, inside):
    p = _problem(("q4block", inside), BF, 3, 128, tqs, [333, 64, 0], [200, 40, 70], inside)
    rows = p["codes"].shape[0]
    need = dodo.attend_q4_workspace_bytes(3, 128, rows)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    O, lse = _run_q4(dodo, p, ws)
    _check(p, O, lse, rounded=True)
    # one byte less: the streaming kernel, whose values are not rounded
    Os, ls = _run_q4(dodo, p, ws[:need - 1])
    _check(p, Os, ls)


def test_attend_q4_without_cache_or_locals(dodo):
    p = _problem("q4none", BF, 2, 128, [1, 3], [50, 9], [0, 0])
    _check(p, *_run_q4(dodo, p))
    # no cache at all: equal to the plain form over the local tokens
    p = _problem("q4noc", F32, 2, 64, [1, 2], [0, 0], [9, 70], slack=0)
    O = torch.empty(p["Q"].shape, device="cuda")
    lse = torch.empty(p["Q"].shape[:2], device="cuda")
    dodo.attend_q4(p["Q"].cuda(), p["q_off"], p["q_pos0"], p["scale"], None, None, None, None, None, p["loc"][0].cuda(),
                   p["loc"][1].cuda(), p["loc_off"], p["llen"], p["loc_pos0"], O, lse, None)
    torch.cuda.synchronize()
    _check(p, O, lse)


def test_q4_cache_as_a_server_uses_it(dodo, oracle):
    """Compress, append to the 4-bit cache, decode; append more; decode; in a captured graph and on another stream."""
    H, dh, d, r = 4, 128, 512, 10
    B, n = 3, [300, 77, 512]
    seq_off = inputs.offsets(n)
    ks = [dodo.num_nuggets(m, r) for m in n]
    nug_off, cache_off = inputs.offsets(ks), inputs.offsets([2 * k for k in ks])
    X = inputs.randn((int(seq_off[-1]), d), "q4srv", "X", dtype=BF).cuda()
    w = inputs.randn((d,), "q4srv", "w", std=d ** -0.5, dtype=BF).cuda()
    K, V = (inputs.randn((int(seq_off[-1]), H, dh), "q4srv", k, dtype=BF).cuda() for k in "KV")
    lK, lV = (inputs.randn((B * 8, H, dh), "q4srv", "l" + k, dtype=BF).cuda() for k in "KV")
    Q = inputs.randn((B, H, dh), "q4srv", "Q", dtype=BF).cuda()
    scores, idx = torch.empty(int(seq_off[-1]), device="cuda"), torch.empty(int(nug_off[-1]), dtype=torch.int32, device="cuda")
    rows = int(cache_off[-1])
    ws = torch.empty(dodo.attend_q4_workspace_bytes(H, dh, rows), dtype=torch.uint8, device="cuda")

    def steps(q4, sc, pos, outs):
        clen = np.zeros(B, np.int32)
        for part in range(2):
            dodo.score_select(X, w, 0.0, seq_off, nug_off, 0, scores, idx)
            dodo.gather_kv_q4(K, V, seq_off, idx, nug_off, np.full(B, 1000 * part, np.int32), q4, sc, pos, cache_off, clen)
            for step in range(2):
                dodo.attend_q4(Q, np.arange(B + 1), np.full(B, 5000 + step, np.int32), dh ** -0.5, q4, sc, pos, cache_off, clen, lK, lV,
                               8 * np.arange(B), np.full(B, 8), np.full(B, 4995), outs[2 * part + step], None, ws)
        return clen

    def fresh():
        return _cache(rows, H, dh, 0), [torch.full(Q.shape, float("nan"), dtype=BF, device="cuda") for _ in range(4)]

    (q4, sc, pos), outs = fresh()
    clen = steps(q4, sc, pos, outs)
    torch.cuda.synchronize()
    assert clen.tolist() == [2 * k for k in ks]
    for b in range(B):
        for part in range(2):
            sel = idx[nug_off[b]:nug_off[b + 1]].long() + int(seq_off[b])
            at = slice(int(cache_off[b]) + part * ks[b], int(cache_off[b]) + (part + 1) * ks[b])
            for kv, T in enumerate((K, V)):
                c, wd = plain64.pack(*plain64.quantise(T[sel].float().cpu().numpy()))
                assert np.array_equal(q4[at, :, kv].cpu().numpy(), c) and np.array_equal(sc[at, :, kv].cpu().numpy(), wd)
    for part in range(2):
        for step in range(2):
            p = dict(B=B, H=H, dh=dh, dtype=BF, scale=dh ** -0.5, q_off=np.arange(B + 1), q_pos0=np.full(B, 5000 + step), Q=Q.cpu(),
                     codes=q4.cpu().numpy(), words=sc.cpu().numpy(), cpos=pos.cpu().numpy(), cache_off=cache_off,
                     clen=np.asarray([(part + 1) * k for k in ks]), loc=[lK.cpu(), lV.cpu()], loc_off=8 * np.arange(B),
                     llen=np.full(B, 8), loc_pos0=np.full(B, 4995))
            _check(p, outs[2 * part + step], None)

    # captured, replayed twice (the append is part of the graph), on a stream of its own
    (g4, gs, gp), gouts = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        steps(g4, gs, gp, gouts)
    for _ in range(2):
        for t in gouts:
            t.fill_(float("nan"))
        g4.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g4, q4) and torch.equal(gs, sc) and torch.equal(gp, pos)
        assert all(torch.equal(a, b) for a, b in zip(gouts, outs))
    assert dodo.device_status() == 0


def test_q4_binding_refuses_wrong_tensors(dodo):
    q4, sc, pos = _cache(4, 2, 64)
    K = torch.zeros((4, 2, 64), device="cuda")
    idx = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = lambda **k: {**dict(K=K, V=K, seq_off=[0, 4], idx=idx, nug_off=[0, 1], pos_base=[0], cache_q4=q4, cache_scale=sc,  # noqa: E731
                               cache_pos=pos, cache_off=[0, 4], cache_len=np.zeros(1, np.int32)), **k}
    for bad, kind in ((dict(V=K.bfloat16()), TypeError), (dict(idx=idx.long()), TypeError), (dict(cache_q4=q4.int()), TypeError),
                      (dict(cache_scale=sc[:, :, :, :1]), ValueError), (dict(K=K.cpu()), ValueError), (dict(V=K[:3]), ValueError),
                      (dict(seq_off=[0, 5]), ValueError), (dict(nug_off=[0, 2]), ValueError), (dict(cache_off=[0, 5]), ValueError),
                      (dict(cache_len=[0]), TypeError), (dict(K=K.transpose(0, 1)), ValueError), (dict(pos_base=[]), ValueError)):
        with pytest.raises(kind):
            dodo.gather_kv_q4(**args(**bad))
    with pytest.raises(api.DodoError) as e:
        dodo.gather_kv_q4(**args(cache_len=np.full(1, 4, np.int32)))
    assert e.value.status == api.ERR_CAPACITY


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 3), (BF, 64, 1), (F32, 128, 1)])
def test_attend_right_behind_an_append_when_the_first_sequences_are_idle(dodo, dtype, dh, tq, four_bits):
    """70 sequences, the first 64 of them (a whole launch group) without queries this step: the others' attention waits for the append."""
    H, B, idle, rows_of = 8, 70, 64, 500
    ks = [8] * idle + [rows_of] * (B - idle)
    off = inputs.offsets(ks)
    rows = int(off[-1])
    K, V = (inputs.randn((rows, H, dh), "q4idle", k, dtype=dtype).cuda() for k in "KV")
    Q = inputs.randn((tq * (B - idle), H, dh), "q4idle", "Q", dtype=dtype).cuda()
    idx = _cuda(np.concatenate([np.arange(k, dtype=np.int32) for k in ks]))
    q_off = np.concatenate([np.zeros(idle, np.int32), tq * np.arange(B - idle + 1)]).astype(np.int32)
    q_pos0, pos_base = np.full(B, 10_000, np.int32), np.zeros(B, np.int32)
    q4, sc, pos = _cache(rows, H, dh)
    cK, cV = torch.empty_like(K), torch.empty_like(V)
    ws = torch.empty(dodo.attend_q4_workspace_bytes(H, dh, rows), dtype=torch.uint8, device="cuda")
    full = np.asarray(ks, np.int32)

    def append():
        clen = np.zeros(B, np.int32)
        if four_bits:
            dodo.gather_kv_q4(K, V, off, idx, off, pos_base, q4, sc, pos, off, clen)
        else:
            dodo.gather_kv(K, V, off, idx, off, pos_base, cK, cV, pos, off, clen)

    def attend():
        O = torch.full_like(Q, float("nan"))
        torch.cuda.synchronize()

        def call():
            args = (q4, sc) if four_bits else (cK, cV)
            fn = dodo.attend_q4 if four_bits else dodo.attend
            fn(Q, q_off, q_pos0, dh ** -0.5, *args, pos, off, full, None, None, None, None, None, O, None, ws)
        return O, call

    append()
    torch.cuda.synchronize()
    want, call = attend()
    call()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(want.float()).all())
    for _ in range(10):
        for t in (q4, sc, pos, cK, cV):
            t.zero_()
        O, call = attend()
        append()
        call()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 5), (BF, 64, 1), (BF, 64, 5), (F32, 64, 1), (F32, 128, 3), (BF, 128, 40)])
def test_attend_q4_between_the_ends_of_the_positions(dodo, dtype, dh, tq):
    """The last query at 2^30 - 1 over local tokens from -2^30 on sees them all (their number behind the first is 2^31), and queries
    from -2^30 on none of those that end at 2^30."""
    p = _problem(("q4corner", tq), dtype, 2, dh, [tq, tq, tq], [30, 30, 0], [70, 70, 70])
    p["q_pos0"] = np.asarray([2 ** 30 - tq, -2 ** 30, 2 ** 30 - tq], np.int32)
    p["loc_pos0"] = np.asarray([-2 ** 30, 2 ** 30 - 70, -2 ** 30], np.int32)
    O, lse = _run_q4(dodo, p)
    _check(p, O, lse, rounded=tq >= 32)
    assert bool(torch.isneginf(lse[tq:2 * tq]).all()) and bool(torch.isfinite(lse[2 * tq:]).all())
    assert dodo.device_status() == 0


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 1), (BF, 128, 5), (BF, 64, 1), (BF, 64, 6), (F32, 128, 2)])
@pytest.mark.parametrize("power", [-110, 60, 118, 121])
def test_attend_q4_range_of_queries(dodo, dtype, dh, tq, power):
    """Queries times 2^power with the softmax's scale times 2^-power have the same logits, to the bit."""
    p = _problem(("q4qrange", tq), dtype, 2, dh, [tq, tq], [300, 40], [tq, tq + 9], kstd=0.25)
    O, lse = _run_q4(dodo, p)
    _check(p, O, lse)
    q = dict(p, Q=(p["Q"].float() * 2.0 ** power).to(dtype), scale=p["scale"] * 2.0 ** -power)
    assert bool(torch.isfinite(q["Q"].float()).all()) and torch.equal((q["Q"].double() * 2.0 ** -power).to(dtype), p["Q"])
    O2, lse2 = _run_q4(dodo, q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,tq", [(BF, 8), (BF, 1), (F32, 4)])
def test_attend_q4_fits_the_workspace_at_its_fullest(dodo, dtype, tq):
    """A unit's share of one and a half blocks is rounded to two: with two such units per SM the partial results take all of
    dodo_attend's workspace, and no byte behind it."""
    H, B, dh = torch.cuda.get_device_properties(0).multi_processor_count // 4, 8, 128
    p = _problem(("q4full", dtype == BF, tq), dtype, H, dh, [tq] * B, [560] * B, [tq] * B)
    n = dodo.attend_workspace_bytes(dh)
    ws = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    O, lse = _run_q4(dodo, p, ws[:n])
    assert bool((ws[n:] == 0xff).all())
    one = dict(p, B=1, q_off=p["q_off"][:2], Q=p["Q"][:tq], cache_off=p["cache_off"][:2])
    _check(one, O[:tq], lse[:tq])
    assert bool(torch.isfinite(O.float()).all())


@pytest.mark.parametrize("tq", [40, 130, 300])
def test_attend_q4_block_masked_rows_may_hold_anything(dodo, tq):
    """Blocks of queries on the tensor cores: nuggets that no query sees, and nuggets and local tokens that only some of them see, hold
    NaN and infinities.  Queries that do not see them keep their bits; the others show them, in the features that have them."""
    p = _problem(("q4blockany", tq), BF, 2, 128, [tq, 33], [150, 70], [tq + 3, 40])
    late = p["q_pos0"][0] + tq // 2
    p["cpos"][[0, 1, 70, 149]] = [late, 10 ** 6, late, 10 ** 6]        # a first tile's, a later one's; two that nobody sees
    clean, lc = _run_q4(dodo, p)
    _check(p, clean, lc, rounded=True)
    _, _, tol, _ = _reference(p, rounded=True)

    def check(q):
        """Against the plain form over what each query sees, with the clean batch's tolerance; the log-sum-exp does not hang on values."""
        O, lse = _run_q4(dodo, q)
        want, got = _reference(q, rounded=True)[0], _f64(O)
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(got), fine) and np.array_equal(np.isnan(got), np.isnan(want))
        assert np.all(np.abs(got[fine] - want[fine]) <= tol[fine]) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        assert torch.equal(lse, lc)
        O2, _ = _run_q4(dodo, q)
        assert torch.equal(O.nan_to_num(7.0, 1e30, -1e30), O2.nan_to_num(7.0, 1e30, -1e30))
        return fine

    q = dict(p, words=p["words"].copy(), loc=[t.clone() for t in p["loc"]])
    q["words"][[1, 149]] = 0x7fc07fc0
    assert check(q).all()                                               # hidden: nothing to be seen of them
    for row in (0, 70):                                                 # a value of head 1, features 32 to 63
        w = dict(q, words=q["words"].copy())
        w["words"][row, 1, 1, 1] = 0x7fc07fc0
        fine = check(w)
        assert fine[:tq // 2].all() and fine[tq:].all() and not fine[tq // 2:tq, 1, 32:64].any() and fine[:, 0].all()
    last = int(p["loc_off"][0]) + tq + 3 - 4                            # the fourth last local token: its own query's and three more see it
    for value in ("nan", "inf", "-inf"):
        w = dict(q, loc=[t.clone() for t in p["loc"]])
        w["loc"][1][last, 0, 5] = float(value)
        w["loc"][1][last + 2, 0, 5] = -float("inf")
        fine = check(w)
        assert fine[:tq - 4].all() and not fine[tq - 4:tq, 0, 5].any() and fine[:, 1].all()
    assert dodo.device_status() == 0


@pytest.mark.parametrize("tq", [40, 200])
def test_attend_q4_block_visible_nan_shows(dodo, tq):
    p = _problem(("q4blockvis", tq), BF, 2, 128, [tq, 1], [90, 20], [tq + 1, 3])
    clean, lc = _run_q4(dodo, p)
    q = dict(p, words=p["words"].copy())
    q["words"][45, 1, 0, 2] = 0x7fc07fc0                         # a group of a key that every query of the first sequence sees
    O, lse = _run_q4(dodo, q)
    assert bool(torch.isnan(O[:tq, 1]).all()) and bool(torch.isnan(lse[:tq, 1]).all())
    assert torch.equal(O[:tq, 0], clean[:tq, 0]) and torch.equal(lse[:tq, 0], lc[:tq, 0]) and torch.equal(O[tq:], clean[tq:])


@pytest.mark.parametrize("power", [30, 60])
def test_attend_q4_block_with_a_tiny_scale(dodo, power):
    """Large queries and a tiny softmax scale: masked keys and rows that see nothing stay out (below a scale of 1e-9 blocks take the
    kernels that mask behind the scale)."""
    p = _problem(("q4tiny", power), BF, 2, 128, [70, 40], [300, 60], [10, 40], inside=True)
    p["q_pos0"][1] = -5                                           # the first queries see nothing
    p["Q"], p["scale"] = (p["Q"].float() * 2.0 ** power).to(BF), p["scale"] * 2.0 ** -power
    O, lse = _run_q4(dodo, p)
    _check(p, O, lse, rounded=p["scale"] >= 1e-9)
    assert bool(torch.isneginf(lse).any())
