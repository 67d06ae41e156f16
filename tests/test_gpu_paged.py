"""The paged nugget cache on the GPU: appends with the rotation on the way, attention over it by chunks and single tokens, against plain
forms in 64 bits; masks, bad pages, shared pages, strides, cuts, captures and streams."""
import struct

import numpy as np
import pytest
import torch

import paged64
import plain64
from paper_2310_02409_b200 import api, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _table(lens, page, spare=2, seed=3):
    """page_off, a page table of scattered pages, pages in all, and every sequence's rows of the pool."""
    need = [-(-n // page) for n in lens]
    off = inputs.offsets(need)
    pages = int(off[-1]) + spare
    table = np.random.RandomState(seed).permutation(pages)[:off[-1]].astype(np.int32)
    rows = [np.array([table[off[b] + r // page] * page + r % page for r in range(n)], np.int64) for b, n in enumerate(lens)]
    return off, table, pages, rows


# ---- append -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,H,dh,rot,layout", [
    (BF, 32, 128, 128, "half"), (BF, 8, 128, 128, "interleaved"), (F32, 4, 64, 64, "half"), (F32, 3, 64, 20, "interleaved"), (BF, 2, 80, 40, "half"),
    (BF, 1, 64, 18, "half"), (BF, 5, 128, 0, "half"), (F32, 1, 12, 6, "half"), (BF, 72, 128, 128, "half"), (BF, 9, 256, 256, "half"), (F32, 2, 512, 256, "interleaved"),
])
@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("every", [False, True])
def test_append_is_gather_and_rotation(dodo, dtype, H, dh, rot, layout, page, every):
    lens, ks, used = [40, 0, 300, 1, 64], [17, 0, 31, 1, 64], [3, 0, 16, 1, 2]
    if every:
        ks = lens
    seq_off, nug_off = inputs.offsets(lens), inputs.offsets(ks)
    page_off, table, pages, rows = _table([k + u for k, u in zip(ks, used)], page)
    N = int(seq_off[-1])
    K, V = (inputs.randn((N, H, dh), "append", H, dh, n, dtype=dtype) for n in "KV")
    rs = np.random.RandomState(1)
    idx = np.concatenate([np.sort(rs.permutation(n)[:k]).astype(np.int32) for n, k in zip(lens, ks)])
    pos_base = np.array([5, 6, 70000, 8, 1 << 30], np.int32)
    cK = inputs.randn((pages, page, H, dh), "append old", dtype=dtype).cuda()
    cV, pos = cK.clone() + 1, torch.full((pages, page), -7, dtype=torch.int32, device="cuda")
    before = [t.flatten(0, 1).clone() for t in (cK, cV, pos)]
    freq = api.rope_frequencies(rot) if rot else None
    rope = api.Rope(freq, api.ROPE_HALF if layout == "half" else api.ROPE_INTERLEAVED, 0.75) if rot else None
    clen = np.asarray(used, np.int32)
    dodo.gather_kv_paged(K.cuda(), V.cuda(), seq_off, None if every else _cuda(idx), None if every else nug_off, pos_base, rope,
                         api.PagedCache(cK, cV, pos, _cuda(table)), page_off, clen)
    torch.cuda.synchronize()
    assert clen.tolist() == [k + u for k, u in zip(ks, used)]
    src = np.concatenate([seq_off[b] + idx[nug_off[b]:nug_off[b + 1]] for b in range(5)])
    dst = np.concatenate([r[u:] for r, u in zip(rows, used)])
    where = np.concatenate([pos_base[b] + idx[nug_off[b]:nug_off[b + 1]].astype(np.int64) for b in range(5)])
    want_v, want_p = before[1].clone(), before[2].clone()
    want_v[dst], want_p[dst] = V[src].cuda(), _cuda(where, torch.int32)
    assert torch.equal(cV.flatten(0, 1), want_v) and torch.equal(pos.view(-1), want_p.view(-1))
    got = cK.flatten(0, 1)
    rest = np.setdiff1d(np.arange(pages * page), dst)
    assert torch.equal(got[rest], before[0][rest])
    if not rot:
        assert torch.equal(got[dst], K[src].cuda())
        return
    want, bound = paged64.rope(_f64(K[src]), where, freq, layout, 0.75)
    half = plain64.HALF[NAME[dtype]]
    assert (np.abs(_f64(got[dst]) - want) <= bound + half * (np.abs(want) + bound)).all()


def test_append_equals_rope_then_append(dodo):
    """Bit for bit: the rotation on the way is the rotation of whole arrays."""
    N, H, dh, page = 33, 6, 128, 8
    K, V = (inputs.randn((N, H, dh), "append two", n, dtype=BF).cuda() for n in "KV")
    rope = api.Rope(api.rope_frequencies(96), api.ROPE_HALF, 1.1)
    off, table, pages, _ = _table([N], page)
    out = []
    for turned in (False, True):
        cK, cV = (torch.zeros((pages, page, H, dh), dtype=BF, device="cuda") for _ in range(2))
        pos = torch.zeros((pages, page), dtype=torch.int32, device="cuda")
        X = K.clone()
        if turned:
            dodo.rope(rope, [0, N], [900], X)
        dodo.gather_kv_paged(X, V, [0, N], None, None, [900], None if turned else rope, api.PagedCache(cK, cV, pos, _cuda(table)), off, np.zeros(1, np.int32))
        out.append((cK, cV, pos))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_append_of_slices_of_many_sequences(dodo):
    """K and V inside a fused projection's rows; more sequences than one launch holds; several appends in a row."""
    B, H, dh, page = 70, 2, 64, 4
    lens = [b % 4 for b in range(B)]
    off = inputs.offsets(lens)
    N = int(off[-1])
    page_off, table, pages, rows = _table([2 * n for n in lens], page)
    cK, cV = (torch.zeros((pages, page, H, dh), dtype=F32, device="cuda") for _ in range(2))
    pos = torch.zeros((pages, page), dtype=torch.int32, device="cuda")
    cache, clen = api.PagedCache(cK, cV, pos, _cuda(table)), np.zeros(B, np.int32)
    freq = api.rope_frequencies(64)
    fused = [inputs.randn((N, 5, H, dh), "append fused", i, dtype=F32).cuda() for i in range(2)]
    for i, f in enumerate(fused):
        dodo.gather_kv_paged(f[:, 3], f[:, 4], off, None, None, np.arange(B) + 100 * i, api.Rope(freq), cache, page_off, clen)
    torch.cuda.synchronize()
    for b in range(B):
        for i, f in enumerate(fused):
            at = rows[b][i * lens[b]:(i + 1) * lens[b]]
            p = b + 100 * i + np.arange(lens[b])
            want, bound = paged64.rope(_f64(f[off[b]:off[b + 1], 3]), p, freq, "half")
            assert (np.abs(_f64(cK.flatten(0, 1)[at]) - want) <= bound + paged64.U * (np.abs(want) + bound)).all()
            assert torch.equal(cV.flatten(0, 1)[at], f[off[b]:off[b + 1], 4]) and pos.view(-1)[at].tolist() == p.tolist()


def test_append_leaves_bad_indices_and_bad_pages_out(libdodo):
    own = api.Dodo(0)
    H, dh, page = 2, 64, 4
    K = inputs.randn((10, H, dh), "append bad", dtype=BF).cuda()
    table = np.array([2, 9, -1, 1], np.int32)                     # five pages
    cK, cV = (torch.zeros((5, page, H, dh), dtype=BF, device="cuda") for _ in range(2))
    pos = torch.full((5, page), -7, dtype=torch.int32, device="cuda")
    idx = np.array([0, 1, 10, 3, 4, 5, 6, 7, 8, 9, -1, 2, 1, 0], np.int32)
    clen = np.zeros(2, np.int32)
    own.gather_kv_paged(K, K, [0, 10, 10], _cuda(idx[:10]), [0, 10, 10], [20, 0], None, api.PagedCache(cK, cV, pos, _cuda(table)), [0, 4, 4], clen)
    torch.cuda.synchronize()
    assert own.device_status() == api.DEV_BAD_INDEX and clen.tolist() == [10, 0]
    want = np.full((5, page), -7)
    want[2] = [20, 21, -7, 23]                                    # the third index is outside; pages 9 and -1 are not there
    assert np.array_equal(pos.cpu().numpy(), want)
    own.reset()
    torch.cuda.synchronize()
    assert own.device_status() == 0
    own.close()


# ---- attention --------------------------------------------------------------------------------------------------------
def _batch(dtype, H, Hkv, dh, tq, nug, loc, page, q_pos0=None, span=10, seed=0, spare=2, fill=None):
    """A batch as a dict of the call's arguments and of what the plain form needs."""
    rs = np.random.RandomState(100 + seed)
    B = len(tq)
    page_off, table, pages, rows = _table(nug, page, spare, seed)
    new = lambda shape, n: inputs.randn(shape, "paged", H, dh, n, seed, dtype=dtype)  # noqa: E731
    cK, cV = new((pages * page, Hkv, dh), "cK"), new((pages * page, Hkv, dh), "cV")
    if fill is not None:            # what no sequence owns may hold anything
        free = np.setdiff1d(np.arange(pages * page), np.concatenate(rows))
        cK[free], cV[free] = fill, fill
    pos = np.full(pages * page, 2 ** 31 - 1, np.int64)
    for r in rows:
        pos[r] = np.sort(rs.permutation(span * len(r))[:len(r)])
    loc_pos0 = [span * n for n in nug]
    q_pos0 = [p + n - t for p, n, t in zip(loc_pos0, loc, tq)] if q_pos0 is None else q_pos0
    return dict(dtype=dtype, H=H, Hkv=Hkv, dh=dh, B=B, q_off=inputs.offsets(tq), q_pos0=np.asarray(q_pos0, np.int32), scale=dh ** -0.5, cK=cK, cV=cV,
                pos=pos, table=table, page_off=page_off, rows=rows, nug=np.asarray(nug, np.int32), page=page, pages=pages, Q=new((sum(tq), H, dh), "Q"),
                lK=new((sum(loc), Hkv, dh), "lK"), lV=new((sum(loc), Hkv, dh), "lV"), loc_off=inputs.offsets(loc), loc=np.asarray(loc, np.int32),
                loc_pos0=np.asarray(loc_pos0, np.int32))


def _run(dodo, s, workspace=True, lse=True, O=None):
    shape = (s["pages"], s["page"], s["Hkv"], s["dh"])
    cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
    O = torch.full(s["Q"].shape, 7.0, dtype=s["dtype"], device="cuda") if O is None else O
    L = torch.full(s["Q"].shape[:2], 7.0, device="cuda") if lse else None
    ws = torch.full((dodo.attend_paged_workspace_bytes(s["dh"]),), 0xff, dtype=torch.uint8, device="cuda") if workspace else None
    dodo.attend_paged(s["Q"].cuda(), s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], s["lK"].cuda(), s["lV"].cuda(), s["loc_off"][:-1],
                      s["loc"], s["loc_pos0"], O, L, ws)
    torch.cuda.synchronize()
    return O, L


def _sequence(s, b):
    q, l = slice(s["q_off"][b], s["q_off"][b + 1]), slice(s["loc_off"][b], s["loc_off"][b] + s["loc"][b])
    r = s["rows"][b][:s["nug"][b]]
    K, V = (np.concatenate([_f64(s[c][r]), _f64(s[n][l])]) for c, n in (("cK", "lK"), ("cV", "lV")))
    kpos = np.concatenate([s["pos"][r], s["loc_pos0"][b] + np.arange(s["loc"][b])]).astype(np.int64)
    return q, _f64(s["Q"][q]), s["q_pos0"][b].astype(np.int64) + np.arange(q.stop - q.start), K, V, kpos


def _check(s, O, L, only=None):
    half = plain64.HALF[NAME[s["dtype"]]]
    wh = half if s["dtype"] is BF else 0.0
    for b in range(s["B"]) if only is None else only:
        q, Q, qpos, K, V, kpos = _sequence(s, b)
        if Q.shape[0] == 0:
            continue
        o, l = paged64.attend(Q, qpos, s["scale"], K, V, kpos)
        tO, tL = paged64.attend_bounds(Q, qpos, s["scale"], K, V, kpos, o, l, half, wh)
        got = _f64(O[q])
        assert (np.abs(got - o) <= tO).all(), (b, float((np.abs(got - o) - tO).max()))
        if L is not None:
            none = np.isneginf(l)
            assert np.array_equal(np.isneginf(_f64(L[q])), none)
            assert (np.abs(_f64(L[q]) - l)[~none] <= tL[~none]).all()


HEADS = [(4, 4), (8, 2), (6, 2), (7, 1), (40, 8)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("page", [1, 16, 40])
def test_single_tokens(dodo, dtype, dh, H, Hkv, page):
    s = _batch(dtype, H, Hkv, dh, [1] * 7, [0, 1, 15, 16, 17, 205, 700], [1, 0, 3, 64, 33, 64, 5], page, fill=float("nan"))
    s["q_pos0"][1] = 11
    _check(s, *_run(dodo, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("tq", [[2, 2, 2], [5, 0, 3], [16, 1, 9], [33, 70, 1], [129, 256, 300]])
def test_chunks(dodo, dtype, dh, H, Hkv, tq):
    """Chunks of new tokens among the local tokens, causal inside."""
    nug = [130, 40, 0]
    s = _batch(dtype, H, Hkv, dh, tq, nug, [t + e for t, e in zip(tq, (0, 17, 200))], 16, fill=float("inf"), seed=sum(tq))
    _check(s, *_run(dodo, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("tq", [1, 3, 40, 200])
@pytest.mark.parametrize("page", [1, 7, 64])
def test_chunks_inside_the_cache(dodo, dtype, dh, tq, page):
    """The new tokens' own rows have been appended: causal inside the cache, whose rows are not in the order of their positions."""
    H, Hkv = 6, 3
    s = _batch(dtype, H, Hkv, dh, [tq, tq], [tq + 100, tq], [0, 0], page, q_pos0=[100, 0], span=1, fill=float("nan"), seed=tq)
    rs = np.random.RandomState(5)
    for r in s["rows"]:
        s["pos"][r] = s["pos"][rs.permutation(r)]
    _check(s, *_run(dodo, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (8, 1, 2), (4, 2, 50), (2, 2, 150)])
def test_queries_inside_and_ahead_of_the_context(dodo, dtype, H, Hkv, tq):
    """Queries that see part of the nuggets, none of them, or (a position before everything) nothing at all."""
    s = _batch(dtype, H, Hkv, 128, [tq] * 4, [300, 300, 300, 0], [0, 10, 10, 10], 16, q_pos0=[1500, 100, -5000, -5000], seed=tq)
    O, L = _run(dodo, s)
    _check(s, O, L)
    blind = slice(int(s["q_off"][2]), int(s["q_off"][4]))
    assert (O[blind] == 0).all() and torch.isneginf(L[blind]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq,dh", [(4, 4, 1, 128), (8, 1, 1, 64), (8, 2, 4, 128), (4, 2, 64, 128), (4, 4, 140, 64), (40, 40, 1, 128)])
def test_long_lists_are_cut_and_joined(dodo, dtype, H, Hkv, tq, dh):
    s = _batch(dtype, H, Hkv, dh, [tq, 1], [9001, 40], [tq + 100, 1], 32, span=2)
    O, L = _run(dodo, s)
    _check(s, O, L)
    O2, L2 = _run(dodo, s)
    assert torch.equal(O, O2) and torch.equal(L, L2)             # the same bits whichever block comes last


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (8, 2, 3), (4, 4, 20), (4, 2, 100)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3e38])
def test_what_a_query_does_not_see_takes_no_part(dodo, dtype, H, Hkv, tq, bad):
    """Rows of K and V that some or all queries of a chunk do not see hold anything; every result is what it is without them."""
    s = _batch(dtype, H, Hkv, 128, [tq, tq], [200, 50], [tq, tq + 3], 16, q_pos0=[1000, 250], seed=tq)
    for b in range(2):
        r = s["rows"][b]
        q_last = int(s["q_pos0"][b]) + tq - 1
        hidden = r[s["pos"][r] > q_last]
        s["pos"][r[3]] = int(s["q_pos0"][b]) + tq // 2 + 1       # seen by the later half of the queries only
        assert len(hidden) > 0
        s["cK"][hidden], s["cV"][hidden] = bad, bad
    clean = _run(dodo, s)
    _check_masked(s, *clean)
    # rows that only the later queries see: the earlier ones stay as they were
    first = [int(s["q_off"][b]) + t for b in range(2) for t in range(min(tq, tq // 2 + 1))]
    for b in range(2):
        s["cV"][s["rows"][b][3]] = bad
    O, L = _run(dodo, s)
    assert torch.equal(L[first], clean[1][first])
    same = (O[first].float() - clean[0][first].float()).abs()
    assert bool((same <= 2.0 ** -7 * clean[0][first].float().abs() + 2.0 ** -7).all())       # finite again, weights rounded or not
    late = [int(s["q_off"][b]) + t for b in range(2) for t in range(tq // 2 + 1, tq)]
    if late and bad != -3e38:
        assert not torch.isfinite(O[late].float()).any()


def _check_masked(s, O, L):
    """_check, with the rows that nobody sees taken out of the plain form's sums as well (0 * inf is no 0)."""
    t = {k: (v.clone() if isinstance(v, torch.Tensor) else v) for k, v in s.items()}
    for n in ("cK", "cV"):
        t[n][~torch.isfinite(t[n])] = 0.0
        t[n][t[n].abs() > 1e38] = 0.0
    _check(t, O, L)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (8, 2, 4), (4, 2, 90)])
def test_a_visible_nan_shows(dodo, dtype, H, Hkv, tq):
    s = _batch(dtype, H, Hkv, 128, [tq, tq], [60, 60], [tq, tq], 16)
    s["cK"][s["rows"][0][7], 0, 5] = float("nan")
    s["cV"][s["rows"][1][9], Hkv - 1, 11] = float("nan")
    O, L = _run(dodo, s)
    g = H // Hkv
    nan_o = torch.zeros(O.shape, dtype=torch.bool)
    nan_o[:tq, :g] = True
    nan_o[tq:, H - g:, 11] = True
    assert torch.equal(torch.isnan(O.float()).cpu(), nan_o)
    want = torch.zeros(L.shape, dtype=torch.bool)
    want[:tq, :g] = True
    assert torch.equal(torch.isnan(L).cpu(), want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-12, 30.0])
@pytest.mark.parametrize("tq", [1, 40, 150])
def test_scales(dodo, dtype, scale, tq):
    s = _batch(dtype, 4, 2, 64, [tq], [300], [tq], 16)
    s["scale"] = scale
    _check(s, *_run(dodo, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tq", [1, 8, 200])
def test_rising_logits(dodo, dtype, tq):
    """Every tile raises the running maximum; large logits of both signs."""
    s = _batch(dtype, 2, 1, 128, [tq], [900], [tq], 16, span=1)
    r = s["rows"][0]
    ramp = torch.linspace(-30.0, 30.0, len(r))[:, None, None].to(s["dtype"])
    s["cK"][r] = torch.sign(s["Q"][:1, :1]) * ramp
    _check(s, *_run(dodo, s))


def test_more_sequences_than_a_launch_holds(dodo):
    B = 150
    for dtype, tq in ((BF, [1] * B), (F32, [b % 3 for b in range(B)]), (BF, [(7 * b) % 40 for b in range(B)])):
        s = _batch(dtype, 4, 2, 64, tq, [(37 * b) % 90 for b in range(B)], [t + b % 5 for b, t in enumerate(tq)], 8)
        _check(s, *_run(dodo, s), only=range(0, B, 7))


def test_sequences_share_pages(dodo):
    """Two sequences over one prefix: the same pages in both tables, pages of their own behind them."""
    for dtype, tq in ((BF, 1), (F32, 1), (BF, 60)):
        s = _batch(dtype, 8, 2, 128, [tq, tq], [64, 100], [tq, tq], 16, span=1)
        s["table"][4:8] = s["table"][:4]
        s["rows"][1][:64] = s["rows"][0]
        s["pos"][s["rows"][1]] = np.arange(100)
        _check(s, *_run(dodo, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tq", [1, 5, 80])
def test_bad_pages_are_not_followed(libdodo, dtype, tq):
    own = api.Dodo(0)
    s = _batch(dtype, 4, 2, 128, [tq, tq], [100, 100], [tq, tq], 16)
    for bad, at in ((-1, 1), (s["pages"], 4), (2 ** 31 - 1, 8), (-2 ** 31, 9)):
        s["table"][at] = bad
    O, L = _run(own, s)
    assert own.device_status() == api.DEV_BAD_INDEX
    for b, gone in ((0, (1, 4)), (1, (1, 2))):
        keep = np.array([r // 16 not in gone for r in range(100)])
        s["rows"][b] = s["rows"][b][keep]
        s["nug"][b] = keep.sum()
    _check(s, O, L)
    own.reset()
    own.close()


def test_without_cache_without_local_without_lse(dodo):
    for dtype, tq in ((BF, 1), (F32, 1), (BF, 130)):
        s = _batch(dtype, 4, 4, 128, [tq, 1], [0, 0], [tq, 3], 16)
        _check(s, _run(dodo, s, workspace=False, lse=False)[0], None)
        s = _batch(dtype, 4, 4, 128, [tq, 1], [50, 0], [0, 0], 16, q_pos0=[600, 4])
        O, _ = _run(dodo, s, lse=False)
        _check(s, O, None)
        assert (O[tq:] == 0).all()


def test_rows_behind_the_last_sequence_stay(dodo):
    for dtype, tq in ((BF, 1), (F32, 2), (BF, 100)):
        s = _batch(dtype, 4, 2, 128, [tq, tq], [30, 30], [tq, tq], 16)
        s["Q"] = torch.cat([s["Q"], s["Q"][:5]])
        O, L = _run(dodo, s)
        assert (O[2 * tq:] == 7.0).all() and (L[2 * tq:] == 7.0).all()
        _check(s, O[:2 * tq], L[:2 * tq])


@pytest.mark.parametrize("dtype,H,Hkv,tq", [(BF, 8, 2, 1), (F32, 4, 4, 1), (BF, 4, 2, 70), (BF, 8, 8, 9)])
def test_captured_replayed_and_on_two_streams(libdodo, dtype, H, Hkv, tq):
    """Graphs of two contexts with a workspace each, replayed at once on two streams; an eager call between."""
    sets = []
    for i in range(2):
        d = api.Dodo(0)
        s = _batch(dtype, H, Hkv, 128, [tq] * 3, [3000, 70, 0], [tq + 64] * 3, 16, seed=i)
        shape = (s["pages"], s["page"], Hkv, 128)
        cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
        Q, lK, lV = s["Q"].cuda(), s["lK"].cuda(), s["lV"].cuda()
        O, L = torch.zeros(Q.shape, dtype=dtype, device="cuda"), torch.zeros(Q.shape[:2], device="cuda")
        ws = torch.empty(d.attend_paged_workspace_bytes(128), dtype=torch.uint8, device="cuda")
        call = lambda d=d, s=s, cache=cache, Q=Q, lK=lK, lV=lV, O=O, L=L, ws=ws: d.attend_paged(  # noqa: E731
            Q, s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], lK, lV, s["loc_off"][:-1], s["loc"], s["loc_pos0"], O, L, ws)
        call()
        torch.cuda.synchronize()
        want = (O.clone(), L.clone())
        _check(s, O, L)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        sets.append((d, O, L, want, side, graph, call))
    for _ in range(3):
        for d, O, L, want, side, graph, call in sets:
            O.zero_()
            L.zero_()
        torch.cuda.synchronize()
        for d, O, L, want, side, graph, call in sets:
            with torch.cuda.stream(side):
                graph.replay()
                call()
                graph.replay()
        torch.cuda.synchronize()
        for d, O, L, want, side, graph, call in sets:
            assert torch.equal(O, want[0]) and torch.equal(L, want[1])
    for d, *_ in sets:
        assert d.device_status() == 0
        d.close()


@pytest.mark.parametrize("dtype,tq", [(BF, 1), (F32, 1), (BF, 64)])
def test_pool_behind_2_31_elements(dodo, dtype, tq):
    """Rows of K and V whose elements have indices beyond 32 bits."""
    H, dh, page = 8, 128, 16
    pages = (2 ** 31 // (H * dh)) // page + 40
    if torch.cuda.mem_get_info()[0] < 2 * pages * page * H * dh * 4 + (2 << 30):
        pytest.skip("needs more device memory")
    n = 300
    table = np.concatenate([np.arange(pages - 15, pages), np.arange(4)]).astype(np.int32)
    rows = np.array([table[r // page] * page + r % page for r in range(n)], np.int64)
    cK, cV = (torch.zeros((pages, page, H, dh), dtype=dtype, device="cuda") for _ in range(2))
    pos = torch.zeros((pages, page), dtype=torch.int32, device="cuda")
    K, V = (inputs.randn((n, H, dh), "far", x, dtype=dtype) for x in "KV")
    cache, clen = api.PagedCache(cK, cV, pos, _cuda(table)), np.zeros(1, np.int32)
    dodo.gather_kv_paged(K.cuda(), V.cuda(), [0, n], None, None, [0], None, cache, [0, len(table)], clen)
    assert torch.equal(cK.flatten(0, 1)[_cuda(rows)].cpu(), K) and torch.equal(cV.flatten(0, 1)[_cuda(rows)].cpu(), V)
    Q = inputs.randn((tq, H, dh), "far", "Q", dtype=dtype)
    O, L = torch.zeros((tq, H, dh), dtype=dtype, device="cuda"), torch.zeros((tq, H), device="cuda")
    ws = torch.empty(dodo.attend_paged_workspace_bytes(dh), dtype=torch.uint8, device="cuda")
    dodo.attend_paged(Q.cuda(), [0, tq], [n - tq], dh ** -0.5, cache, [0, len(table)], clen, None, None, None, None, None, O, L, ws)
    torch.cuda.synchronize()
    qpos, kpos, half = n - tq + np.arange(tq), np.arange(n), plain64.HALF[NAME[dtype]]
    o, l = paged64.attend(_f64(Q), qpos, dh ** -0.5, _f64(K), _f64(V), kpos)
    tO, tL = paged64.attend_bounds(_f64(Q), qpos, dh ** -0.5, _f64(K), _f64(V), kpos, o, l, half, half if dtype is BF else 0.0)
    assert (np.abs(_f64(O) - o) <= tO).all() and (np.abs(_f64(L) - l) <= tL).all()


# ---- a run of them together -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,H,Hkv", [(BF, 8, 2), (F32, 4, 4)])
def test_a_server(dodo, dtype, H, Hkv):
    """Two sequences: a prompt is scored, selected, appended to pages with its positions; then chunks and single tokens are projected (Q, K
    and V side by side in a row), turned, appended and attended, pages handed out as the caches grow."""
    dh, page, d = 128, 8, 256
    rope_freq = api.rope_frequencies(dh, 10000.0, api.ROPE_LINEAR, 2.0)
    rope = api.Rope(rope_freq)
    pages, per = 64, 32
    cK, cV = (torch.full((pages, page, Hkv, dh), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    pos = torch.zeros((pages, page), dtype=torch.int32, device="cuda")
    order = np.random.RandomState(0).permutation(pages).astype(np.int32)
    cache, clen = api.PagedCache(cK, cV, pos, _cuda(order)), np.zeros(2, np.int32)
    page_off = np.array([0, per, 2 * per], np.int32)
    lens = [120, 77]
    off = inputs.offsets(lens)
    X = inputs.randn((off[-1], d), "server", "X", dtype=dtype).cuda()
    w = inputs.randn((d,), "server", "w", std=d ** -0.5, dtype=dtype).cuda()
    nug = inputs.offsets([dodo.num_nuggets(n, 3) for n in lens])
    scores, idx = torch.empty(int(off[-1]), device="cuda"), torch.empty(int(nug[-1]), dtype=torch.int32, device="cuda")
    dodo.score_select(X, w, 0.0, off, nug, 0, scores, idx)
    fused = lambda n, tag: inputs.randn((n, H + 2 * Hkv, dh), "server", tag, dtype=dtype).cuda()  # noqa: E731
    P = fused(int(off[-1]), "prompt")
    dodo.gather_kv_paged(P[:, H:H + Hkv], P[:, H + Hkv:], off, idx, nug, [0, 0], rope, cache, page_off, clen)
    half = plain64.HALF[NAME[dtype]]
    # what the caches hold: K rounded once on the way, taken from the pages and checked against the formula
    seen = [[], []]
    chosen = idx.cpu().numpy()
    for b in range(2):
        seen[b] += [(off[b] + i, int(i), P) for i in chosen[nug[b]:nug[b + 1]]]
    at = list(lens)
    ws = torch.empty(dodo.attend_paged_workspace_bytes(dh), dtype=torch.uint8, device="cuda")
    for step, tq in enumerate(([33, 5], [1, 1], [1, 1], [40, 1], [1, 0])):
        qo = inputs.offsets(tq)
        n = int(qo[-1])
        Y = fused(n, f"step {step}")
        raw = Y.clone()
        dodo.rope(rope, qo, at, Y[:, :H])
        dodo.gather_kv_paged(Y[:, H:H + Hkv], Y[:, H + Hkv:], qo, None, None, at, rope, cache, page_off, clen)
        O, L = torch.empty((n, H, dh), dtype=dtype, device="cuda"), torch.empty((n, H), device="cuda")
        Q = Y[:, :H].contiguous()
        dodo.attend_paged(Q, qo, at, dh ** -0.5, cache, page_off, clen, None, None, None, None, None, O, L, ws)
        torch.cuda.synchronize()
        for b in range(2):
            seen[b] += [(int(qo[b]) + t, at[b] + t, raw) for t in range(tq[b])]
            assert len(seen[b]) == clen[b]
            rows = np.array([order[page_off[b] + r // page] * page + r % page for r in range(clen[b])], np.int64)
            kpos = np.array([p for _, p, _ in seen[b]])
            assert pos.view(-1)[rows].tolist() == kpos.tolist()
            plain = np.stack([_f64(src[r, H:H + Hkv]) for r, _, src in seen[b]])
            want, bound = paged64.rope(plain, kpos, rope_freq, "half")
            K = _f64(cK.flatten(0, 1)[rows])
            assert (np.abs(K - want) <= bound + half * (np.abs(want) + bound)).all()
            if tq[b] == 0:
                continue
            q, qpos = _f64(Q[qo[b]:qo[b + 1]]), at[b] + np.arange(tq[b])
            want, bound = paged64.rope(_f64(raw[qo[b]:qo[b + 1], :H]), qpos, rope_freq, "half")
            assert (np.abs(q - want) <= bound + half * (np.abs(want) + bound)).all()
            V = _f64(cV.flatten(0, 1)[rows])
            o, l = paged64.attend(q, qpos, dh ** -0.5, K, V, kpos)
            tO, tL = paged64.attend_bounds(q, qpos, dh ** -0.5, K, V, kpos, o, l, half, half if dtype is BF else 0.0)
            assert (np.abs(_f64(O[qo[b]:qo[b + 1]]) - o) <= tO).all() and (np.abs(_f64(L[qo[b]:qo[b + 1]]) - l) <= tL).all()
        at = [a + t for a, t in zip(at, tq)]


def test_training_step_with_rotations(dodo):
    """Q and K turned, attended, the gradient of attend turned back: against differences of the whole in 64 bits."""
    T, H, dh = 12, 2, 64
    freq = api.rope_frequencies(dh)
    rope = api.Rope(freq, api.ROPE_INTERLEAVED)
    new = lambda n: inputs.randn((T, H, dh), "train rope", n, dtype=F32).cuda()  # noqa: E731
    Q, K, V, dO = new("Q"), new("K"), new("V"), new("dO")
    q, k = torch.empty_like(Q), torch.empty_like(K)
    dodo.rope(rope, [0, T], [50], Q, K, q, k)
    O, L = torch.empty_like(Q), torch.empty((T, H), device="cuda")
    scale = dh ** -0.5
    ws = torch.empty(max(dodo.attend_workspace_bytes(dh), dodo.attend_backward_workspace_bytes(T, H, dh, 0)), dtype=torch.uint8, device="cuda")
    dodo.attend(q, [0, T], [50], scale, None, None, None, None, None, k, V, [0], [T], [50], O, L, ws)
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    dodo.attend_backward(q, [0, T], [50], scale, None, None, None, None, None, k, V, [0], [T], [50], O, L, dO, dQ, None, None, dK, dV, None, ws)
    dodo.rope_backward(rope, [0, T], [50], dQ, dK)
    torch.cuda.synchronize()
    pos = 50 + np.arange(T)

    def loss(x, y):
        a, b = (paged64.rope(v, pos, freq, "interleaved")[0] for v in (x, y))
        return float((plain64.attend(a, pos, scale, b, _f64(V), pos)[0] * _f64(dO)).sum())

    rs, h = np.random.RandomState(2), 1e-4
    for _ in range(4):
        dx, dy = rs.standard_normal((T, H, dh)), rs.standard_normal((T, H, dh))
        slope = (loss(_f64(Q) + h * dx, _f64(K) + h * dy) - loss(_f64(Q) - h * dx, _f64(K) - h * dy)) / (2 * h)
        got = float((_f64(dQ) * dx).sum() + (_f64(dK) * dy).sum())
        # fp32 chains of some dh + T operations on each of the sums' terms, and the difference's h^2
        size = float((np.abs(_f64(dQ)) * np.abs(dx)).sum() + (np.abs(_f64(dK)) * np.abs(dy)).sum())
        assert abs(got - slope) <= (dh + T + 32) * 2.0 ** -23 * size * 4 + h * h * size * 10


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (8, 2, 4), (4, 2, 90)])
def test_rows_whose_every_logit_is_nan(dodo, dtype, H, Hkv, tq):
    """Nothing but a NaN in sight is no empty row: O and the log-sum-exp are NaN."""
    s = _batch(dtype, H, Hkv, 64, [tq], [1], [0], 16, q_pos0=[50], span=1)
    s["cK"][s["rows"][0]] = float("nan")
    O, L = _run(dodo, s)
    assert torch.isnan(O.float()).all() and torch.isnan(L).all()


@pytest.mark.parametrize("dtype,H,Hkv,tq", [(BF, 4, 2, 1), (F32, 4, 2, 3), (BF, 4, 4, 60)])
def test_without_a_workspace_no_list_is_cut(dodo, dtype, H, Hkv, tq):
    s = _batch(dtype, H, Hkv, 128, [tq], [3000], [tq], 16)
    O, L = _run(dodo, s, workspace=False)
    _check(s, O, L)


@pytest.mark.parametrize("tq,H,Hkv,dh", [(20, 16, 4, 64), (70, 16, 4, 128), (1, 8, 8, 128)])
@pytest.mark.parametrize("page", [5, 16])
def test_sequences_that_see_nothing_between_others(dodo, tq, H, Hkv, dh, page):
    """Every key of most sequences lies ahead of their queries: blocks with several pieces of work that have no key to read."""
    B = 48
    s = _batch(BF, H, Hkv, dh, [tq] * B, [300 + 7 * (b % 5) for b in range(B)], [0] * B, page)
    s["q_pos0"][:] = 10 ** 5
    for b in range(B):
        if b % 4 != 1:
            s["pos"][s["rows"][b]] = 10 ** 6
    O, L = _run(dodo, s)
    _check(s, O, L, only=[0, 1, 2, 3, 5, 45, 47])
    for b in range(B):
        if b % 4 != 1:
            q = slice(s["q_off"][b], s["q_off"][b + 1])
            assert not O[q].any() and torch.isneginf(L[q]).all()


@pytest.mark.parametrize("dtype,tq", [(BF, 1), (BF, 60), (F32, 3)])
def test_pool_of_no_pages(libdodo, dtype, tq):
    """No entry of the table is a page then: what is cached is not seen, the local tokens are."""
    own = api.Dodo(0)
    s = _batch(dtype, 4, 2, 64, [tq, tq], [40, 24], [tq, tq + 3], 8)
    s["pages"] = 0
    s["cK"], s["cV"] = s["cK"][:0], s["cV"][:0]
    shape = (0, 8, 2, 64)
    held = torch.zeros(64, device="cuda")         # an address to give: empty tensors have none
    cache = api.PagedCache(torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda"),
                           torch.empty(0, dtype=torch.int32, device="cuda"), _cuda(s["table"]))
    at = held.data_ptr()
    cache.spec = struct.pack("QQQQiiiiii", at, at, at, cache.table.data_ptr(), cache.code, 2, 64, 0, 8, 0)
    O, L = torch.full(s["Q"].shape, 7.0, dtype=dtype, device="cuda"), torch.full(s["Q"].shape[:2], 7.0, device="cuda")
    ws = torch.empty(own.attend_paged_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    own.attend_paged(s["Q"].cuda(), s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], s["lK"].cuda(), s["lV"].cuda(), s["loc_off"][:-1],
                     s["loc"], s["loc_pos0"], O, L, ws)
    torch.cuda.synchronize()
    assert own.device_status() == api.DEV_BAD_INDEX
    s["rows"], s["nug"] = [r[:0] for r in s["rows"]], np.zeros(2, np.int32)
    _check(s, O, L)
    own.reset()
    own.close()


@pytest.mark.parametrize("H,Hkv,tq,dh", [(16, 8, 12, 128), (16, 8, 40, 128), (24, 8, 11, 64), (8, 8, 70, 64)])
@pytest.mark.parametrize("kind", ["plain", "nan", "inf", "unseen", "seen nan", "long", "alone"])
def test_many_f32_rows(dodo, H, Hkv, tq, dh, kind):
    """Batches of fp32 rows that fill the device: rows of a tile that see different keys, tiles that end inside a page, cut lists."""
    B = 3 if kind in ("long", "alone") else 24
    nug = [1300, 1999, 771] if kind == "long" else [900, 0, 700] if kind == "alone" else [(53 * b) % 190 for b in range(B)]
    s = _batch(F32, H, Hkv, dh, [tq - b % 3 for b in range(B)], nug, [tq - b % 3 + b % 4 for b in range(B)], 24, span=3,
               fill=float("nan") if kind == "nan" else None)
    some = [0, 1, 2] if B == 3 else [0, 1, 5, 13, 14, 23]
    if kind in ("nan", "inf"):      # in keys that the last token of a sequence alone sees, and behind it
        for b in range(B):
            at = s["loc_off"][b] + max(int(s["q_off"][b + 1] - s["q_off"][b]) - 1, 0)
            s["lV"][at], s["lK"][at] = float(kind), 1.0
    if kind == "unseen":
        s["q_pos0"][::2] = -5 * tq
        s["pos"][s["rows"][1]] = 10 ** 6
    if kind == "seen nan":
        s["lK"][s["loc_off"][5] + 3] = float("nan")
    O, L = _run(dodo, s)
    if kind == "seen nan":
        q = slice(s["q_off"][5], s["q_off"][6])
        assert torch.isfinite(O[q][:2]).all() and torch.isnan(O[q][4:]).all()
        some.remove(5)
    if kind in ("nan", "inf"):
        for b in some:
            q, l = slice(s["q_off"][b], s["q_off"][b + 1]), s["loc_off"][b]
            n = q.stop - q.start - 1
            first = int(s["loc_pos0"][b] + n - s["q_pos0"][b])       # the first token that sees it
            assert torch.isfinite(O[q][:first]).all() and not torch.isfinite(O[q][first:]).any()
            s["lV"][l + n] = 0.0
            O[q][first:] = 0.0
            qq, Q, qpos, K, V, kpos = _sequence(s, b)
            o, lse = paged64.attend(Q, qpos, s["scale"], K, V, kpos)
            tO, _ = paged64.attend_bounds(Q, qpos, s["scale"], K, V, kpos, o, lse, plain64.HALF["f32"], 0.0)
            assert (np.abs(_f64(O[q]) - o) <= tO)[:first].all()
        return
    _check(s, O, L, only=some)
    if kind == "long":
        O2, L2 = _run(dodo, s, workspace=False)
        _check(s, O2, L2, only=some)


def test_many_f32_rows_behind_bad_pages_and_again(libdodo):
    own = api.Dodo(0)
    s = _batch(F32, 16, 8, 64, [20] * 20, [100] * 20, [20] * 20, 16)
    s["table"][1], s["table"][4], s["table"][8] = -1, s["pages"], 2 ** 31 - 1
    O, L = _run(own, s)
    assert own.device_status() == api.DEV_BAD_INDEX
    for b, gone in ((0, (1, 4)), (1, (1,))):
        keep = np.array([r // 16 not in gone for r in range(100)])
        s["rows"][b] = s["rows"][b][keep]
        s["nug"][b] = keep.sum()
    _check(s, O, L, only=[0, 1, 2, 19])
    own.reset()
    own.close()


@pytest.mark.parametrize("H,Hkv,tq,dh,nug", [(4, 4, 140, 64, 9001), (4, 2, 64, 128, 9001), (8, 8, 128, 128, 16000), (8, 2, 100, 64, 5000), (8, 4, 9, 128, 7000)])
def test_the_same_bits_every_time(dodo, H, Hkv, tq, dh, nug):
    """Lists that many blocks share: whichever of them comes last, the order of every sum is the same."""
    s = _batch(BF, H, Hkv, dh, [tq, 1], [nug, 40], [tq + 100, 1], 32, span=2)
    O, L = _run(dodo, s)
    for _ in range(20):
        O2, L2 = _run(dodo, s)
        assert torch.equal(O, O2) and torch.equal(L, L2)


@pytest.mark.parametrize("H,Hkv,tq", [(1, 1, 40), (4, 2, 37), (2, 2, 140)])
def test_ragged_batches_of_many_short_lists(dodo, H, Hkv, tq):
    """Units of one tile and of many side by side: shares that end within a unit's begin, blocks with nothing to do, order of the short ones."""
    B = 60
    nug = [(97 * b) % 250 if b % 19 else 3000 for b in range(B)]
    for page in (16, 5):
        s = _batch(BF, H, Hkv, 64, [tq - b % 4 for b in range(B)], nug, [tq - b % 4 if b % 3 else 0 for b in range(B)], page)
        s["q_pos0"][:] += 2000
        _check(s, *_run(dodo, s), only=[0, 1, 2, 18, 19, 20, 38, 57, 59])
        t = _batch(F32, H, Hkv, 64, [1 + b % 9 for b in range(B)], nug, [9] * B, page)
        _check(t, *_run(dodo, t), only=[0, 1, 19, 20, 59])
