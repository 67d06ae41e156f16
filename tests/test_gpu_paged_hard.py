"""Attention over the paged nugget cache where it can go wrong, on each of the kernels for many rows: the tensor cores' with tiles of 128 and of 256
rows, the fp32 tiles of 32 rows, and of 64 where there are enough.  Every test names the kernel that the call has to take, so that no rule of choice leads it elsewhere."""
import struct

import numpy as np
import pytest
import torch

import launched
import paged64
import plain64
from paper_2310_02409_b200 import api, inputs
from test_gpu_paged import BF, F32, NAME, _batch, _check, _check_masked, _cuda, _f64
from test_gpu_paged_choice import TENSOR_CORES, TILE, prepared, run_on, tensor_cores

pytestmark = pytest.mark.gpu

# kernel, type, query heads, KV heads, tokens, sequences, head size, rows of a page
FORMS = [pytest.param(*f, id="-".join(str(v) for v in (NAME[f[1]],) + f[2:])) for f in [
    (TENSOR_CORES, BF, 4, 2, 40, 2, 64, 16), (TENSOR_CORES, BF, 4, 2, 40, 2, 128, 16), (TENSOR_CORES, BF, 2, 2, 140, 2, 64, 16), (TENSOR_CORES, BF, 4, 2, 100, 2, 128, 16),
    (TENSOR_CORES, BF, 4, 2, 40, 2, 128, 5), (TENSOR_CORES, BF, 4, 2, 100, 2, 64, 1), (TENSOR_CORES, BF, 4, 2, 3, 2, 128, 64),
    (TILE, F32, 16, 8, 12, 20, 64, 16), (TILE, F32, 16, 8, 20, 20, 128, 24), (TILE, F32, 16, 8, 40, 20, 64, 5), (TILE, F32, 16, 8, 64, 56, 128, 16)]]
forms = pytest.mark.parametrize("kernel,dtype,H,Hkv,tq,B,dh,page", FORMS)
SOME = [0, 1]                        # sequences that are compared


@pytest.fixture()
def on(dodo):
    """Many bf16 rows on the tensor cores, whatever the work."""
    with tensor_cores(dodo, 1):
        yield dodo


@forms
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3e38])
def test_what_a_query_does_not_see_takes_no_part(on, kernel, dtype, H, Hkv, tq, B, dh, page, bad):
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [200] + [50] * (B - 1), [tq] + [tq + 3] * (B - 1), page, q_pos0=[1000] + [250] * (B - 1), seed=tq)
    for b in range(B):
        r = s["rows"][b]
        hidden = r[s["pos"][r] > int(s["q_pos0"][b]) + tq - 1]
        s["pos"][r[3]] = int(s["q_pos0"][b]) + tq // 2 + 1          # seen by the later queries only
        assert len(hidden) > 0
        s["cK"][hidden], s["cV"][hidden] = bad, bad
    clean = run_on(on, s, kernel)
    t = {k: (v.clone() if isinstance(v, torch.Tensor) else v) for k, v in s.items()}
    _check_masked(dict(t, B=2), *clean)
    early = [int(s["q_off"][b]) + t for b in range(B) for t in range(min(tq, tq // 2 + 1))]
    late = [int(s["q_off"][b]) + t for b in range(B) for t in range(tq // 2 + 1, tq)]
    for b in range(B):
        s["cV"][s["rows"][b][3]] = bad
    O, L = run_on(on, s, kernel)
    assert torch.equal(L, clean[1])
    if bad != -3e38:
        assert late and not torch.isfinite(O[late].float()).any()
    # what the earlier queries get is the plain form's still
    for b in range(B):
        s["cV"][s["rows"][b][3]] = 0.0
    O[late] = run_on(on, s, kernel)[0][late]
    _check_masked(dict(s, B=2), O, L)
    assert torch.isfinite(O[early].float()).all()


@forms
def test_a_visible_nan_shows(on, kernel, dtype, H, Hkv, tq, B, dh, page):
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [60] * B, [tq] * B, page)
    s["cK"][s["rows"][0][7], 0, 5] = float("nan")
    s["cV"][s["rows"][1][9], Hkv - 1, 11] = float("nan")
    s["lK"][s["loc_off"][0] + tq - 1, 1, 0] = float("nan")         # seen by the last query of the sequence alone
    O, L = run_on(on, s, kernel)
    g = H // Hkv
    nan_o, nan_l = torch.zeros(O.shape, dtype=torch.bool), torch.zeros(L.shape, dtype=torch.bool)
    nan_o[:tq, :g], nan_l[:tq, :g] = True, True
    nan_o[tq - 1, g:2 * g], nan_l[tq - 1, g:2 * g] = True, True
    nan_o[tq:2 * tq, H - g:, 11] = True
    assert torch.equal(torch.isnan(O.float()).cpu(), nan_o) and torch.equal(torch.isnan(L).cpu(), nan_l)


@forms
def test_rows_whose_every_logit_is_nan(on, kernel, dtype, H, Hkv, tq, B, dh, page):
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [1] * B, [0] * B, page, q_pos0=[500] * B, span=1)
    for b in range(B):
        s["cK"][s["rows"][b]] = float("nan")
    O, L = run_on(on, s, kernel)
    assert torch.isnan(O.float()).all() and torch.isnan(L).all()


@forms
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-12, 2e-9, 30.0])
def test_scales(on, kernel, dtype, H, Hkv, tq, B, dh, page, scale):
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [300] * B, [tq] * B, page)
    s["scale"] = scale
    if kernel == TENSOR_CORES and scale < 1e-9:
        pytest.skip("the tensor cores do not take such scales")
    _check(s, *run_on(on, s, kernel), only=SOME)


@forms
@pytest.mark.parametrize("octaves", [20, 26, 40])
@pytest.mark.parametrize("n", [500, 2500])
def test_weights_that_rise_from_tile_to_tile(on, kernel, dtype, H, Hkv, tq, B, dh, page, octaves, n):
    """Every 128 (630) keys the weights are so many octaves up and V as many down: each of four parts has its share in the result, and results
    so far have to be scaled by a factor that is neither 1 nor 0.  Rows of the same tile rise at different keys."""
    if kernel == TILE:
        B = B if n == 500 else 4
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [n] * B, [tq] * B, page, span=1)
    s["scale"] = 1.0
    s["Q"].zero_()
    for t in range(2):
        s["Q"][t::2, :, t] = 1.0                                   # even tokens see feature 0 of K, odd ones feature 1
    s["lK"].zero_()
    s["lK"][:, :, :2] = -200.0
    for b in range(B):
        r = s["rows"][b]
        s["cK"][r] = 0.0
        for t in range(2):
            part = np.minimum((np.arange(n) + 37 * t) // (n // 4 + 3), 3)
            s["cK"][r, :, t] = torch.tensor(part * octaves * np.log(2.0), dtype=torch.float64)[:, None].to(dtype)
        s["cV"][r] = (s["cV"][r].double() * torch.tensor(2.0 ** (octaves * (3 - part)))[:, None, None]).to(dtype)
    O, L = run_on(on, s, kernel)
    _check(s, O, L, only=[0])
    for _ in range(3):
        O2, L2 = run_on(on, s, kernel)
        assert torch.equal(O, O2) and torch.equal(L, L2)


@forms
def test_sequences_share_pages(on, kernel, dtype, H, Hkv, tq, B, dh, page):
    """All sequences over one prefix: the same pages in every table, pages of their own behind them."""
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [80] + [120] * (B - 1), [tq] * B, page, span=1)
    shared = 80 // page if page < 64 else 1
    for b in range(1, B):
        n, at = shared * page, int(s["page_off"][b])
        s["table"][at:at + shared] = s["table"][:shared]
        s["rows"][b][:n] = (s["table"][np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page)
    for b in range(B):
        s["pos"][s["rows"][b]] = np.arange(len(s["rows"][b]))
    _check(s, *run_on(on, s, kernel), only=SOME)


@forms
def test_bad_pages_are_not_followed(libdodo, kernel, dtype, H, Hkv, tq, B, dh, page):
    own = api.Dodo(0)
    n = 7 * page + page // 2 + 1
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [n] * B, [tq] * B, page)
    per = int(s["page_off"][1])
    gone = ((0, 1, -1), (0, 4, s["pages"]), (1, 0, 2 ** 31 - 1), (1, per - 1, -2 ** 31))
    for b, entry, bad in gone:
        s["table"][per * b + entry] = bad
    with tensor_cores(own, 1):
        O, L = run_on(own, s, kernel)
    assert own.device_status() == api.DEV_BAD_INDEX
    for b in range(2):
        keep = np.array([r // page not in [e for c, e, _ in gone if c == b] for r in range(n)])
        s["rows"][b] = s["rows"][b][keep]
        s["nug"][b] = keep.sum()
    _check(s, O, L, only=SOME)
    own.reset()
    own.close()


@forms
def test_queries_inside_and_ahead_of_the_context(on, kernel, dtype, H, Hkv, tq, B, dh, page):
    """Queries that see part of the nuggets, none of them, or (a position before everything) nothing at all."""
    B += 2
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [300] * (B - 1) + [0], [0] + [10] * (B - 1), page, q_pos0=[1500, 100] + [-5000] * (B - 2), seed=tq)
    O, L = run_on(on, s, kernel)
    _check(s, O, L, only=[0, 1, 2, B - 1])
    blind = slice(int(s["q_off"][2]), int(s["q_off"][B]))
    assert (O[blind] == 0).all() and torch.isneginf(L[blind]).all()


@forms
def test_without_cache_without_local_without_lse(on, kernel, dtype, H, Hkv, tq, B, dh, page):
    B = 20 if kernel == TILE else 2
    for nug, loc, pos in (([0] * B, [tq + 2] * B, None), ([50] * (B - 1) + [0], [0] * B, [600] * B)):
        s = _batch(dtype, H, Hkv, dh, [tq] * (B - 1) + [1], nug, loc, page, q_pos0=pos)
        call, O, L = prepared(on, s)
        shape = (s["pages"], s["page"], Hkv, dh)
        cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
        ws, Q = torch.empty(on.attend_paged_workspace_bytes(dh), dtype=torch.uint8, device="cuda"), s["Q"].cuda()
        local = (s["lK"].cuda(), s["lV"].cuda(), s["loc_off"][:-1], s["loc"], s["loc_pos0"]) if pos is None else (None,) * 5
        no_lse = lambda: on.attend_paged(Q, s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], *local, O, None, ws)  # noqa: E731
        no_lse()
        torch.cuda.synchronize()
        assert all(kernel in n for n in launched.kernels(no_lse)) and (L == 7.0).all()
        _check(s, O, None, only=[0, 1, B - 1])
        if pos is not None:
            assert (O[-1] == 0).all()


@forms
def test_pool_of_no_pages(libdodo, kernel, dtype, H, Hkv, tq, B, dh, page):
    """No entry of the table is a page then: what is cached is not seen, the local tokens are."""
    own = api.Dodo(0)
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [40] * B, [tq + 1] * B, page)
    held, empty = torch.zeros(64, device="cuda"), torch.empty((0, page, Hkv, dh), dtype=dtype, device="cuda")
    cache, at = api.PagedCache(empty, empty, torch.empty((0, page), dtype=torch.int32, device="cuda"), _cuda(s["table"])), held.data_ptr()
    cache.spec = struct.pack("QQQQiiiiii", at, at, at, cache.table.data_ptr(), cache.code, Hkv, dh, 0, page, 0)     # empty tensors have no address
    O, L = torch.full(s["Q"].shape, 7.0, dtype=dtype, device="cuda"), torch.full(s["Q"].shape[:2], 7.0, device="cuda")
    ws = torch.empty(own.attend_paged_workspace_bytes(dh), dtype=torch.uint8, device="cuda")
    Q, lK, lV = s["Q"].cuda(), s["lK"].cuda(), s["lV"].cuda()
    call = lambda: own.attend_paged(Q, s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], lK, lV, s["loc_off"][:-1], s["loc"],  # noqa: E731
                                    s["loc_pos0"], O, L, ws)
    with tensor_cores(own, 1):
        call()
        torch.cuda.synchronize()
        assert all(kernel in n for n in launched.kernels(call))
    assert own.device_status() == api.DEV_BAD_INDEX
    s["rows"], s["nug"] = [r[:0] for r in s["rows"]], np.zeros(B, np.int32)
    _check(s, O, L, only=SOME)
    own.reset()
    own.close()


@forms
def test_captured_replayed_and_on_two_streams(libdodo, kernel, dtype, H, Hkv, tq, B, dh, page):
    """Graphs of two contexts with a workspace each, replayed at once on two streams, lists that are cut among them; an eager call between."""
    sets = []
    for i in range(2):
        d = api.Dodo(0)
        s = _batch(dtype, H, Hkv, dh, [tq] * B, [2000] + [70] * (B - 1), [tq + 64] * B, page, seed=i)
        with tensor_cores(d, 1):
            call, O, L = prepared(d, s)
            call()
            torch.cuda.synchronize()
            _check(s, O, L, only=[i])
            assert all(kernel in n for n in launched.kernels(call))
            side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call()
        sets.append((d, O, L, (O.clone(), L.clone()), side, graph, call))
    for _ in range(3):
        for d, O, L, want, side, graph, call in sets:
            O.zero_()
            L.zero_()
        torch.cuda.synchronize()
        for d, O, L, want, side, graph, call in sets:
            with torch.cuda.stream(side), tensor_cores(d, 1):
                graph.replay()
                call()
                graph.replay()
        torch.cuda.synchronize()
        for d, O, L, want, side, graph, call in sets:
            assert torch.equal(O, want[0]) and torch.equal(L, want[1])
    for d, *_ in sets:
        assert d.device_status() == 0
        d.close()


@pytest.mark.parametrize("kernel,dtype,tq,B", [(TENSOR_CORES, BF, 64, 1), (TENSOR_CORES, BF, 200, 2), (TILE, F32, 64, 10), (TILE, F32, 30, 10)])
def test_pool_behind_2_31_elements(on, kernel, dtype, tq, B):
    """Rows of K and V whose elements have indices beyond 32 bits; every sequence reads the same pages."""
    H, dh, page, n = 8, 128, 16, 300
    pages = (2 ** 31 // (H * dh)) // page + 40
    if torch.cuda.mem_get_info()[0] < 2 * pages * page * H * dh * 4 + (2 << 30):
        pytest.skip("needs more device memory")
    one = np.concatenate([np.arange(pages - 15, pages), np.arange(4)]).astype(np.int32)
    rows = np.array([one[r // page] * page + r % page for r in range(n)], np.int64)
    cK, cV = (torch.zeros((pages, page, H, dh), dtype=dtype, device="cuda") for _ in range(2))
    pos = torch.zeros((pages, page), dtype=torch.int32, device="cuda")
    K, V = (inputs.randn((n, H, dh), "far", x, dtype=dtype) for x in "KV")
    on.gather_kv_paged(K.cuda(), V.cuda(), [0, n], None, None, [0], None, api.PagedCache(cK, cV, pos, _cuda(one)), [0, len(one)], np.zeros(1, np.int32))
    assert torch.equal(cK.flatten(0, 1)[_cuda(rows)].cpu(), K)
    cache, off = api.PagedCache(cK, cV, pos, _cuda(np.tile(one, B))), np.arange(B + 1, dtype=np.int32) * len(one)
    Q = inputs.randn((B * tq, H, dh), "far", "Q", dtype=dtype)
    Qd, O, L = Q.cuda(), torch.zeros((B * tq, H, dh), dtype=dtype, device="cuda"), torch.zeros((B * tq, H), device="cuda")
    ws = torch.empty(on.attend_paged_workspace_bytes(dh), dtype=torch.uint8, device="cuda")
    call = lambda: on.attend_paged(Qd, np.arange(B + 1) * tq, [n - tq] * B, dh ** -0.5, cache, off, [n] * B, None, None, None, None, None, O, L, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    assert all(kernel in k for k in launched.kernels(call))
    qpos, kpos, half = n - tq + np.arange(tq), np.arange(n), plain64.HALF[NAME[dtype]]
    for b in (0, B - 1):
        q = slice(b * tq, (b + 1) * tq)
        o, l = paged64.attend(_f64(Q[q]), qpos, dh ** -0.5, _f64(K), _f64(V), kpos)
        tO, tL = paged64.attend_bounds(_f64(Q[q]), qpos, dh ** -0.5, _f64(K), _f64(V), kpos, o, l, half, half if dtype is BF else 0.0)
        assert (np.abs(_f64(O[q]) - o) <= tO).all() and (np.abs(_f64(L[q]) - l) <= tL).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv,tq,B,nug", [(4, 4, 64, 60, 300), (4, 4, 130, 60, 200), (2, 1, 300, 8, 4000), (2, 2, 20, 1, 9000)])
def test_whole_units_and_units_in_equal_pieces(on, dh, H, Hkv, tq, B, nug):
    """Alike units, more and fewer than the device has blocks for: whole ones, and ones cut into as many pieces each."""
    s = _batch(BF, H, Hkv, dh, [tq] * B, [nug] * B, [tq] * B, 16, span=2)
    O, L = run_on(on, s, TENSOR_CORES)
    _check(s, O, L, only=[0, B // 2, B - 1])
