"""attend's gradient on the GPU against the formula in 64 bits, with bounds from the number of operations, and as a training step
uses it: behind the forward call, in a captured graph, with rows and regions that are not its own left alone."""
import numpy as np
import pytest
import torch

import plain64
from paper_2310_02409_b200 import api, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def problem(tag, dtype, H, dh, tqs, clens, llens, inside=False, slack=2, scale=None, std=1.0, nan_slack=True):
    """A ragged batch with slack rows (NaN) behind every region; O and lse come from dodo_attend (see forward)."""
    rs = np.random.RandomState(inputs.seed_for(tag) % 2 ** 32)
    B = len(tqs)
    p = dict(B=B, H=H, dh=dh, dtype=dtype, scale=dh ** -0.5 if scale is None else scale)
    p["q_off"], p["cache_off"] = inputs.offsets(tqs), inputs.offsets([c + slack for c in clens])
    p["clen"], p["llen"] = np.asarray(clens, np.int32), np.asarray(llens, np.int32)
    p["loc_off"] = inputs.offsets([n + slack for n in llens])[:-1].copy()
    rows, lrows = int(p["cache_off"][-1]), int(sum(n + slack for n in llens))
    span = [5 * c + 3 for c in clens]
    p["loc_pos0"] = np.asarray(span, np.int32)
    p["q_pos0"] = np.asarray([max(0, s // 2 - t // 2 - 1) if inside else s + n - t for s, n, t in zip(span, llens, tqs)], np.int32)
    draw = lambda r: torch.from_numpy(std * rs.standard_normal((r, H, dh))).to(dtype)  # noqa: E731
    p["cK"], p["cV"], p["lK"], p["lV"] = draw(rows), draw(rows), draw(lrows), draw(lrows)
    p["Q"], p["dO"] = draw(int(p["q_off"][-1])), draw(int(p["q_off"][-1]))
    p["cpos"] = np.zeros(rows, np.int32)
    p["live_c"], p["live_l"] = np.zeros(rows, bool), np.zeros(lrows, bool)
    for b in range(B):
        c0 = int(p["cache_off"][b])
        p["cpos"][c0:c0 + clens[b]] = np.sort(rs.permutation(span[b])[:clens[b]])
        p["live_c"][c0:c0 + clens[b]] = True
        p["live_l"][p["loc_off"][b]:p["loc_off"][b] + llens[b]] = True
    if nan_slack:
        for n, live in (("cK", "live_c"), ("cV", "live_c"), ("lK", "live_l"), ("lV", "live_l")):
            p[n][torch.from_numpy(~p[live])] = float("nan")
    return p


def forward(dodo, p):
    d = {n: p[n].cuda() for n in ("Q", "cK", "cV", "lK", "lV", "dO")}
    d["cpos"] = _cuda(p["cpos"])
    d["O"] = torch.zeros_like(d["Q"])
    d["lse"] = torch.full(d["Q"].shape[:2], -float("inf"), device="cuda")
    ws = torch.empty(dodo.attend_workspace_bytes(p["dh"]), dtype=torch.uint8, device="cuda")
    dodo.attend(d["Q"], p["q_off"], p["q_pos0"], p["scale"], d["cK"], d["cV"], d["cpos"], p["cache_off"], p["clen"], d["lK"], d["lV"],
                p["loc_off"], p["llen"], p["loc_pos0"], d["O"], d["lse"], ws)
    return d


def buffers(d, fill=7.0):
    out = {n: torch.full_like(d[s], fill) for n, s in (("dQ", "Q"), ("dcK", "cK"), ("dcV", "cV"), ("dlK", "lK"), ("dlV", "lV"))}
    out["dscore"] = torch.full((d["cK"].shape[0],), fill, device="cuda")
    return out


def backward(dodo, p, d, out=None, scores=True, ws=None):
    out = buffers(d) if out is None else out
    if ws is None:
        n = dodo.attend_backward_workspace_bytes(d["Q"].shape[0], p["H"], p["dh"], int(p["cache_off"][-1]))
        ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")      # (NaN in every format)
        guard = ws[n:]
        ws = ws[:n]
    else:
        guard = None
    dodo.attend_backward(d["Q"], p["q_off"], p["q_pos0"], p["scale"], d["cK"], d["cV"], d["cpos"], p["cache_off"], p["clen"], d["lK"],
                         d["lV"], p["loc_off"], p["llen"], p["loc_pos0"], d["O"], d["lse"], d["dO"], out["dQ"], out["dcK"], out["dcV"],
                         out["dlK"], out["dlV"], out["dscore"] if scores else None, ws)
    if guard is not None:
        assert bool((guard == 0xff).all())
    return out


def check(p, d, out, dense=False, fill=7.0, scores=True):
    half = plain64.HALF["bf16" if p["dtype"] == BF else "f32"]
    Q, O, dO, lse = (_f64(d[n]) for n in ("Q", "O", "dO", "lse"))
    cK, cV, lK, lV = (_f64(p[n]) for n in ("cK", "cV", "lK", "lV"))
    got = {n: _f64(t) for n, t in out.items()}
    worst = {}
    for b in range(p["B"]):
        q = slice(int(p["q_off"][b]), int(p["q_off"][b + 1]))
        c = slice(int(p["cache_off"][b]), int(p["cache_off"][b]) + int(p["clen"][b]))
        l = slice(int(p["loc_off"][b]), int(p["loc_off"][b]) + int(p["llen"][b]))
        n = c.stop - c.start
        k, v = np.concatenate([cK[c], lK[l]]), np.concatenate([cV[c], lV[l]])
        kpos = np.concatenate([p["cpos"][c], p["loc_pos0"][b] + np.arange(p["llen"][b])])
        ref, tol = plain64.backward_with_bounds(Q[q], p["q_pos0"][b] + np.arange(q.stop - q.start), p["scale"], k, v, kpos, O[q], lse[q],
                                                dO[q], half, plain64.HALF["bf16"] if dense else 0.0)
        pairs = [("dQ", got["dQ"][q], ref[0], tol[0]), ("dcK", got["dcK"][c], ref[1][:n], tol[1][:n]), ("dlK", got["dlK"][l], ref[1][n:], tol[1][n:]),
                 ("dcV", got["dcV"][c], ref[2][:n], tol[2][:n]), ("dlV", got["dlV"][l], ref[2][n:], tol[2][n:])]
        if scores:
            pairs.append(("dscore", got["dscore"][c], ref[3][:n], tol[3][:n]))
        for name, g, r, t in pairs:
            assert np.all(np.isfinite(g)), (name, b)
            bad = np.abs(g - r) > t + 1e-30
            assert not bad.any(), (name, b, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.max(np.abs(g - r) - t)))
            if r.size:
                worst[name] = max(worst.get(name, 0.0), float(np.linalg.norm(g - r) / max(1e-30, np.linalg.norm(r))))
    # rows that belong to nobody keep what they held
    assert np.all(got["dcK"][~p["live_c"]] == fill) and np.all(got["dcV"][~p["live_c"]] == fill)
    assert np.all(got["dlK"][~p["live_l"]] == fill) and np.all(got["dlV"][~p["live_l"]] == fill)
    assert np.all(got["dscore"][~p["live_c"] if scores else slice(None)] == fill)
    return worst


SHAPES = [
    # dtype, H, dh, query tokens, cached rows, local rows
    (BF, 4, 128, [1] * 8, [205] * 8, [64] * 8),
    (BF, 2, 128, [1, 1, 0, 1, 1], [0, 1, 50, 129, 1000], [1, 0, 3, 7, 130]),
    (F32, 3, 64, [1, 1, 1], [700, 5, 0], [64, 1, 33]),
    (F32, 2, 128, [2, 1, 2], [33, 300, 64], [2, 9, 70]),
    (BF, 3, 64, [3, 4, 1, 0, 2], [257, 31, 8, 40, 0], [5, 4, 1, 3, 66]),
    (F32, 4, 64, [16], [52], [16]),
    (F32, 2, 128, [33, 5, 64], [70, 0, 129], [40, 5, 64]),
    (BF, 2, 64, [7, 100, 0, 31], [300, 64, 20, 1], [7, 130, 9, 31]),
    (F32, 1, 64, [65], [2000], [65]),
    (F32, 3, 128, [8, 5, 0, 1], [205, 1300, 9, 64], [64, 5, 3, 1]),
    (F32, 2, 128, [9, 16, 2], [130, 0, 700], [9, 80, 33]),
    (F32, 3, 64, [5, 17, 8], [64, 65, 300], [70, 17, 8]),
]


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_gradient_against_plain(dodo, errlog, case, inside):
    dtype, H, dh, tqs, cl, ll = SHAPES[case]
    p = problem(("bwd", case, inside), dtype, H, dh, tqs, cl, ll, inside)
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    worst = check(p, d, out, dense=dtype == BF and max(tqs) > 4)
    errlog.add(f"attend_backward {SHAPES[case]} {inside}", **{"rel_" + n: v for n, v in worst.items()})
    again = backward(dodo, p, d)                                  # bit for bit the same again, with and without scores
    bare = backward(dodo, p, d, scores=False)
    torch.cuda.synchronize()
    assert all(torch.equal(out[n].nan_to_num(5.0), again[n].nan_to_num(5.0)) for n in out)
    assert all(torch.equal(out[n], bare[n]) for n in out if n != "dscore") and bool((bare["dscore"] == 7.0).all())
    assert dodo.device_status() == 0


DENSE = [
    # H, query tokens, cached rows, local rows (bf16, head size 128, more than four queries: tensor cores)
    (2, [64], [128], [64]),
    (1, [5], [1], [5]),
    (2, [128], [0], [128]),
    (3, [16, 200, 0, 1], [70, 333, 129, 0], [16, 230, 9, 65]),
    (2, [256], [717], [320]),
    (1, [512], [130], [512]),
    (4, [33, 7], [2000, 64], [40, 7]),
    (32, [130] * 3, [205] * 3, [194] * 3),
    (1, [65, 127, 129], [63, 64, 65], [65, 191, 129]),
]
DENSE_64 = [(2, [64], [128], [64]), (3, [16, 200, 0, 1], [70, 333, 129, 0], [16, 230, 9, 65]), (5, [33, 7], [2000, 64], [40, 7]),
            (31, [76, 100, 69], [29, 591, 3], [94, 627, 74]), (1, [5], [0], [700])]


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("dh,case", [(128, i) for i in range(len(DENSE))] + [(64, i) for i in range(len(DENSE_64))])
def test_gradient_on_tensor_cores(dodo, errlog, dh, case, inside):
    H, tqs, cl, ll = (DENSE if dh == 128 else DENSE_64)[case]
    p = problem(("bwdtc", case, inside, dh), BF, H, dh, tqs, cl, ll, inside)
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    assert dodo.device_status() == 0
    worst = check(p, d, out, dense=True)
    errlog.add(f"attend_backward tensor cores {dh} {(H, tqs, cl, ll)} {inside}", **{"rel_tc_" + n: v for n, v in worst.items()})
    again = backward(dodo, p, d)
    bare = backward(dodo, p, d, scores=False)
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], again[n]) for n in out)
    assert all(torch.equal(out[n], bare[n]) for n in out if n != "dscore") and bool((bare["dscore"] == 7.0).all())


@pytest.mark.parametrize("dh", [128, 64])
def test_gradient_on_tensor_cores_many_sequences(dodo, dh):
    rs = np.random.RandomState(12)
    tqs, cl, ll = rs.randint(0, 90, 67), rs.randint(0, 200, 67), rs.randint(0, 100, 67)
    p = problem("bwdtcmany", BF, 2, dh, tqs.tolist(), cl.tolist(), ll.tolist())
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    check(p, d, out, dense=True)
    assert dodo.device_status() == 0


def test_gradient_of_many_sequences(dodo):
    # 70 sequences: two launch groups share the workspace
    rs = np.random.RandomState(2)
    for most in (1, 9):
        tqs, cl, ll = rs.randint(0, most + 1, 70), rs.randint(0, 90, 70), rs.randint(0, 40, 70)
        p = problem(("bwdmany", most), F32, 2, 64, tqs.tolist(), cl.tolist(), ll.tolist())
        d = forward(dodo, p)
        out = backward(dodo, p, d)
        torch.cuda.synchronize()
        check(p, d, out)


@pytest.mark.parametrize("dtype,dh,tq", [(F32, 64, 1), (F32, 64, 20), (BF, 128, 3), (BF, 64, 40), (BF, 128, 40)])
def test_gradient_negative_and_zero_scale(dodo, dtype, dh, tq):
    for scale in (-0.1, 0.0):
        p = problem(("bwdscale", dh, tq, scale), dtype, 2, dh, [tq], [100], [tq + 3], scale=scale)
        d = forward(dodo, p)
        out = backward(dodo, p, d)
        torch.cuda.synchronize()
        check(p, d, out, dense=dtype == BF and tq > 4)


@pytest.mark.parametrize("dtype,H,dh,tq", [(F32, 2, 64, 2), (F32, 2, 128, 40), (F32, 2, 128, 8), (F32, 2, 64, 12), (BF, 2, 64, 70), (BF, 2, 128, 4), (BF, 2, 128, 70)])
def test_gradient_masked_rows_may_hold_anything(dodo, dtype, H, dh, tq):
    """Nuggets ahead of every query, and local tokens behind it, hold NaN and infinities: their own gradients are 0, nobody
    else's changes; queries before the first key get 0."""
    p = problem(("bwdnan", dh, tq), dtype, H, dh, [tq, tq], [200, 90], [tq, 5], inside=True)
    p["q_pos0"][1] = -tq                       # sees nothing at all
    d = forward(dodo, p)
    clean = backward(dodo, p, d)
    torch.cuda.synchronize()
    check(p, d, clean, dense=dtype == BF and tq > 4)
    bad = dict(p)
    for b in range(2):
        c0, n = int(p["cache_off"][b]), int(p["clen"][b])
        hidden = torch.from_numpy(c0 + np.flatnonzero(p["cpos"][c0:c0 + n] > p["q_pos0"][b] + tq - 1))
        assert len(hidden) > 10
        for name, v in (("cK", float("nan")), ("cV", float("inf"))):
            bad[name] = bad[name].clone()
            bad[name][hidden] = v
    for name in ("lK", "lV"):
        bad[name] = torch.full_like(p[name], float("-inf"))
    db = {**d, **{n: bad[n].cuda() for n in ("cK", "cV", "lK", "lV")}}
    out = backward(dodo, bad, db)
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], clean[n]) for n in out)
    assert bool((out["dQ"][tq:] == 0).all())


@pytest.mark.parametrize("dtype,dh,tq", [(F32, 64, 2), (F32, 128, 24), (F32, 128, 7), (F32, 64, 13), (BF, 64, 40), (BF, 128, 100)])
def test_gradient_partly_visible_nan_key(dodo, dtype, dh, tq):
    """A key that only later queries see holds NaN: earlier queries' dQ is untouched."""
    p = problem(("bwdpart", dh, tq), dtype, 1, dh, [tq], [0], [tq], slack=0)
    d = forward(dodo, p)
    clean = backward(dodo, p, d)
    d2 = dict(d)
    d2["lK"] = d["lK"].clone()
    d2["lK"][tq - 1] = float("nan")            # the last query's own token
    out = backward(dodo, p, d2)
    torch.cuda.synchronize()
    assert torch.equal(out["dQ"][:tq - 1], clean["dQ"][:tq - 1])
    assert bool(torch.isnan(out["dQ"][tq - 1]).all())


def test_gradient_against_differences(dodo):
    # the whole step by differences of the plain forward: dQ, dK, dV of the fp32 kernels
    p = problem("bwddiff", F32, 2, 64, [6], [20], [6], slack=0)
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    Q, dO = _f64(p["Q"]), _f64(p["dO"])
    kpos = np.concatenate([p["cpos"], p["loc_pos0"][0] + np.arange(6)])
    K, V = np.concatenate([_f64(p["cK"]), _f64(p["lK"])]), np.concatenate([_f64(p["cV"]), _f64(p["lV"])])
    qpos = p["q_pos0"][0] + np.arange(6)
    loss = lambda a: float(np.sum(plain64.attend(a[0], qpos, p["scale"], a[1], a[2], kpos)[0] * dO))  # noqa: E731
    got = [_f64(out["dQ"]), np.concatenate([_f64(out["dcK"]), _f64(out["dlK"])]), np.concatenate([_f64(out["dcV"]), _f64(out["dlV"])])]
    rs, e = np.random.RandomState(4), 1e-5
    for which in range(3):
        for _ in range(25):
            a, b = [Q.copy(), K.copy(), V.copy()], [Q.copy(), K.copy(), V.copy()]
            i = tuple(rs.randint(0, s) for s in a[which].shape)
            a[which][i] += e
            b[which][i] -= e
            # central differences: cut-off of order e^2, 64-bit cancellation of order 1e-16 |loss| / e; fp32 results about 1e-5
            assert abs((loss(a) - loss(b)) / (2 * e) - got[which][i]) < 1e-4


@pytest.mark.parametrize("dtype,H,dh,tqs", [(F32, 2, 64, [1, 2]), (F32, 2, 64, [20, 3]), (BF, 2, 128, [2, 1]), (BF, 2, 128, [40, 65]), (BF, 2, 64, [40, 65])])
def test_gradient_captured_and_replayed(dodo, dtype, H, dh, tqs):
    """Forward and gradient of two problems in one graph on a stream of its own, with a shared workspace, replayed on new data."""
    ps = [problem(("bwdgraph", i, dh, tqs[0]), dtype, H, dh, tqs, [150, 60], [tqs[0] + 3, tqs[1]], inside=bool(i)) for i in range(2)]
    ws = torch.empty(max(dodo.attend_backward_workspace_bytes(int(p["q_off"][-1]), H, dh, int(p["cache_off"][-1])) for p in ps),
                     dtype=torch.uint8, device="cuda")
    ds = [forward(dodo, p) for p in ps]
    eager = [backward(dodo, p, d, ws=ws) for p, d in zip(ps, ds)]
    torch.cuda.synchronize()
    outs = [buffers(d) for d in ds]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for p, d, o in zip(ps, ds, outs):
            backward(dodo, p, d, o, ws=ws)
    for t in ds:
        t["dO"].mul_(2.0)                      # exact in either type: every gradient doubles
    for _ in range(2):
        for o in outs:
            for t in o.values():
                t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for p, o, e in zip(ps, outs, eager):
            for n in e:
                live = p["live_c"] if n in ("dcK", "dcV", "dscore") else p["live_l"] if n in ("dlK", "dlV") else np.ones(o[n].shape[0], bool)
                live = torch.from_numpy(live).cuda()
                assert torch.equal(o[n][live], 2.0 * e[n][live]), n
                assert bool((o[n][~live] == 7.0).all())


def test_gradient_without_a_segment_or_queries(dodo):
    p = problem("bwdseg", F32, 2, 64, [3, 9], [40, 20], [0, 0], slack=0)
    d = forward(dodo, p)
    out = buffers(d)
    ws = torch.empty(dodo.attend_backward_workspace_bytes(12, 2, 64, 60), dtype=torch.uint8, device="cuda")
    dodo.attend_backward(d["Q"], p["q_off"], p["q_pos0"], p["scale"], d["cK"], d["cV"], d["cpos"], p["cache_off"], p["clen"], None, None, None,
                         None, None, d["O"], d["lse"], d["dO"], out["dQ"], out["dcK"], out["dcV"], None, None, out["dscore"], ws)
    torch.cuda.synchronize()
    check(p, d, out)
    # no queries: the keys' gradients are zeros
    z = np.zeros(3, np.int32)
    empty = torch.empty((0, 2, 64), device="cuda")
    dodo.attend_backward(empty, z, p["q_pos0"], p["scale"], d["cK"], d["cV"], d["cpos"], p["cache_off"], p["clen"], None, None, None, None,
                         None, empty, torch.empty((0, 2), device="cuda"), empty, empty, out["dcK"], out["dcV"], None, None, out["dscore"], ws)
    torch.cuda.synchronize()
    assert not out["dcK"].any() and not out["dcV"].any() and not out["dscore"].any()


def test_training_step_of_the_scorer(dodo, oracle):
    """Score, select, gather, attend, gradient, and from the nuggets' score gradients the Scorer's (dw = sum dscore_j x_j): the
    whole against the formula in 64 bits on the rows that the GPU selected."""
    n, dm, H, dh, r, tq = 300, 256, 4, 64, 10, 16
    X = inputs.randn((n, dm), "bwdtrain", "X")
    w = inputs.randn((dm,), "bwdtrain", "w", std=dm ** -0.5)
    K, V = (inputs.randn((n, H, dh), "bwdtrain", k) for k in "KV")
    Q, lK, lV, dO = (inputs.randn((tq, H, dh), "bwdtrain", k) for k in ("Q", "lK", "lV", "dO"))
    k = dodo.num_nuggets(n, r)
    scores, idx = torch.empty(n, device="cuda"), torch.empty(k, dtype=torch.int32, device="cuda")
    cK, cV = torch.zeros((k, H, dh), device="cuda"), torch.zeros((k, H, dh), device="cuda")
    cpos, clen = torch.zeros(k, dtype=torch.int32, device="cuda"), np.zeros(1, np.int32)
    dodo.compress(X.cuda(), w.cuda(), 0.0, K.cuda(), V.cuda(), [0, n], [0, k], [0], 0, scores, idx, cK, cV, cpos, [0, k], clen)
    p = dict(B=1, H=H, dh=dh, dtype=F32, scale=dh ** -0.5, q_off=np.array([0, tq], np.int32), q_pos0=np.array([n], np.int32),
             cache_off=np.array([0, k], np.int32), clen=clen, loc_off=np.array([0], np.int32), llen=np.array([tq], np.int32),
             loc_pos0=np.array([n], np.int32), cK=cK.cpu(), cV=cV.cpu(), lK=lK, lV=lV, Q=Q, dO=dO, cpos=cpos.cpu().numpy(),
             live_c=np.ones(k, bool), live_l=np.ones(tq, bool))
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    dw = X.cuda()[idx.long()].T @ out["dscore"]
    torch.cuda.synchronize()
    check(p, d, out)
    i = idx.cpu().numpy()
    assert np.array_equal(i, oracle.select(scores.cpu().numpy(), k))
    ref = plain64.attend_backward(_f64(Q), n + np.arange(tq), p["scale"], np.concatenate([_f64(K)[i], _f64(lK)]),
                                  np.concatenate([_f64(V)[i], _f64(lV)]), np.concatenate([i, n + np.arange(tq)]), _f64(d["O"]), _f64(d["lse"]), _f64(dO))
    ref_dw = _f64(X)[i].T @ ref[3][:k]
    assert np.linalg.norm(_f64(dw) - ref_dw) <= 1e-5 * np.linalg.norm(ref_dw) + 1e-6


@pytest.mark.parametrize("dtype,dh,tq", [(BF, 128, 2), (BF, 128, 40), (BF, 64, 7), (F32, 128, 3), (F32, 128, 7), (F32, 64, 20)])
def test_gradient_at_the_least_alignment(dodo, dtype, dh, tq):
    """Every tensor at a multiple of 16 bytes that is not one of 32."""
    def at16(t):
        k = 16 // t.element_size()
        buf = torch.empty(t.numel() + 2 * k, dtype=t.dtype, device="cuda")
        first = k if (buf.data_ptr() + 16) % 32 else 0
        out = buf[first:first + t.numel()].view(t.shape)
        out.copy_(t)
        assert out.data_ptr() % 32 == 16
        return out
    p = problem(("bwdalign", dh, tq), dtype, 3, dh, [tq], [600], [tq + 5])
    d = forward(dodo, p)
    want = backward(dodo, p, d)
    ws = torch.empty(dodo.attend_backward_workspace_bytes(tq, 3, dh, int(p["cache_off"][-1])), dtype=torch.uint8, device="cuda")
    moved = {n: at16(t) for n, t in d.items()}
    got = backward(dodo, p, moved, {n: at16(t) for n, t in buffers(d).items()}, ws=at16(ws))
    torch.cuda.synchronize()
    assert all(torch.equal(got[n].nan_to_num(5.0), want[n].nan_to_num(5.0)) for n in want)


@pytest.mark.parametrize("dtype,tq", [(BF, 2), (BF, 40), (F32, 9)])
def test_gradient_of_rows_behind_two_to_the_31_elements(dodo, dtype, tq):
    """A region that starts behind 2^31 elements of the cache and of the local rows: the same gradients as in small arrays."""
    H, dh, far, n, nl = 64, 128, 263_000, 130, 70
    assert far * H * dh > 2 ** 31
    small = [inputs.randn((r, H, dh), "bwdfar", i, dtype=dtype).cuda() for i, r in enumerate((tq, tq, n, n, nl, nl))]
    Q, dO = small[:2]
    got = []
    for base in (0, far):
        cK, cV, lK, lV = (torch.empty((base + t.shape[0], H, dh), dtype=dtype, device="cuda") for t in small[2:])
        for t, src in zip((cK, cV, lK, lV), small[2:]):
            t[base:] = src
        pos = torch.arange(base + n, dtype=torch.int32, device="cuda") - base
        tables = dict(q_off=[0, 0, tq], q_pos0=[0, n + nl - tq], cache_off=[0, base, base + n], cache_len=[0, n], loc_off=[0, base],
                      loc_len=[0, nl], loc_pos0=[0, n])
        O, lse = torch.empty_like(Q), torch.empty((tq, H), device="cuda")
        ws = torch.empty(dodo.attend_backward_workspace_bytes(tq, H, dh, base + n), dtype=torch.uint8, device="cuda")
        dodo.attend(Q, tables["q_off"], tables["q_pos0"], 0.09, cK, cV, pos, tables["cache_off"], tables["cache_len"], lK, lV, tables["loc_off"],
                    tables["loc_len"], tables["loc_pos0"], O, lse, torch.empty(dodo.attend_workspace_bytes(dh), dtype=torch.uint8, device="cuda"))
        dcK, dcV, dlK, dlV = (torch.empty_like(t) for t in (cK, cV, lK, lV))
        dQ, ds = torch.empty_like(Q), torch.empty(base + n, device="cuda")
        dodo.attend_backward(Q, tables["q_off"], tables["q_pos0"], 0.09, cK, cV, pos, tables["cache_off"], tables["cache_len"], lK, lV,
                             tables["loc_off"], tables["loc_len"], tables["loc_pos0"], O, lse, dO, dQ, dcK, dcV, dlK, dlV, ds, ws)
        torch.cuda.synchronize()
        got.append([dQ] + [t[base:].clone() for t in (dcK, dcV, dlK, dlV, ds)])
        del cK, cV, lK, lV, dcK, dcV, dlK, dlV, ws
    assert all(bool(torch.isfinite(t.float()).all()) for t in got[0])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_backward_binding_refuses_wrong_tensors(dodo):
    p = problem("bwdref", F32, 2, 64, [3], [8], [3], slack=0)
    d = forward(dodo, p)
    out = buffers(d)
    ws = torch.empty(dodo.attend_backward_workspace_bytes(3, 2, 64, 8), dtype=torch.uint8, device="cuda")
    base = dict(Q=d["Q"], q_off=p["q_off"], q_pos0=p["q_pos0"], sm_scale=p["scale"], cacheK=d["cK"], cacheV=d["cV"], cache_pos=d["cpos"],
                cache_off=p["cache_off"], cache_len=p["clen"], locK=d["lK"], locV=d["lV"], loc_off=p["loc_off"], loc_len=p["llen"],
                loc_pos0=p["loc_pos0"], O=d["O"], lse=d["lse"], dO=d["dO"], dQ=out["dQ"], dcacheK=out["dcK"], dcacheV=out["dcV"],
                dlocK=out["dlK"], dlocV=out["dlV"], dscore=out["dscore"], workspace=ws)
    for bad, kind in ((dict(dO=d["dO"].bfloat16()), TypeError), (dict(lse=d["lse"].double()), TypeError), (dict(dQ=out["dQ"][:2]), ValueError),
                      (dict(dcacheV=out["dcV"].cpu()), ValueError), (dict(dscore=out["dscore"][:7]), ValueError), (dict(q_off=[0, 4]), ValueError),
                      (dict(cacheK=d["cK"].transpose(0, 1)), ValueError), (dict(cache_off=[0, 9]), ValueError), (dict(loc_len=[]), ValueError),
                      (dict(dlocK=out["dlK"].bfloat16()), TypeError), (dict(O=d["O"].transpose(1, 2)), ValueError)):
        with pytest.raises(kind):
            dodo.attend_backward(**{**base, **bad})
    with pytest.raises(api.DodoError) as e:
        dodo.attend_backward(**{**base, "workspace": ws[:-16]})
    assert e.value.status == api.ERR_CAPACITY


@pytest.mark.parametrize("dtype,dh,tq", [(F32, 64, 2), (F32, 128, 7), (F32, 128, 20), (BF, 128, 3), (BF, 64, 7), (BF, 64, 70), (BF, 128, 40), (BF, 128, 130)])
def test_gradient_with_positions_at_the_ends_of_their_range(dodo, dtype, dh, tq):
    """cache_pos may hold anything: nuggets at -2^31 (always seen) and 2^31 - 1 (never) among ordinary ones, for queries at positive and
    negative positions and at both ends of what a query may have."""
    q_pos0 = [100, -40, -2 ** 30, 2 ** 30 - tq]
    p = problem(("bwdends", dh, tq), dtype, 2, dh, [tq] * 4, [150] * 4, [tq + 2] * 4)
    p["q_pos0"] = np.asarray(q_pos0, np.int32)
    p["loc_pos0"] = np.asarray([100, -60, -2 ** 30, 2 ** 30 - tq - 2], np.int32)     # some or all of the local tokens are seen
    ends = np.array([-2 ** 31, -2 ** 31 + 1, -2 ** 30 - 1, -2 ** 30, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1], np.int64)
    for b, q0 in enumerate(q_pos0):
        c0 = int(p["cache_off"][b])
        near = np.clip(q0 + np.arange(150) - 50, -2 ** 31, 2 ** 31 - 1)              # before, among and behind the queries
        near[::5] = np.tile(ends, 4)[:30]
        near[64:96] = np.tile(ends, 4)                                               # (all rows of a warp)
        p["cpos"][c0:c0 + 150] = near
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    assert dodo.device_status() == 0
    check(p, d, out, dense=dtype == BF and tq > 4)


@pytest.mark.parametrize("dtype,dh,tq", [(F32, 64, 3), (F32, 128, 20), (BF, 128, 3), (BF, 64, 70), (BF, 128, 40), (BF, 128, 300)])
def test_attend_and_gradient_between_the_ends_of_the_positions(dodo, dtype, dh, tq):
    """The last query at 2^30 - 1 over local tokens from -2^30 on sees them all (positions 2^31 apart, counted), and queries from -2^30
    on none of those that end at 2^30."""
    p = problem(("bwdcorner", dh, tq), dtype, 2, dh, [tq] * 3, [30, 30, 0], [70] * 3)
    p["q_pos0"] = np.asarray([2 ** 30 - tq, -2 ** 30, 2 ** 30 - tq], np.int32)
    p["loc_pos0"] = np.asarray([-2 ** 30, 2 ** 30 - 70, -2 ** 30], np.int32)
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    assert dodo.device_status() == 0
    seen = torch.isfinite(d["lse"]).all(1)
    assert bool(seen[:tq].all()) and not bool(seen[tq:2 * tq].any()) and bool(seen[2 * tq:].all())
    # the forward's log-sum-exp: the error of an fp32 logit, of the exponentials and of the sum of a hundred of them
    Q, lK, cK, lse = _f64(p["Q"]), _f64(p["lK"]), _f64(p["cK"]), _f64(d["lse"])
    for b in (0, 2):
        l = slice(int(p["loc_off"][b]), int(p["loc_off"][b]) + 70)
        c = slice(int(p["cache_off"][b]), int(p["cache_off"][b]) + int(p["clen"][b]))
        q = Q[b * tq:(b + 1) * tq]
        k = np.concatenate([cK[c], lK[l]])
        want = plain64.attend(q, np.zeros(tq), p["scale"], k, k, np.zeros(len(k)))[1]
        assert np.all(np.abs(lse[b * tq:(b + 1) * tq] - want) <= plain64.logit_bound(q, k, p["scale"], dh) + 2.0 ** -20 + 100 * 2.0 ** -24 + 2.0 ** -22 * np.abs(want))
    check(p, d, out, dense=dtype == BF and tq > 4)


@pytest.mark.parametrize("balance", [0, 1, 3])
@pytest.mark.parametrize("tq,nug", [(40, 200), (200, 4000)])
def test_attend_of_blocks_with_anything_in_masked_rows(libdodo, tq, nug, balance):
    """The forward that a gradient starts from, on the tensor cores: keys that some queries of a block do not see hold NaN and
    infinities, in the first tile and in later ones, in every way of spreading the work."""
    dodo = api.Dodo(0)
    dodo.set_tuning(api.TUNE_DENSE_BALANCE, balance)
    p = problem(("bwdblockany", tq), BF, 2, 128, [tq, 32], [nug, 64], [tq + 2, 32], slack=0)
    half = int(p["q_pos0"][0]) + tq // 2
    p["cpos"][[0, 63, 100]] = half
    p["cpos"][[1, nug - 1]] = 10 ** 6
    clean = forward(dodo, p)
    torch.cuda.synchronize()
    q = dict(p, **{n: p[n].clone() for n in ("cK", "cV", "lK", "lV")})
    for n in ("cK", "cV"):
        q[n][[1, nug - 1]] = float("nan")
    q["cV"][0, 1, 3], q["cV"][63, 0, 64], q["cV"][100, 1, 127], q["lV"][tq + 1, 0, 0] = float("nan"), float("inf"), -float("inf"), float("nan")
    out = forward(dodo, q)
    again = forward(dodo, q)
    torch.cuda.synchronize()
    fixed = lambda t: t.nan_to_num(7.0, 1e30, -1e30)  # noqa: E731
    assert torch.equal(out["lse"], clean["lse"]) and torch.equal(fixed(out["O"]), fixed(again["O"]))
    assert torch.equal(out["O"][tq:], clean["O"][tq:])
    Q, K, V = _f64(p["Q"][:tq]), np.concatenate([_f64(q["cK"][:nug]), _f64(q["lK"][:tq + 2])]), np.concatenate([_f64(q["cV"][:nug]), _f64(q["lV"][:tq + 2])])
    kpos, qpos = np.concatenate([p["cpos"][:nug], p["loc_pos0"][0] + np.arange(tq + 2)]), p["q_pos0"][0] + np.arange(tq)
    want, got = plain64.attend(Q, qpos, p["scale"], K, V, kpos)[0], _f64(out["O"][:tq])
    # a weight's error: its logit's, its rounding to bf16 (2^-8), the exponential's and the sum's; the result is rounded once
    keys = np.concatenate([_f64(p["cK"][:nug]), _f64(p["lK"][:tq + 2])])
    w = 2.0 * plain64.logit_bound(Q, keys, p["scale"], 128) + 2.0 ** -8 + 2.0 ** -20 + len(K) * 2.0 ** -24
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert np.all(np.abs(got[fine] - want[fine]) <= 2.0 ** -8 * np.abs(want[fine]) + w * np.max(np.abs(V[np.isfinite(V)])))
    assert fine[:tq // 2].all() and not fine[tq // 2:, 1, 3].any() and not fine[tq // 2:, 0, 64].any() and not fine[tq - 1, 0, 0]
    assert dodo.device_status() == 0
    dodo.close()


@pytest.mark.parametrize("dtype,dh,tq,nug", [(F32, 64, 1, 40), (F32, 128, 3, 5000), (BF, 128, 1, 300), (BF, 128, 1, 6000), (BF, 64, 5, 70), (BF, 128, 40, 90), (BF, 128, 260, 6000)])
def test_a_key_that_is_no_number_shows(dodo, dtype, dh, tq, nug):
    """A visible key that holds a NaN: its head's output and log-sum-exp are NaN, not the 0 and -inf of a query that sees nothing, and
    so is the query's gradient; other heads and sequences keep their bits."""
    p = problem(("bwdnankey", dh, tq, nug), dtype, 2, dh, [tq, 2], [nug, 20], [tq + 1, 2], slack=0)
    clean = forward(dodo, p)
    q = dict(p, cK=p["cK"].clone())
    q["cK"][nug // 2, 1, 5] = float("nan")
    d = forward(dodo, q)
    out = backward(dodo, q, d)
    torch.cuda.synchronize()
    assert bool(torch.isnan(d["O"][:tq, 1]).all()) and bool(torch.isnan(d["lse"][:tq, 1]).all())
    assert torch.equal(d["O"][:tq, 0], clean["O"][:tq, 0]) and torch.equal(d["lse"][:tq, 0], clean["lse"][:tq, 0])
    assert torch.equal(d["O"][tq:], clean["O"][tq:]) and torch.equal(d["lse"][tq:], clean["lse"][tq:])
    assert bool(torch.isnan(out["dQ"][:tq, 1]).all()) and bool(torch.isfinite(out["dQ"][:tq, 0]).all()) and bool(torch.isfinite(out["dQ"][tq:]).all())
    assert dodo.device_status() == 0


@pytest.mark.parametrize("power", [20, 60])
def test_gradient_of_a_block_with_a_tiny_scale(dodo, power):
    p = problem(("bwdtiny", power), BF, 2, 128, [70, 40], [300, 60], [10, 40], inside=True)
    p["q_pos0"][1] = -5                                           # the first queries see nothing
    p["Q"], p["scale"] = (p["Q"].float() * 2.0 ** power).to(BF), p["scale"] * 2.0 ** -power
    d = forward(dodo, p)
    out = backward(dodo, p, d)
    torch.cuda.synchronize()
    lse = _f64(d["lse"])
    for b in range(2):
        q = slice(int(p["q_off"][b]), int(p["q_off"][b + 1]))
        c = slice(int(p["cache_off"][b]), int(p["cache_off"][b]) + int(p["clen"][b]))
        l = slice(int(p["loc_off"][b]), int(p["loc_off"][b]) + int(p["llen"][b]))
        k, v = np.concatenate([_f64(p["cK"])[c], _f64(p["lK"])[l]]), np.concatenate([_f64(p["cV"])[c], _f64(p["lV"])[l]])
        kpos = np.concatenate([p["cpos"][c], p["loc_pos0"][b] + np.arange(p["llen"][b])])
        O, want = plain64.attend(_f64(p["Q"])[q], p["q_pos0"][b] + np.arange(q.stop - q.start), p["scale"], k, v, kpos)
        seen = np.isfinite(want)
        assert np.array_equal(np.isneginf(lse[q]), ~seen)
        e = plain64.logit_bound(_f64(p["Q"])[q], k, p["scale"], 128) + 2.0 ** -20 + len(k) * 2.0 ** -24
        assert np.all(np.abs(lse[q][seen] - want[seen]) <= e + 2.0 ** -22 * np.abs(want[seen]))
        assert np.all(np.abs(_f64(d["O"])[q] - O) <= 2.0 ** -8 * np.abs(O) + (2 * e + 2.0 ** -8) * np.max(np.abs(v)))
    check(p, d, out, dense=True)


def test_two_contexts_on_two_streams(libdodo):
    """Gradients and 4-bit appends, expansions and attends of two contexts at once, each on its own stream with its own buffers: the
    bits of one after the other."""
    H, dh = 4, 128
    rs = np.random.RandomState(6)

    def job(i, ctx):
        p = problem(("bwdtwo", i), BF, H, dh, [100 + 30 * i, 3], [700, 90], [130, 40])
        few = problem(("bwdtwofew", i), F32, 2, 64, [20, 2], [300, 9], [22, 2])
        K, V = (inputs.randn((600, H, dh), "bwdtwo", i, k, dtype=BF).cuda() for k in "KV")
        Q = inputs.randn((40, H, dh), "bwdtwo", i, "Q", dtype=BF).cuda()
        idx = _cuda(np.sort(rs.permutation(600)[:200]).astype(np.int32))
        d, df = forward(ctx, p), forward(ctx, few)
        n, nf = (ctx.attend_backward_workspace_bytes(int(x["q_off"][-1]), x["H"], x["dh"], int(x["cache_off"][-1])) for x in (p, few))
        w, wf, w4 = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in (n, nf, ctx.attend_q4_workspace_bytes(H, dh, 200)))
        torch.cuda.synchronize()

        def run():
            q4, sc = torch.zeros((200, H, 2, dh // 2), dtype=torch.uint8, device="cuda"), torch.zeros((200, H, 2, dh // 32), dtype=torch.int32, device="cuda")
            pos, clen, outs = torch.zeros(200, dtype=torch.int32, device="cuda"), np.zeros(1, np.int32), []
            for _ in range(4):
                outs += list(backward(ctx, p, d, ws=w).values()) + list(backward(ctx, few, df, ws=wf).values())
                clen[:] = 0
                ctx.gather_kv_q4(K, V, [0, 600], idx, [0, 200], [0], q4, sc, pos, [0, 200], clen)
                for t in (1, 5, 40):
                    O = torch.empty((t, H, dh), dtype=BF, device="cuda")
                    ctx.attend_q4(Q[:t].contiguous(), [0, t], [600], dh ** -0.5, q4, sc, pos, [0, 200], clen, K, V, [500], [100], [550], O, None, w4)
                    outs.append(O)
            return outs + [q4, sc, pos]
        return run

    ctxs, streams = [api.Dodo(0), api.Dodo(0)], [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = [job(i, c) for i, c in enumerate(ctxs)]
    alone = []
    for run in jobs:
        alone.append(run())
        torch.cuda.synchronize()
    together = []
    for run, s in zip(jobs, streams):
        with torch.cuda.stream(s):
            together.append(run())
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert len(a) == len(b) and all(torch.equal(x.float().nan_to_num(5.0), y.float().nan_to_num(5.0)) for x, y in zip(a, b))
    for c in ctxs:
        assert c.device_status() == 0
        c.close()
