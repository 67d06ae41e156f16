"""Calls of the paged cache's and the rotation's entry points that a program may make and that are off the usual path: workspaces between none and
all that can be used, many query heads on one KV head, four arrays in one rotation, one position for many sequences."""
import struct

import numpy as np
import pytest
import torch

from paper_2310_02409_b200 import api, inputs
from test_gpu_paged import BF, F32, _batch, _check, _cuda
from test_gpu_paged_choice import tensor_cores
from test_gpu_rope import LAYOUT, _close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,Hkv,tq,B", [(BF, 8, 2, 1, 2), (BF, 4, 4, 16, 2), (BF, 4, 2, 70, 2), (F32, 4, 2, 1, 2), (F32, 4, 2, 12, 2), (F32, 16, 8, 40, 20)])
@pytest.mark.parametrize("mode", [0, 1])
def test_workspaces_of_any_size(dodo, dtype, H, Hkv, tq, B, mode):
    """Fewer bytes than are asked for: other cuts and other kernels, the same results; what lies behind the bytes that are given stays."""
    s = _batch(dtype, H, Hkv, 128, [tq] * B, [1500] + [300] * (B - 1), [tq] * B, 16)
    shape = (s["pages"], s["page"], Hkv, 128)
    cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
    Q, lK, lV = s["Q"].cuda(), s["lK"].cuda(), s["lV"].cuda()
    whole = dodo.attend_paged_workspace_bytes(128)
    held = torch.empty(whole + 4096, dtype=torch.uint8, device="cuda")
    for n in (0, 4096, 5 << 20, 20 << 20, whole - 16, whole):
        held.fill_(0xff)
        O, L = torch.full(Q.shape, 7.0, dtype=dtype, device="cuda"), torch.full(Q.shape[:2], 7.0, device="cuda")
        with tensor_cores(dodo, mode):
            dodo.attend_paged(Q, s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], lK, lV, s["loc_off"][:-1], s["loc"], s["loc_pos0"], O, L, held[:n])
        torch.cuda.synchronize()
        assert (held[n:] == 0xff).all()
        _check(s, O, L, only=[0])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,tq", [(64, 1, 1), (71, 1, 1), (128, 1, 2), (96, 3, 3), (142, 2, 5), (3, 1, 300)])
@pytest.mark.parametrize("page,mode", [(16, 0), (16, 1), (3, 0)])
def test_many_query_heads_on_a_kv_head(dodo, dtype, H, Hkv, tq, page, mode):
    s = _batch(dtype, H, Hkv, 64, [tq, 1], [200, 90], [tq + 5, 0], page, seed=H)
    s["q_pos0"][1] = 500
    shape = (s["pages"], s["page"], Hkv, 64)
    cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
    O, L = torch.full(s["Q"].shape, 7.0, dtype=dtype, device="cuda"), torch.full(s["Q"].shape[:2], 7.0, device="cuda")
    ws = torch.empty(dodo.attend_paged_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    with tensor_cores(dodo, mode):
        dodo.attend_paged(s["Q"].cuda(), s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], s["lK"].cuda(), s["lV"].cuda(), s["loc_off"][:-1],
                          s["loc"], s["loc_pos0"], O, L, ws)
    torch.cuda.synchronize()
    _check(s, O, L)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows", [3, 3000])
def test_four_arrays_in_one_rotation(dodo, layout, rows):
    """One of no heads among them, one in place, one with its heads far apart."""
    heads, dh = (5, 0, 2, 9), 64
    freq = api.rope_frequencies(48)
    rope = api.Rope(freq, LAYOUT[layout], 0.5)
    X = [inputs.randn((rows, max(h, 1), dh), "rope four", h, dtype=BF).cuda() for h in heads]
    Y = [torch.full_like(x, 7.0) for x in X]
    Y[2] = X[2].clone()
    wide = torch.full((9, rows, dh), 7.0, dtype=BF, device="cuda")
    Y[3] = wide.transpose(0, 1)
    packed = b"".join(struct.pack("QQiiqqqq", (y if i == 2 else x).data_ptr(), y.data_ptr(), h, 0, x.stride(0), x.stride(1), y.stride(0), y.stride(1))
                      for i, (x, y, h) in enumerate(zip(X, Y, heads)))
    off, pos = np.array([0, rows], np.int32), np.array([1000], np.int32)
    assert dodo._lib.dodo_rope(dodo._ctx, rope._spec, packed, 4, api.BF16, dh, off.ctypes.data, pos.ctypes.data, 1, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for x, y, h in zip(X, Y, heads):
        if h:
            _close(y, x, 1000 + np.arange(rows), freq, layout, 0.5, BF)
    assert (Y[1] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_same_token_and_the_same_page_twice(dodo, dtype):
    """An index that is there twice is appended twice; a page that is there twice in a table is seen twice."""
    H, dh, page = 2, 64, 8
    K, V = (inputs.randn((10, H, dh), "twice", n, dtype=dtype).cuda() for n in "KV")
    cK, cV = (torch.zeros((4, page, H, dh), dtype=dtype, device="cuda") for _ in range(2))
    pos = torch.zeros((4, page), dtype=torch.int32, device="cuda")
    cache, clen = api.PagedCache(cK, cV, pos, torch.tensor([2, 2], dtype=torch.int32, device="cuda")), np.zeros(1, np.int32)
    idx = torch.tensor([3, 3, 9, 0, 0, 0, 9, 1], dtype=torch.int32, device="cuda")
    dodo.gather_kv_paged(K, V, [0, 10], idx, [0, 8], [5], None, cache, [0, 2], clen)
    torch.cuda.synchronize()
    assert torch.equal(cK[2], K[idx.long()]) and torch.equal(cV[2], V[idx.long()]) and torch.equal(pos[2], idx + 5) and clen[0] == 8
    Q = inputs.randn((1, H, dh), "twice", "Q", dtype=dtype).cuda()
    out = []
    for n in (8, 16):
        O, L = torch.empty_like(Q), torch.empty((1, H), device="cuda")
        dodo.attend_paged(Q, [0, 1], [100], 0.125, cache, [0, 2], [n], None, None, None, None, None, O, L, None)
        out.append((O.float(), L))
    torch.cuda.synchronize()
    # Twice the same keys: the same result, a sum twice as large.  On either side O has half a step of its type, in bf16 2^-16 of every weight, and sums
    # of 16 terms; the log-sum-exp 2^-21 of the exponentials, 2^-19 of their sum and a rounding.
    half, weights = (2.0 ** -8, 2.0 ** -16) if dtype is BF else (2.0 ** -24, 0.0)
    assert ((out[0][0] - out[1][0]).abs() <= 2 * half * out[0][0].abs() + 2 * (weights + 32 * 2.0 ** -23) * V.float().abs().max()).all()
    assert ((out[1][1] - out[0][1]) - np.log(2.0)).abs().max() <= 2.0 ** -17 * (1.0 + float(out[1][1].abs().max()))
