"""Attention over the paged nugget cache: the caller's choice of the kernel, and of what a weight is rounded to with it."""
import contextlib

import pytest
import torch

import launched
import plain64
from paper_2310_02409_b200 import api
from test_gpu_paged import BF, F32, _batch, _check, _cuda
from test_gpu_paged_weights import TWO_PIECES, _cancelling, _holds

pytestmark = pytest.mark.gpu
TENSOR_CORES, FEW, FMA, TILE = "attend_paged_dense_kernel", "attend_paged_token_kernel", "attend_paged_rows_kernel", "attend_paged_tile_kernel"


@contextlib.contextmanager
def tensor_cores(dodo, mode):
    """0: by the work; 1: wherever they can; 2: never."""
    dodo.set_tuning(api.TUNE_PAGED_DENSE, mode)
    try:
        yield
    finally:
        dodo.set_tuning(api.TUNE_PAGED_DENSE, 0)


def prepared(dodo, s, workspace=True):
    """The call on a batch of test_gpu_paged, ready to be repeated or captured, and its outputs."""
    shape = (s["pages"], s["page"], s["Hkv"], s["dh"])
    cache = api.PagedCache(s["cK"].view(shape).cuda(), s["cV"].view(shape).cuda(), _cuda(s["pos"], torch.int32), _cuda(s["table"]))
    Q, lK, lV = s["Q"].cuda(), s["lK"].cuda(), s["lV"].cuda()
    O, L = torch.full(Q.shape, 7.0, dtype=s["dtype"], device="cuda"), torch.full(Q.shape[:2], 7.0, device="cuda")
    ws = torch.full((dodo.attend_paged_workspace_bytes(s["dh"]),), 0xff, dtype=torch.uint8, device="cuda") if workspace else None
    call = lambda: dodo.attend_paged(Q, s["q_off"], s["q_pos0"], s["scale"], cache, s["page_off"], s["nug"], lK, lV, s["loc_off"][:-1], s["loc"],  # noqa: E731
                                     s["loc_pos0"], O, L, ws)
    return call, O, L


def run_on(dodo, s, kernel, workspace=True):
    """Outputs of the call, which has to take this kernel and no other."""
    call, O, L = prepared(dodo, s, workspace)
    call()
    torch.cuda.synchronize()
    names = launched.kernels(call)
    assert names and all(kernel in n for n in names), names
    return O, L


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (4, 2, 40), (2, 2, 150)])
@pytest.mark.parametrize("page", [16, 5])
def test_the_choice_is_the_callers(dodo, dh, H, Hkv, tq, page):
    s = _cancelling(H, Hkv, dh, tq, 205, 84, page)
    with tensor_cores(dodo, 2):
        _holds(s, *run_on(dodo, s, FEW if page == 16 else FMA), TWO_PIECES)
    with tensor_cores(dodo, 1):
        O, L = run_on(dodo, s, TENSOR_CORES)
        _check(s, O, L)
        run_on(dodo, s, FEW if page == 16 else FMA, workspace=False)
    s["scale"] = -1.0
    with tensor_cores(dodo, 1):
        run_on(dodo, s, FEW if page == 16 else FMA)


def test_the_choice_by_the_work(dodo):
    run_on(dodo, _batch(BF, 8, 2, 128, [4], [300], [4], 16), FEW)
    run_on(dodo, _batch(BF, 8, 2, 128, [30], [300], [30], 16), FEW)
    run_on(dodo, _batch(BF, 32, 8, 128, [256] * 4, [700] * 4, [256] * 4, 16), TENSOR_CORES)
    run_on(dodo, _batch(F32, 8, 2, 128, [30], [300], [30], 16), FMA)
    run_on(dodo, _batch(F32, 32, 8, 128, [64] * 4, [700] * 4, [64] * 4, 16), TILE)
    assert plain64.HALF["bf16"] > TWO_PIECES
