"""Argument checks of the 4-bit cache's entry points, on the host: every call is refused before anything is launched, so the
context needs no device and the pointers are never followed."""
import ctypes

import numpy as np
import pytest

P = 0x10000     # a 16-byte aligned address that nothing reads
BAD, UNSUP, CAP = -1, -2, -3


@pytest.fixture(scope="module")
def ctx(libdodo):
    import torch
    from paper_2310_02409_b200 import api
    lib = api.load()
    c = ctypes.c_void_p()
    rc = lib.dodo_create(ctypes.byref(c), 0)
    assert c.value and (rc == api.OK) == torch.cuda.is_available()
    yield lib, c
    lib.dodo_destroy(c)


def _i32(*v):
    return np.asarray(v, np.int32)


def _call(ctx, name, **args):
    lib, c = ctx
    vals = [v.ctypes.data if isinstance(v, np.ndarray) else v for v in args.values()]
    return getattr(lib, name)(c, *vals)


def _gather(**k):
    return {**dict(K=P, V=P, dtype=1, H=2, dh=64, seq_off=_i32(0, 4, 9), idx=P, nug_off=_i32(0, 1, 3), pos_base=_i32(0, 0), B=2, q4=P,
                   scale=P, pos=P, cache_off=_i32(0, 2, 4), cache_len=_i32(0, 0), stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(dtype=2), UNSUP), (dict(dh=32), UNSUP), (dict(dh=96), UNSUP), (dict(H=0), BAD), (dict(K=None), BAD), (dict(V=P + 8), BAD),
    (dict(idx=None), BAD), (dict(q4=None), BAD), (dict(q4=P + 4), BAD), (dict(scale=None), BAD), (dict(scale=P + 4), BAD), (dict(pos=None), BAD),
    (dict(seq_off=_i32(0, 4, 3)), BAD), (dict(seq_off=_i32(1, 4, 9)), BAD), (dict(nug_off=_i32(0, 5, 6)), BAD), (dict(pos_base=None), BAD),
    (dict(cache_len=None), BAD), (dict(cache_len=_i32(-1, 0)), BAD), (dict(cache_len=_i32(2, 0)), CAP), (dict(cache_off=_i32(0, 2, 3)), CAP),
    (dict(cache_off=None), BAD),
])
def test_gather_q4_refuses(ctx, change, status):
    args = _gather(**change)
    before = args["cache_len"].copy() if args["cache_len"] is not None else None
    assert _call(ctx, "dodo_gather_kv_q4", **args) == status
    if before is not None:
        assert np.array_equal(args["cache_len"], before)
    assert len(ctx[0].dodo_last_error(ctx[1])) > 0


def _expand(**k):
    return {**dict(q4=P, scale=P, H=2, dh=64, cache_off=_i32(0, 2, 4), cache_len=_i32(1, 2), B=2, dtype=1, K=P, V=P, stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(dtype=3), UNSUP), (dict(dh=80), UNSUP), (dict(H=-2), BAD), (dict(q4=None), BAD), (dict(scale=P + 2), BAD), (dict(K=None), BAD),
    (dict(V=P + 8), BAD), (dict(cache_off=None), BAD), (dict(cache_len=None), BAD), (dict(cache_len=_i32(3, 0)), BAD), (dict(cache_len=_i32(0, -1)), BAD),
])
def test_expand_q4_refuses(ctx, change, status):
    assert _call(ctx, "dodo_expand_kv_q4", **_expand(**change)) == status


def test_expand_q4_of_an_empty_cache_is_nothing(ctx):
    assert _call(ctx, "dodo_expand_kv_q4", **_expand(cache_len=_i32(0, 0), q4=None, K=None)) == 0


def _attend(**k):
    return {**dict(Q=P, q_off=_i32(0, 1, 2), q_pos0=_i32(9, 9), dtype=1, H=2, dh=64, sm_scale=0.125, q4=P, scale=P, pos=P,
                   cache_off=_i32(0, 2, 4), cache_len=_i32(1, 2), locK=P, locV=P, loc_off=_i32(0, 3), loc_len=_i32(3, 1), loc_pos0=_i32(0, 0),
                   loc_rows=4, B=2, O=P, lse=None, workspace=None, workspace_bytes=0, stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(dtype=7), UNSUP), (dict(dh=256), UNSUP), (dict(H=0), BAD), (dict(Q=None), BAD), (dict(O=P + 8), BAD), (dict(q_pos0=None), BAD),
    (dict(q_off=_i32(0, 2, 1)), BAD), (dict(q4=None), BAD), (dict(scale=None), BAD), (dict(pos=None), BAD), (dict(cache_len=_i32(3, 0)), BAD),
    (dict(cache_off=None), BAD), (dict(loc_len=_i32(-1, 0)), BAD), (dict(loc_len=_i32(3, 2)), BAD), (dict(loc_off=None), BAD), (dict(loc_pos0=None), BAD),
    (dict(locK=None), BAD), (dict(locV=P + 8), BAD),
])
def test_attend_q4_refuses(ctx, change, status):
    assert _call(ctx, "dodo_attend_q4", **_attend(**change)) == status


def test_attend_q4_without_queries_is_nothing(ctx):
    assert _call(ctx, "dodo_attend_q4", **_attend(q_off=_i32(0, 0, 0), Q=None)) == 0


def test_attend_q4_workspace_grows_with_the_cache(ctx):
    lib, c = ctx
    a, b = (lib.dodo_attend_q4_workspace_bytes(c, 2, 128, rows) for rows in (0, 100))
    assert b - a == 2 * 100 * 2 * 128 * 2
    assert lib.dodo_attend_q4_workspace_bytes(c, 0, 128, 1) == 0 and lib.dodo_attend_q4_workspace_bytes(c, 2, 128, -1) == 0


def _backward(**k):
    return {**dict(Q=P, q_off=_i32(0, 1, 2), q_pos0=_i32(9, 9), dtype=1, H=2, dh=64, sm_scale=0.125, cacheK=P, cacheV=P, pos=P,
                   cache_off=_i32(0, 2, 4), cache_len=_i32(1, 2), locK=P, locV=P, loc_off=_i32(0, 3), loc_len=_i32(3, 1), loc_pos0=_i32(0, 0),
                   loc_rows=4, B=2, O=P, lse=P, dO=P, dQ=P, dcacheK=P, dcacheV=P, dlocK=P, dlocV=P, dscore=P, workspace=P,
                   workspace_bytes=1 << 16, stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(dtype=7), UNSUP), (dict(dh=96), UNSUP), (dict(H=0), BAD), (dict(Q=None), BAD), (dict(O=None), BAD), (dict(lse=None), BAD),
    (dict(dO=P + 8), BAD), (dict(dQ=None), BAD), (dict(q_pos0=None), BAD), (dict(q_off=_i32(0, 2, 1)), BAD), (dict(cacheK=None), BAD),
    (dict(cacheV=P + 4), BAD), (dict(pos=None), BAD), (dict(dcacheK=None), BAD), (dict(dcacheV=P + 8), BAD), (dict(cache_len=_i32(3, 0)), BAD),
    (dict(cache_off=None), BAD), (dict(loc_len=_i32(-1, 0)), BAD), (dict(loc_off=None), BAD), (dict(dlocK=None), BAD), (dict(dlocV=P + 8), BAD),
    (dict(loc_off=_i32(0, 2)), BAD), (dict(loc_off=_i32(1, 0), loc_len=_i32(2, 2)), BAD),       # windows that share a row
    (dict(workspace=None), CAP), (dict(workspace=P + 8), CAP), (dict(workspace_bytes=64), CAP),
])
def test_attend_backward_refuses(ctx, change, status):
    assert _call(ctx, "dodo_attend_backward", **_backward(**change)) == status


def test_attend_backward_of_nothing_is_nothing(ctx):
    nothing = dict(q_off=_i32(0, 0, 0), cache_len=None, loc_len=None, Q=None, O=None, lse=None, dO=None, dQ=None, workspace=None)
    assert _call(ctx, "dodo_attend_backward", **_backward(**nothing)) == 0
    assert _call(ctx, "dodo_attend_backward", **_backward(B=0, q_off=_i32(0), q_pos0=None, cache_len=None, loc_len=None)) == 0


@pytest.mark.parametrize("change", [dict(q_pos0=_i32(9, 2 ** 30)), dict(q_pos0=_i32(-2 ** 30 - 1, 0)), dict(q_pos0=_i32(2 ** 31 - 1, 0)),
                                    dict(loc_pos0=_i32(2 ** 30 - 2, 0)), dict(loc_pos0=_i32(0, -2 ** 31))])
@pytest.mark.parametrize("name", ["dodo_attend_q4", "dodo_attend_backward"])
def test_positions_leave_room(ctx, name, change):
    assert _call(ctx, name, **(_attend if name == "dodo_attend_q4" else _backward)(**change)) == BAD
