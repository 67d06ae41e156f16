"""Argument checks of the rotary positions' and the paged cache's entry points, on the host: every call is refused before anything is
launched, so the context needs no device and the pointers are never followed."""
import ctypes
import struct

import numpy as np
import pytest
import torch

P = 0x10000     # a 16-byte aligned address that nothing reads
BAD, UNSUP, CAP = -1, -2, -3


@pytest.fixture(scope="module")
def ctx(libdodo):
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


def _spec(rot=64, layout=0):
    from paper_2310_02409_b200 import api
    return api.Rope(np.ones(rot // 2), layout)._spec


def _array(p=P, out=P, heads=2, strides=(128, 64, 128, 64)):
    return struct.pack("QQiiqqqq", p or 0, out or 0, heads, 0, *strides)


def _rope(**k):
    return {**dict(rope=_spec(), arrays=_array(), n=1, dtype=1, dh=64, row_off=_i32(0, 2, 5), pos0=_i32(0, 9), B=2, stream=None), **k}


@pytest.mark.parametrize("name", ["dodo_rope", "dodo_rope_backward"])
@pytest.mark.parametrize("change,status", [
    (dict(rope=None), BAD), (dict(rope=bytes(1040)), BAD), (dict(arrays=None), BAD), (dict(n=-1), BAD), (dict(n=5), BAD), (dict(dtype=2), UNSUP),
    (dict(dh=62), BAD), (dict(dh=65), UNSUP), (dict(dh=0), UNSUP), (dict(dh=514), UNSUP), (dict(row_off=None), BAD), (dict(row_off=_i32(0, 3, 2)), BAD),
    (dict(row_off=_i32(1, 2, 3)), BAD), (dict(pos0=None), BAD), (dict(pos0=_i32(0, 2 ** 31 - 2)), BAD), (dict(B=-1), BAD), (dict(arrays=_array(0)), BAD),
    (dict(arrays=_array(P, 0)), BAD), (dict(arrays=_array(P + 1)), BAD), (dict(arrays=_array(P, P + 2), dtype=0), BAD), (dict(arrays=_array(heads=-1)), BAD),
])
def test_rope_refuses(ctx, name, change, status):
    assert _call(ctx, name, **_rope(**change)) == status
    assert len(ctx[0].dodo_last_error(ctx[1])) > 0


@pytest.mark.parametrize("change", [dict(n=0, arrays=None), dict(B=0, row_off=_i32(0), pos0=None), dict(row_off=_i32(0, 0, 0), arrays=_array(0, 0)),
                                    dict(arrays=_array(0, 0, 0))])
def test_rope_of_nothing_is_nothing(ctx, change):
    assert _call(ctx, "dodo_rope", **_rope(**change)) == 0


def test_rope_frequencies_and_specs(libdodo):
    from paper_2310_02409_b200 import api
    i = np.arange(32)
    f = 10000.0 ** (-i / 32.0)
    near = lambda a, b: np.allclose(a, b, rtol=1e-14, atol=0)  # noqa: E731
    assert near(api.rope_frequencies(64), f)
    assert near(api.rope_frequencies(64, 10000.0, api.ROPE_LINEAR, 4.0), f / 4)
    g = api.rope_frequencies(64, 10000.0, api.ROPE_BASE, 4.0)
    assert g[0] == 1.0 and near(g[-1], f[-1] / 4) and (np.diff(g / f) < 0).all()
    g = api.rope_frequencies(64, 10000.0, api.ROPE_PARTS, 4.0, 2048, 1.0, 32.0)
    turns = 2048 * f / (2 * np.pi)
    assert near(g[turns >= 32], f[turns >= 32]) and near(g[turns <= 1], f[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 4).all()
    assert near(api.rope_frequencies(2, 10000.0, api.ROPE_BASE, 4.0), [1.0])
    for bad in (dict(rot=0), dict(rot=63), dict(rot=258), dict(rot=-2), dict(base=0.0), dict(base=float("inf")), dict(scaling=4), dict(scaling=-1),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=float("nan")), dict(scaling=3, trained=0), dict(scaling=3, trained=5, low=2.0, high=2.0)):
        with pytest.raises(api.DodoError):
            api.rope_frequencies(**{**dict(rot=64), **bad})
    for freq, layout, scale in ((np.zeros(0), 0, 1.0), (np.zeros(129), 0, 1.0), ([np.nan], 0, 1.0), ([np.inf], 1, 1.0), ([1.0], 2, 1.0), ([1.0], 0, np.inf)):
        with pytest.raises(api.DodoError):
            api.Rope(freq, layout, scale)
    with pytest.raises(ValueError):
        api.Rope(np.ones((2, 2)))


def test_rope_turns_are_fractions_of_a_turn(libdodo):
    """64 bits of freq / (2 pi) modulo 1: exact to the 53 bits that a double frequency gives at least."""
    from fractions import Fraction

    from paper_2310_02409_b200 import api
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)
    freq = [1.0, 1e-4, 0.7, 3.0, -0.7, 0.0, 1e-9, 6.283185307179586, 1234.5]
    turn = struct.unpack_from("<9Q", api.Rope(freq)._spec.raw, 16)
    for f, t in zip(freq, turn):
        exact = Fraction(f) / (2 * pi)
        off = abs((exact - exact.__floor__()) - Fraction(t, 2 ** 64))
        assert min(off, 1 - off) <= Fraction(1, 2 ** 64) * (2 + int(abs(f)))


def _cache(K=P, V=P, pos=P, table=P, dtype=1, H=2, dh=64, pages=6, page=2):
    return struct.pack("QQQQiiiiii", K or 0, V or 0, pos or 0, table or 0, dtype, H, dh, pages, page, 0)


def _gather(**k):
    return {**dict(K=P, V=P, kv_row=128, seq_off=_i32(0, 4, 9), idx=P, nug_off=_i32(0, 1, 3), pos_base=_i32(0, 0), B=2, rope=_spec(), cache=_cache(),
                   page_off=_i32(0, 1, 2), cache_len=_i32(0, 0), stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(cache=None), BAD), (dict(cache=_cache(dtype=2)), UNSUP), (dict(cache=_cache(dh=62)), BAD), (dict(cache=_cache(dh=63)), UNSUP),
    (dict(cache=_cache(dh=514), rope=None), UNSUP), (dict(cache=_cache(H=0)), BAD), (dict(cache=_cache(page=0)), BAD), (dict(cache=_cache(pages=-1)), BAD),
    (dict(cache=_cache(pages=2 ** 30, page=2)), BAD), (dict(cache=_cache(K=None)), BAD), (dict(cache=_cache(V=P + 8)), BAD), (dict(cache=_cache(pos=None)), BAD),
    (dict(cache=_cache(table=None)), BAD), (dict(cache=_cache(H=1, dh=66), rope=None), BAD), (dict(K=None), BAD), (dict(V=P + 8), BAD), (dict(kv_row=132), BAD),
    (dict(seq_off=_i32(0, 4, 3)), BAD), (dict(seq_off=None), BAD), (dict(nug_off=_i32(0, 5, 6)), BAD), (dict(nug_off=None), BAD), (dict(pos_base=None), BAD),
    (dict(pos_base=_i32(0, 2 ** 31 - 4)), BAD), (dict(page_off=None), BAD), (dict(page_off=_i32(0, 2, 1)), BAD), (dict(cache_len=None), BAD),
    (dict(cache_len=_i32(-1, 0)), BAD), (dict(cache_len=_i32(3, 0)), BAD), (dict(cache_len=_i32(2, 0)), CAP), (dict(cache_len=_i32(0, 1)), CAP),
    (dict(idx=None), CAP), (dict(rope=bytes(1040)), BAD), (dict(rope=_spec(66)), BAD),
])
def test_gather_paged_refuses(ctx, change, status):
    args = _gather(**change)
    before = args["cache_len"].copy() if args["cache_len"] is not None else None
    assert _call(ctx, "dodo_gather_kv_paged", **args) == status
    if before is not None:
        assert np.array_equal(args["cache_len"], before)
    assert len(ctx[0].dodo_last_error(ctx[1])) > 0


def test_gather_paged_of_nothing_is_nothing(ctx):
    assert _call(ctx, "dodo_gather_kv_paged", **_gather(nug_off=_i32(0, 0, 0), K=None, cache=_cache(None, None, None, None))) == 0
    assert _call(ctx, "dodo_gather_kv_paged", **_gather(seq_off=_i32(0, 0, 0), idx=None, K=None, cache=_cache(None, None, None, None))) == 0


def _attend(**k):
    return {**dict(Q=P, q_off=_i32(0, 1, 2), q_pos0=_i32(9, 9), H=4, sm_scale=0.125, cache=_cache(), page_off=_i32(0, 1, 2), cache_len=_i32(1, 2),
                   locK=P, locV=P, loc_off=_i32(0, 3), loc_len=_i32(3, 1), loc_pos0=_i32(0, 0), loc_rows=4, B=2, O=P, lse=None, workspace=None,
                   workspace_bytes=0, stream=None), **k}


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), BAD), (dict(cache=None), BAD), (dict(cache=_cache(dtype=7)), UNSUP), (dict(cache=_cache(dh=96)), UNSUP), (dict(H=0), BAD), (dict(H=3), BAD),
    (dict(H=1), BAD), (dict(cache=_cache(H=0)), BAD), (dict(Q=None), BAD), (dict(O=P + 8), BAD), (dict(q_pos0=None), BAD), (dict(q_off=_i32(0, 2, 1)), BAD),
    (dict(q_off=None), BAD), (dict(cache=_cache(K=None)), BAD), (dict(cache=_cache(V=P + 4)), BAD), (dict(cache=_cache(pos=None)), BAD),
    (dict(cache=_cache(table=None)), BAD), (dict(cache_len=_i32(3, 0)), BAD), (dict(cache_len=_i32(-1, 0)), BAD), (dict(cache_len=None), BAD),
    (dict(page_off=None), BAD), (dict(page_off=_i32(0, 2, 1)), BAD), (dict(loc_len=_i32(-1, 0)), BAD), (dict(loc_len=_i32(3, 2)), BAD), (dict(loc_off=None), BAD),
    (dict(loc_pos0=None), BAD), (dict(locK=None), BAD), (dict(locV=P + 8), BAD), (dict(q_pos0=_i32(9, 2 ** 30)), BAD), (dict(q_pos0=_i32(-2 ** 30 - 1, 0)), BAD),
    (dict(loc_pos0=_i32(2 ** 30 - 2, 0)), BAD), (dict(workspace=P + 8), BAD),
])
def test_attend_paged_refuses(ctx, change, status):
    assert _call(ctx, "dodo_attend_paged", **_attend(**change)) == status
    assert len(ctx[0].dodo_last_error(ctx[1])) > 0


def test_attend_paged_without_queries_is_nothing(ctx):
    assert _call(ctx, "dodo_attend_paged", **_attend(q_off=_i32(0, 0, 0), Q=None)) == 0


# ---- what the binding refuses by itself -------------------------------------------------------------------------------
@pytest.fixture()
def host(libdodo, monkeypatch):
    from paper_2310_02409_b200 import api
    monkeypatch.setattr(api, "_stream", lambda: 0)
    d = api.Dodo.__new__(api.Dodo)
    d._lib, d._ctx = api.load(), ctypes.c_void_p()
    d._lib.dodo_create(ctypes.byref(d._ctx), 0)
    d._index, d.device = -1, torch.device("cpu")
    yield d
    d.close()


def _pool(pages=4, page=2, H=2, dh=64, dtype=torch.float32, entries=2):
    from paper_2310_02409_b200 import api
    z = lambda *s, t=dtype: torch.zeros(s, dtype=t)  # noqa: E731
    return api.PagedCache(z(pages, page, H, dh), z(pages, page, H, dh), z(pages, page, t=torch.int32), z(entries, t=torch.int32))


def test_paged_cache_checks_its_tensors(libdodo):
    from paper_2310_02409_b200 import api
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)  # noqa: E731
    good = dict(K=z(4, 2, 2, 64), V=z(4, 2, 2, 64), pos=z(4, 2, t=torch.int32), table=z(2, t=torch.int32))
    api.PagedCache(**good)
    for bad in (dict(K=z(8, 2, 64)), dict(V=z(4, 2, 2, 32)), dict(V=z(4, 2, 2, 64, t=torch.bfloat16)), dict(pos=z(4, 2)), dict(pos=z(7, t=torch.int32)),
                dict(table=z(2)), dict(table=z(4, t=torch.int32)[::2]), dict(K=z(4, 2, 64, 2).transpose(2, 3)), dict(K=z(4, 2, 2, 64, t=torch.float64))):
        with pytest.raises((TypeError, ValueError)):
            api.PagedCache(**{**good, **bad})
    cache = api.PagedCache(**good)
    with pytest.raises(TypeError):
        cache.table = z(5)
    cache.table = z(5, t=torch.int32)
    assert cache.entries == 5


def test_binding_refuses_shapes_and_tables(host):
    from paper_2310_02409_b200 import api
    rope = api.Rope(np.ones(32))
    Q, K = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    for args in ((rope, [0, 6], [0], Q, K), (rope, [0, 5], [], Q), (rope, [0, 5], [0], Q, K[:4]), (rope, [0, 5], [0], Q, K[..., :32]),
                 (rope, [0, 5], [0], Q, None, Q[:4]), (rope, [0, 5], [0], Q, None, None, K), (rope, [0, 5], [0], torch.zeros(5, 64, 4).transpose(1, 2)),
                 (rope, [0, 5], [0], Q[0])):
        with pytest.raises(ValueError):
            host.rope(*args)
    with pytest.raises(TypeError):
        host.rope(rope, [0, 5], [0], Q, K.bfloat16())
    cache, n = _pool(), np.zeros(1, np.int32)
    g = dict(K=K, V=K, seq_off=[0, 5], idx=None, nug_off=None, pos_base=[0], rope=rope, cache=cache, page_off=[0, 2], cache_len=n)
    for bad in (dict(K=Q, V=Q), dict(V=K[:4]), dict(seq_off=[0, 6]), dict(pos_base=[]), dict(page_off=[0, 3]), dict(page_off=[0]), dict(cache_len=n[:0]),
                dict(idx=torch.zeros(2, dtype=torch.int32), nug_off=[0, 3]), dict(V=torch.zeros(5, 4, 64)[:, :2]), dict(K=torch.zeros(2, 5, 64).transpose(0, 1))):
        with pytest.raises(ValueError):
            host.gather_kv_paged(**{**g, **bad})
    with pytest.raises(TypeError):
        host.gather_kv_paged(**{**g, "K": K.bfloat16()})
    a = dict(Q=Q, q_off=[0, 5], q_pos0=[0], sm_scale=0.1, cache=cache, page_off=[0, 2], cache_len=[2], locK=None, locV=None, loc_off=None, loc_len=None,
             loc_pos0=None, O=torch.zeros_like(Q), lse=None, workspace=None)
    for bad in (dict(Q=Q[..., :32].contiguous()), dict(q_off=[0, 6]), dict(q_pos0=[]), dict(O=torch.zeros(4, 4, 64)), dict(page_off=[0, 3]), dict(cache_len=[]),
                dict(lse=torch.zeros(3)), dict(locK=torch.zeros(3, 2, 64), locV=torch.zeros(2, 2, 64), loc_off=[0], loc_len=[1], loc_pos0=[0]),
                dict(locK=torch.zeros(3, 2, 64), locV=torch.zeros(3, 2, 64)), dict(loc_len=[])):
        with pytest.raises(ValueError):
            host.attend_paged(**{**a, **bad})


@pytest.mark.parametrize("heads,status", [((65536,), UNSUP), ((40000, 40000), UNSUP), ((2 ** 31 - 1, 2 ** 31 - 1), UNSUP)])
def test_rope_refuses_more_heads_than_a_launch_counts(ctx, heads, status):
    arrays = b"".join(_array(heads=h) for h in heads)
    assert _call(ctx, "dodo_rope", **_rope(arrays=arrays, n=len(heads))) == status
