"""PagedCache holds what it was made of: what the library is given and what the program sees of it cannot drift apart."""
import ctypes

import pytest
import torch


def _tensors(pages=4, page=2, H=2, dh=64):
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)  # noqa: E731
    return dict(K=z(pages, page, H, dh), V=z(pages, page, H, dh), pos=z(pages, page, t=torch.int32), table=z(2, t=torch.int32))


@pytest.mark.parametrize("name", ["K", "V", "pos"])
def test_the_pool_of_a_paged_cache_is_not_replaced(libdodo, name):
    """The library's copy of the addresses is made with the cache: a program that grows its pool makes another one."""
    from paper_2310_02409_b200 import api
    cache, bigger = api.PagedCache(**_tensors()), _tensors(pages=8)
    held, spec = getattr(cache, name), cache.spec
    with pytest.raises(AttributeError):
        setattr(cache, name, bigger[name])
    assert getattr(cache, name) is held and cache.spec == spec
    cache.table = bigger["table"]
    assert cache.table is bigger["table"] and cache.spec != spec


def test_a_paged_cache_refuses_tensors_of_other_shapes(libdodo):
    """As many elements are not enough."""
    from paper_2310_02409_b200 import api
    good = _tensors()
    for bad in (dict(V=good["V"].reshape(4, 4, 1, 64)), dict(V=good["V"].reshape(2, 4, 2, 64)), dict(V=good["V"].reshape(-1)), dict(V=good["V"].reshape(4, 2, 64, 2)),
                dict(pos=good["pos"].reshape(2, 4)), dict(pos=good["pos"].reshape(1, 8)), dict(pos=good["pos"].reshape(4, 2, 1))):
        with pytest.raises(ValueError):
            api.PagedCache(**{**good, **bad})
    api.PagedCache(**{**good, "pos": good["pos"].reshape(-1)})        # positions one after the other are the same array
    assert api.PagedCache(**{**good, "table": torch.zeros((3, 5), dtype=torch.int32)}).entries == 15        # a row for each sequence


def test_attend_paged_refuses_local_tokens_of_other_heads(libdodo, monkeypatch):
    from paper_2310_02409_b200 import api
    monkeypatch.setattr(api, "_stream", lambda: 0)
    host = api.Dodo.__new__(api.Dodo)
    host._lib, host._ctx, host._index, host.device = api.load(), ctypes.c_void_p(), -1, torch.device("cpu")
    host._lib.dodo_create(ctypes.byref(host._ctx), 0)
    z, cache = torch.zeros, api.PagedCache(**_tensors())
    Q = z(5, 4, 64)
    for shape in ((3, 1, 128), (3, 4, 32), (3, 128), (6, 1, 64), (3, 2, 64, 1)):
        with pytest.raises(ValueError):
            host.attend_paged(Q, [0, 5], [0], 0.1, cache, [0, 2], [2], z(shape), z(shape), [0], [3], [0], z(5, 4, 64), None, None)
    host.close()
