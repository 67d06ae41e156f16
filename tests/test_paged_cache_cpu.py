"""PagedCache holds what it was made of: what the library is given and what the program sees of it cannot drift apart."""
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
