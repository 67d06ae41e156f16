"""What the binding checks by itself, on the host: a call is refused before it reaches the library, or reaches it with nothing to do,
so neither a device nor device memory is needed (the tensors are the host's, on "device" -1)."""
import ctypes

import numpy as np
import pytest
import torch


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


class Reached:
    """In the library's place: notes that the call came this far."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if not name.startswith("dodo_attend"):
            return lambda *a: 0
        return lambda *a: self.calls.append(name) or 0


H, DH = 2, 64


def _empty(n=0):
    return torch.zeros((n, H, DH))


def _attend(**k):
    return {**dict(Q=_empty(), q_off=[0, 0, 0], q_pos0=[0, 0], sm_scale=0.125, cache_q4=None, cache_scale=None, cache_pos=None, cache_off=None,
                   cache_len=None, locK=None, locV=None, loc_off=None, loc_len=None, loc_pos0=None, O=_empty(), lse=None, workspace=None), **k}


def _backward(**k):
    return {**dict(Q=_empty(), q_off=[0, 0, 0], q_pos0=[0, 0], sm_scale=0.125, cacheK=None, cacheV=None, cache_pos=None, cache_off=None,
                   cache_len=None, locK=None, locV=None, loc_off=None, loc_len=None, loc_pos0=None, O=_empty(), lse=torch.zeros((0, H)), dO=_empty(),
                   dQ=_empty(), dcacheK=None, dcacheV=None, dlocK=None, dlocV=None, dscore=None, workspace=None), **k}


CALLS = [("attend_q4", _attend), ("attend_backward", _backward)]


@pytest.mark.parametrize("name,args", CALLS)
@pytest.mark.parametrize("change", [
    dict(cache_len=[0, 0], cache_off=[0]), dict(cache_len=[0, 0], cache_off=[0, 0]), dict(cache_len=[0, 0]), dict(cache_len=[0], cache_off=[0, 0, 0]),
    dict(loc_len=[0]), dict(loc_len=[0, 0], loc_off=[0]), dict(loc_len=[0, 0], loc_off=[0, 0], loc_pos0=[0]),
])
def test_tables_are_checked_without_their_tensors_too(host, name, args, change):
    """The library reads a table that it is given whether or not there is a cache or a local array beside it."""
    host._lib = Reached()
    with pytest.raises(ValueError):
        getattr(host, name)(**args(**change))
    assert host._lib.calls == []


@pytest.mark.parametrize("name,args", CALLS)
@pytest.mark.parametrize("change", [dict(), dict(cache_len=[0, 0], cache_off=[0, 0, 3]), dict(cache_off=[0]), dict(loc_len=[0, 0]), dict(loc_len=[0, 0], loc_off=[0, 0], loc_pos0=[5, 5])])
def test_calls_without_a_segment_reach_the_library(host, name, args, change):
    getattr(host, name)(**args(**change))
