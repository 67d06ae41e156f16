"""Rotations whose output's rows or heads lie over one another are refused on the host; nothing is launched, the pointers are never followed."""
import ctypes
import struct

import numpy as np
import pytest
import torch

P = 0x10000     # an address that nothing reads


@pytest.fixture(scope="module")
def host(libdodo):
    from paper_2310_02409_b200 import api
    d = api.Dodo.__new__(api.Dodo)
    d._lib, d._ctx, d._index, d.device = api.load(), ctypes.c_void_p(), -1, torch.device("cpu")
    d._lib.dodo_create(ctypes.byref(d._ctx), 0)
    yield d
    d.close()


def _lies_over_itself(rows, heads, row, head, dh):
    at = np.sort((np.arange(rows)[:, None] * row + np.arange(heads)[None] * head).ravel())
    return bool((np.diff(at) < dh).any())


@pytest.mark.parametrize("entry", ["dodo_rope", "dodo_rope_backward"])
@pytest.mark.parametrize("rows,heads,row,head", [
    (5, 4, 0, 64), (5, 4, 256, 0), (5, 1, 0, 64), (1, 4, 256, 0), (5, 4, 32, 320), (5, 4, 256, 63), (5, 4, -63, 1000), (5, 4, 64, 64), (5, 4, 192, 64), (5, 4, 128, 192),
    (5, 4, -192, 64), (7, 5, 320, 255), (5, 4, 0, 0), (100, 2, 64, 6336 - 1), (3, 4, 2 ** 62, 0),
])
def test_outputs_that_lie_over_one_another_are_refused(host, entry, rows, heads, row, head):
    from paper_2310_02409_b200 import api
    assert _lies_over_itself(rows, heads, row, head, 64)
    array = struct.pack("QQiiqqqq", P, P, heads, 0, heads * 64, 64, row, head)
    off, pos = np.array([0, rows], np.int32), np.zeros(1, np.int32)
    rc = getattr(host._lib, entry)(host._ctx, api.Rope(np.ones(32))._spec, array, 1, 1, 64, off.ctypes.data, pos.ctypes.data, 1, None)
    assert rc == api.ERR_INVALID_ARG and b"over one another" in host._lib.dodo_last_error(host._ctx)


def test_in_place_on_a_broadcast_tensor_is_refused(host, monkeypatch):
    from paper_2310_02409_b200 import api
    monkeypatch.setattr(api, "_stream", lambda: 0)
    rope = api.Rope(np.ones(32))
    for x in (torch.zeros(5, 1, 64).expand(5, 4, 64), torch.zeros(1, 4, 64).expand(5, 4, 64)):
        with pytest.raises(api.DodoError):
            host.rope(rope, [0, 5], [0], x)
        with pytest.raises(api.DodoError):
            host.rope_backward(rope, [0, 5], [0], torch.zeros(5, 4, 64), None, x)
