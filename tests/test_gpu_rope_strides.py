"""Rotations of arrays in unusual orders of rows and heads, and of broadcast inputs, which lie over one another only where they are read."""
import pytest
import torch

import numpy as np
from paper_2310_02409_b200 import api, inputs
from test_gpu_rope import BF, F32, LAYOUT, _close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,heads,row,head", [(5, 4, 64, 320), (5, 4, 64, 384), (2, 3, 128, 192), (3, 3, 192, 256), (1, 4, 0, 64), (4, 1, 64, 0), (5, 4, 257, 64)])
def test_outputs_in_any_order_that_keeps_them_apart(dodo, layout, dtype, rows, heads, row, head):
    at = np.sort((np.arange(rows)[:, None] * row + np.arange(heads)[None] * head).ravel())
    assert (np.diff(at) >= 64).all()
    base = torch.full((rows * max(row, 1) + heads * max(head, 1) + 64,), 3.0, dtype=dtype, device="cuda")
    X, Y = inputs.randn((rows, heads, 64), "rope order", rows, heads, dtype=dtype).cuda(), base.as_strided((rows, heads, 64), (row, head, 1))
    freq = api.rope_frequencies(64)
    dodo.rope(api.Rope(freq, LAYOUT[layout]), [0, rows], [11], X, None, Y)
    torch.cuda.synchronize()
    _close(Y, X, 11 + np.arange(rows), freq, layout, 1.0, dtype)
    Y.fill_(3.0)
    assert (base == 3.0).all()                 # nothing else was written


@pytest.mark.parametrize("back", [False, True])
def test_broadcast_inputs(dodo, back):
    freq = api.rope_frequencies(64)
    for x in (inputs.randn((5, 1, 64), "rope shared", dtype=BF).cuda().expand(5, 4, 64), inputs.randn((1, 4, 64), "rope shared", dtype=BF).cuda().expand(5, 4, 64)):
        Y = torch.empty((5, 4, 64), dtype=BF, device="cuda")
        (dodo.rope_backward if back else dodo.rope)(api.Rope(freq), [0, 5], [11], x, None, Y)
        torch.cuda.synchronize()
        _close(Y, x, 11 + np.arange(5), freq, "half", 1.0, BF, back)
