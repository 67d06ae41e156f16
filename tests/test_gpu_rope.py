"""Rotary positions on the GPU against the formula in 64 bits and more: layouts, partial rotation, far and negative positions, odd head
sizes, strides and alignment, in place, the gradient."""
import numpy as np
import pytest
import torch

import paged64
import plain64
from paper_2310_02409_b200 import api, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LAYOUT = {"half": api.ROPE_HALF, "interleaved": api.ROPE_INTERLEAVED}


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _half(dtype):
    return plain64.HALF["bf16" if dtype is BF else "f32"]


def _positions(off, pos0):
    return np.concatenate([p + np.arange(b - a) for a, b, p in zip(off, off[1:], pos0)]) if len(pos0) else np.zeros(0)


def _close(got, x, pos, freq, layout, scale, dtype, back=False):
    want, bound = paged64.rope(_f64(x), pos, freq, layout, scale, back)
    err = np.abs(_f64(got) - want)
    assert (err <= bound + _half(dtype) * (np.abs(want) + bound)).all(), float((err - bound - _half(dtype) * np.abs(want)).max())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,H,Hkv,dh,rot", [
    (BF, 32, 32, 128, 128), (BF, 32, 8, 128, 64), (BF, 5, 1, 64, 64), (F32, 4, 4, 64, 64), (F32, 12, 3, 64, 24), (BF, 3, 3, 80, 80), (BF, 7, 7, 96, 30),
    (F32, 2, 1, 256, 256), (BF, 2, 2, 512, 256), (F32, 3, 1, 10, 6), (BF, 1, 1, 2, 2), (BF, 40, 40, 128, 2), (F32, 5, 5, 20, 8), (F32, 70, 70, 64, 64),
])
@pytest.mark.parametrize("back", [False, True])
def test_rope_is_the_formula(dodo, layout, dtype, H, Hkv, dh, rot, back):
    lens, pos0 = [3, 0, 1, 37], [5, 9, 123456, 2 ** 31 - 37]
    off = inputs.offsets(lens)
    N = int(off[-1])
    freq = api.rope_frequencies(rot, 10000.0)
    rope = api.Rope(freq, LAYOUT[layout], 1.25)
    Q, K = inputs.randn((N, H, dh), "rope", H, dh, "Q", dtype=dtype).cuda(), inputs.randn((N, Hkv, dh), "rope", H, dh, "K", dtype=dtype).cuda()
    oq, ok = torch.full_like(Q, 7.0), torch.full_like(K, 7.0)
    (dodo.rope_backward if back else dodo.rope)(rope, off, pos0, Q, K, oq, ok)
    torch.cuda.synchronize()
    for x, y in ((Q, oq), (K, ok)):
        _close(y, x, _positions(off, pos0), freq, layout, 1.25, dtype, back)
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,H", [(1, 32), (5000, 6), (4737, 3), (8, 300)])
def test_rope_of_many_rows_and_heads(dodo, layout, rows, H):
    freq = api.rope_frequencies(64, 500000.0, api.ROPE_PARTS, 8.0, 4096)
    X = inputs.randn((rows, H, 64), "rope rows", rows, dtype=BF).cuda()
    Y = torch.empty_like(X)
    dodo.rope(api.Rope(freq, LAYOUT[layout]), [0, rows], [-17], X, None, Y)
    torch.cuda.synchronize()
    _close(Y, X, -17 + np.arange(rows), freq, layout, 1.0, BF)


def test_rope_of_many_sequences_and_of_the_ends_of_the_range(dodo):
    B = 131
    off, pos0 = np.arange(B + 1, dtype=np.int32) * 2, np.linspace(-2 ** 31, 2 ** 31 - 2, B).astype(np.int64)
    freq = np.concatenate([api.rope_frequencies(12), [3.0, -0.7, 0.0, 1e-9]])
    X = inputs.randn((2 * B + 3, 2, 40), "rope ends", dtype=F32).cuda()
    Y = torch.full_like(X, 3.0)
    dodo.rope(api.Rope(freq, api.ROPE_HALF), off, pos0.astype(np.int32), X, None, Y)
    torch.cuda.synchronize()
    _close(Y[:2 * B], X[:2 * B], _positions(off, pos0), freq, "half", 1.0, F32)
    assert (Y[2 * B:] == 3.0).all()            # rows behind the last sequence


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_rope_takes_strides_and_works_in_place(dodo, layout, dtype, shift):
    """Q and K as slices of a fused projection, at any alignment; what lies between them stays."""
    N, H, Hkv, dh = 19, 6, 2, 64
    width = (H + 2 * Hkv) * dh + shift + 8
    base = inputs.randn((N, width), "rope fused", shift, dtype=dtype).cuda()
    view = lambda b, a, h: b.as_strided((N, h, dh), (width, dh, 1), shift + a * dh)  # noqa: E731
    before = base.clone()
    freq = api.rope_frequencies(64)
    rope = api.Rope(freq, LAYOUT[layout], 0.5)
    dodo.rope(rope, [0, 7, N], [3, 1000], view(base, 0, H), view(base, H, Hkv))
    torch.cuda.synchronize()
    pos = _positions([0, 7, N], [3, 1000])
    for a, h in ((0, H), (H, Hkv)):
        _close(view(base, a, h), view(before, a, h), pos, freq, layout, 0.5, dtype)
    assert torch.equal(view(base, H + Hkv, Hkv), view(before, H + Hkv, Hkv)) and torch.equal(base[:, width - 8:], before[:, width - 8:])
    # heads that do not lie side by side, to a dense output
    out = torch.empty((N, H, dh), dtype=dtype, device="cuda")
    wide = inputs.randn((N, H, 3, dh), "rope heads", dtype=dtype).cuda()
    dodo.rope(rope, [0, N], [0], wide[:, :, 1], None, out)
    torch.cuda.synchronize()
    _close(out, wide[:, :, 1], np.arange(N), freq, layout, 0.5, dtype)


def test_rope_not_finite_stays_in_its_pair(dodo):
    X = inputs.randn((4, 2, 64), "rope nan", dtype=F32).cuda()
    X[1, 0, 3] = float("nan")
    X[2, 1, 40] = float("inf")
    Y = torch.empty_like(X)
    dodo.rope(api.Rope(api.rope_frequencies(64)), [0, 4], [1], X, None, Y)
    bad = torch.nonzero(~torch.isfinite(Y)).tolist()
    assert bad == [[1, 0, 3], [1, 0, 35], [2, 1, 8], [2, 1, 40]]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_backward_is_the_gradient(dodo, layout):
    """Against the formula above; here against differences of the rotation itself, along random directions."""
    N, H, dh, rot = 11, 3, 64, 48
    rope = api.Rope(api.rope_frequencies(rot, 10000.0, api.ROPE_LINEAR, 4.0), LAYOUT[layout], 1.5)
    new = lambda name: inputs.randn((N, H, dh), "rope grad", name, dtype=F32).cuda()  # noqa: E731
    X, D, G = new("X"), new("D"), new("G")
    turn = lambda x, call: (lambda y: (call(rope, [0, N], [70000], x, None, y), y)[1])(torch.empty_like(x))  # noqa: E731
    slope = (turn(X + D, dodo.rope).double() - turn(X - D, dodo.rope).double()) / 2.0      # the rotation is linear
    lhs, rhs = (slope * G.double()).sum().item(), (D.double() * turn(G, dodo.rope_backward).double()).sum().item()
    # 10 roundings (8 of a turn, one of a sum or difference, one of the result) of values of up to 1.5 (|x| + |d|) a feature, each side
    size = 10 * paged64.U * 1.5 * 2.0 * float(((X.abs() + D.abs()).amax() + G.abs().amax()) * (G.abs().sum() + D.abs().sum()))
    assert abs(lhs - rhs) <= size


def test_rope_captured_and_replayed_on_another_stream(dodo):
    X = inputs.randn((9, 4, 128), "rope graph", dtype=BF).cuda()
    Y, Z = torch.empty_like(X), torch.empty_like(X)
    rope = api.Rope(api.rope_frequencies(128))
    dodo.rope(rope, [0, 9], [77], X, None, Y)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dodo.rope(rope, [0, 9], [77], X, None, Z)
    for _ in range(2):
        Z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, Z)


def test_rope_behind_2_31_elements(dodo):
    """Rows whose elements have indices beyond 32 bits: a row stride of 2^30."""
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GB of device memory")
    base = torch.zeros(3 * 2 ** 30 + 128, dtype=BF, device="cuda")
    X = base.as_strided((4, 1, 128), (2 ** 30, 128, 1))
    X.copy_(inputs.randn((4, 1, 128), "rope far", dtype=BF))
    before = X.contiguous()
    freq = api.rope_frequencies(128)
    dodo.rope(api.Rope(freq), [0, 4], [100], X)
    torch.cuda.synchronize()
    _close(X.contiguous(), before, 100 + np.arange(4), freq, "half", 1.0, BF)
