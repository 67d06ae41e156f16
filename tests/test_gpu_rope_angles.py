"""Rotary positions on the GPU: how exact the angle is, seen where its sine is small."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2310_02409_b200 import api

pytestmark = pytest.mark.gpu

PI = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


def _turns(freq, pos):
    """The angle's fraction of a turn in (-1/2, 1/2], exact to 200 bits."""
    t = Fraction(freq) * int(pos) / (2 * PI)
    t -= t.__floor__()
    return t if t <= Fraction(1, 2) else t - 1


@pytest.mark.parametrize("layout", [api.ROPE_HALF, api.ROPE_INTERLEAVED])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("pos", [2 ** 31 - 1, -2 ** 31, 1 << 24, 70001, 1])
def test_angles_are_exact_to_the_rounding_of_their_top_32_bits(dodo, layout, back, pos):
    """Frequencies of up to a radian that turn a pair by almost whole turns up to this position: the sine is then as exact as the angle.  Half a
    unit of the 32 bits, and position times what the frequency's 64 bits are off (rounded once when made, and an 80-bit product of two rounded
    factors below 1/4: one and a half of their half units): 2^-33 + 1.5 x 2^-65 |position| turns.  The sine's own arithmetic: 8 roundings of it."""
    rs = np.random.RandomState(7)
    k = np.maximum(rs.randint(1, max(abs(pos) // 7, 2), 128), 1)
    freq = np.minimum(2.0 * np.pi * k / abs(pos), 1.0) if abs(pos) > 7 else 1e-6 * k
    rope = api.Rope(freq, layout)
    X = torch.zeros((1, 1, 256), device="cuda")
    a, b = (slice(0, 128), slice(128, 256)) if layout == api.ROPE_HALF else (slice(0, 256, 2), slice(1, 256, 2))
    X[..., a] = 1.0
    Y = torch.empty_like(X)
    (dodo.rope_backward if back else dodo.rope)(rope, [0, 1], [pos], X, None, Y)
    got = Y[0, 0, b].double().cpu().numpy() * (-1.0 if back else 1.0)
    for f, y in zip(freq, got):
        want = float(np.sin(2.0 * np.pi * float(_turns(f, pos))))
        bound = 2.0 * np.pi * (2.0 ** -33 + 1.5 * 2.0 ** -65 * abs(pos)) + 8 * 2.0 ** -24 * abs(want)
        assert abs(y - want) <= bound, (f, y, want, bound)
