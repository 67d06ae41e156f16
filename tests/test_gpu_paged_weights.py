"""Attention over the paged nugget cache: how many bits of a weight meet V."""
import numpy as np
import pytest
import torch

import paged64
import plain64
from test_gpu_paged import BF, _batch, _f64, _run, _sequence

pytestmark = pytest.mark.gpu

# A weight as the sum of two bf16 numbers: the first is off by at most 2^-8 of it, the second by 2^-8 of what the first left.
TWO_PIECES = 2.0 ** -16


def _bf16(v):
    return float(torch.tensor(v, dtype=torch.float64).to(BF))


def _logit():
    """A bf16 logit below 0 whose weight lies far from every bf16 number, but not half way between two."""
    best = max((abs(np.exp(x) - _bf16(np.exp(x))), x) for x in (_bf16(-0.1 - i / 64.0) for i in range(38)) if abs(np.exp(x) - _bf16(np.exp(x))) < 0.9 * 2.0 ** -9)
    return best[1]


def _cancelling(H, Hkv, dh, tq, n, at, page):
    """Two visible keys in one group of sixteen, with logits 0 and x; V of the first is -bf16(exp(x)), of the second 1.  What is left of the sum is
    what a rounding of the weight to bf16 would lose."""
    x = _logit()
    s = _batch(BF, H, Hkv, dh, [tq], [n], [0], page, q_pos0=[1000], span=1)
    s["scale"] = 1.0
    s["Q"].zero_()
    s["Q"][:, :, 0] = 1.0
    s["pos"][s["rows"][0]] = 10 ** 6
    a, b = s["rows"][0][at], s["rows"][0][at + 1]
    s["pos"][[a, b]] = [3, 4]
    s["cK"][a], s["cK"][b] = 0.0, 0.0
    s["cK"][b, :, 0] = x
    s["cV"][a], s["cV"][b] = -_bf16(np.exp(x)), 1.0
    return s


def _holds(s, O, L, weight_half):
    half = plain64.HALF["bf16"]
    q, Q, qpos, K, V, kpos = _sequence(s, 0)
    o, l = paged64.attend(Q, qpos, s["scale"], K, V, kpos)
    tO, tL = paged64.attend_bounds(Q, qpos, s["scale"], K, V, kpos, o, l, half, weight_half)
    assert (np.abs(o) > 4 * tO).all()                  # a result of 0 would not do
    assert (np.abs(_f64(O[q]) - o) <= tO).all(), float((np.abs(_f64(O[q]) - o) - tO).max())
    assert (np.abs(_f64(L[q]) - l) <= tL).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv,tq", [(4, 4, 1), (8, 1, 1), (4, 2, 5), (3, 3, 16)])
@pytest.mark.parametrize("n,at,page", [(2, 0, 16), (205, 84, 16), (9000, 4003, 64), (300, 17, 5)])
def test_few_tokens_keep_sixteen_bits_of_a_weight(dodo, dh, H, Hkv, tq, n, at, page):
    for workspace in (True, False):
        s = _cancelling(H, Hkv, dh, tq, n, at, page)
        _holds(s, *_run(dodo, s, workspace=workspace), TWO_PIECES)
