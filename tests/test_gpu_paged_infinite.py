"""Attention over the paged nugget cache: a key whose logit is -infinity counts as one not seen, whatever its V holds."""
import pytest
import torch

from test_gpu_paged import BF, F32, _batch, _check
from test_gpu_paged_choice import FEW, FMA, TENSOR_CORES, TILE, run_on, tensor_cores

pytestmark = pytest.mark.gpu


def _minus_infinity(s, bad):
    """Some cached keys of every sequence, and all of the last one's, get a logit of -infinity; what is left for the plain form."""
    s["Q"][..., 0] = s["Q"][..., 0].abs() + 0.5
    want = {k: (v.clone() if isinstance(v, torch.Tensor) else v.copy() if hasattr(v, "copy") else v) for k, v in s.items()}
    for b in range(s["B"]):
        r = s["rows"][b]
        gone = r if b == s["B"] - 1 else r[3::7]
        s["cK"][gone, :, 0] = float("-inf")
        s["cV"][gone] = bad
        want["pos"][gone] = 2 ** 31 - 1
    return want


@pytest.mark.parametrize("kernel,dtype,H,Hkv,tq,B,page", [
    (FEW, BF, 4, 4, 1, 3, 16), (FEW, BF, 8, 2, 3, 3, 16), (FEW, BF, 4, 2, 40, 3, 16), (FMA, BF, 4, 2, 4, 3, 5), (FMA, F32, 4, 4, 1, 3, 16), (FMA, F32, 8, 2, 3, 3, 24),
    (FMA, F32, 4, 4, 20, 3, 16), (TILE, F32, 16, 8, 20, 40, 16), (TENSOR_CORES, BF, 4, 2, 40, 3, 16), (TENSOR_CORES, BF, 4, 2, 140, 3, 16), (TENSOR_CORES, BF, 4, 2, 90, 3, 5)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 1.0])
def test_a_logit_of_minus_infinity_counts_as_not_seen(dodo, kernel, dtype, H, Hkv, tq, B, page, dh, bad):
    s = _batch(dtype, H, Hkv, dh, [tq] * B, [200] * (B - 1) + [50], [tq] * (B - 1) + [0], page, seed=tq)
    want = _minus_infinity(s, bad)
    with tensor_cores(dodo, 1 if kernel == TENSOR_CORES else 2):
        O, L = run_on(dodo, s, kernel)
    _check(want, O, L, only=[0, 1, B - 1])
    last = int(s["q_off"][B - 1])
    assert (O[last:] == 0).all() and torch.isneginf(L[last:]).all()
