"""A rotation of as many rows as 32 bits count."""
import pytest
import torch

import numpy as np
import paged64
import plain64
from paper_2310_02409_b200 import api

pytestmark = pytest.mark.gpu


def test_rows_up_to_the_end_of_32_bits(dodo):
    """2^31 - 1 rows of one head of two features, in place: the last block of two rows has one."""
    rows = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 11 << 30:
        pytest.skip("needs 11 GB of device memory")
    X = torch.ones((rows, 1, 2), dtype=torch.bfloat16, device="cuda")
    X[:, :, 1] = 0.5
    dodo.rope(api.Rope([0.37]), [0, rows], [-5], X)
    torch.cuda.synchronize()
    for at in (slice(0, 300), slice(2 ** 30 - 3, 2 ** 30 + 3), slice(rows - 300, rows)):
        pos = -5 + np.arange(at.start, at.stop, dtype=np.int64)
        want, bound = paged64.rope(np.tile([1.0, 0.5], (len(pos), 1, 1)), pos, [0.37], "half")
        half = plain64.HALF["bf16"]
        assert (np.abs(X[at].float().cpu().numpy().astype(np.float64) - want) <= bound + half * (np.abs(want) + bound)).all()
