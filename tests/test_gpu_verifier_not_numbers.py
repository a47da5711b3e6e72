"""Entries that are not numbers, in places that rows of the verifier's attention see, on the GPU against plain fp64 forms."""
import math

import numpy as np
import pytest
import torch

from test_gpu_verifier import BF, Q8, _attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk,D", [(20, 16, 2, 128), (33, 8, 2, 64)])
def test_values_that_are_not_numbers_in_units_that_follow_one_another(rows, Hq, Hk, D, dtype):
    """Hundreds of short units of 129 to 256 rows, several a thread block, each with new values that are not numbers: every row that sees
    them has them, in all units."""
    B = 150
    rng = np.random.default_rng(rows)
    lens = rng.integers(1, 90, B).tolist()

    def spoil(key, value):
        for b, n in enumerate(lens):
            value[b, n - 1 + b % 3] = math.nan
            value[b, n - 1 + 3 + b % 5, :, b % D] = math.inf
            value[b, n - 1 + 9 + b % 7, b % Hk, 5] = -math.inf

    out = _attend(rows, B, rows, Hq, Hk, D, 16, lens, [rows] * B, dtype, "tree", spoil=spoil)
    assert all(torch.isnan(out[b]).any() for b in range(B))
