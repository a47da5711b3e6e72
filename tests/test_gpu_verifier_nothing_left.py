"""The sampled walk at nodes whose children hold nearly all of the target's distribution, on the GPU."""
import math

import numpy as np
import pytest
import torch

from test_gpu_verifier import BF, _verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_a_token_that_is_ruled_out_is_never_kept(dtype):
    """Children with less and less weight, each rejected by the largest number below 1, until what is left is of the size of a rounding, or
    less than nothing; behind them children that the target rules out."""
    from paper_2608_20375_b200 import Graft
    B, N, V, L = 2048, 13, 64, 2
    rng, gen = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(1)
    g = Graft(V, L, 4, 16, 8, B, 1, N - 1, 1, 0.0)
    parent = np.tile(np.array([-1] + [0] * (N - 1), np.int32), (B, 1))
    token = np.stack([rng.permutation(V)[:N] for _ in range(B)]).astype(np.int32)
    z = torch.full((B, N, V), -math.inf, device="cuda")
    for b in range(B):  # (e^-16.6 is half a rounding of u below 1: the second child is why the first is rejected, the third why the second is)
        a, c = rng.uniform(13.0, 16.6), rng.uniform(12.0, 16.6)
        for k, x in enumerate((0.0, -a, -a - c)):
            z[b, 0, token[b, k + 1]] = 3.0 + x
    z[:, 1:] = torch.randn((B, N - 1, V), generator=gen, device="cuda")
    u = torch.full((B, N), float(np.nextafter(np.float32(1), np.float32(0))), device="cuda")
    alen, path, bonus, st = _verify(g, B, N, N, np.full(B, N), parent, token, z.to(dtype), None, u, L)
    assert not st.any()
    assert (path[:, 0] < 4).all(), (path[:, 0] >= 4).sum()
    assert 0 < (path[:, 0] > 1).sum()  # the first child was rejected somewhere
