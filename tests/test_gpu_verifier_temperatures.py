"""The sampled walk at temperatures far from 1, on the GPU against the plain fp64 walk."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
from test_gpu_verifier import BF, _trees, _verify

pytestmark = pytest.mark.gpu


def _walks(seed, dtype, V, T, logits):
    """Walks of random trees at temperature T against the plain ones: all decisions are equal.  `logits(gen, shape)` -> fp32 numbers."""
    from paper_2608_20375_b200 import Graft
    B, nmax, L = 48, 30, 8
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    g = Graft(V, L, 4, 16, 8, B, 1, nmax - 1, 1, 0.0)
    counts = rng.integers(2, nmax + 1, B)
    parent, _, _, token = _trees(rng, B, nmax, counts, V, L)
    z = logits(gen, (B, nmax, V))
    for b in range(B):  # most of what was drafted is among the target's likeliest
        for i in range(1, counts[b]):
            if rng.random() < 0.8:
                row = z[b, parent[b, i]]
                row[token[b, i]] = row.max()
    z = z.to(dtype)
    Ts = np.full(B, T, np.float32)
    u = torch.rand((B, nmax), generator=gen, device="cuda")
    zc = z.cpu().double().numpy()
    for small in (1.0, 2.0 ** -9):  # (at numbers this small a child with any weight to speak of is kept)
        u[:, 1:] *= small
        alen, path, bonus, st = _verify(g, B, nmax, nmax, counts, parent, token, z, Ts, u, L)
        assert not st.any()
        uc = u.cpu().double().numpy()
        for b in range(B):
            a, pa, bo = ref.walk(counts[b], parent[b], token[b], lambda i: zc[b, i], Ts[b], uc[b], L)
            assert (alen[b], bonus[b]) == (a, bo) and np.array_equal(path[b], pa), (b, alen[b], a, bonus[b], bo)
        assert len(set(bonus.tolist())) > 4


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T", [1e-3, 1e-6, 1e-10, 1e-16, 1e-20, 1e-30, 1e-40])
@pytest.mark.parametrize("top", [0.0, 20.0, -3000.0])
def test_low_temperatures_draw_among_the_likeliest(T, top, dtype):
    """Logits in steps, the largest of each row many times: what is left at a low temperature is a draw among those, not the first of them."""
    def logits(gen, shape):
        z = torch.randint(-12, 1, shape, generator=gen, device="cuda").float() * (16.0 if abs(top) > 100 else 0.25)
        return z + top

    _walks(1, dtype, 501, T, logits)


@pytest.mark.parametrize("T", [1e-3, 1e-6, 1e-10, 1e-18])
def test_low_temperatures_of_logits_as_small(T):
    """Logits of the temperature's size: all weights count."""
    _walks(2, torch.float32, 4001, T, lambda gen, shape: 2.0 * T * torch.randn(shape, generator=gen, device="cuda"))


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T", [1e4, 1e20, 1e35, 1e36, 1e38, 3.4e38])
def test_high_temperatures_leave_out_what_is_ruled_out(T, dtype):
    """-inf weighs nothing at any temperature; the type's lowest number does when the temperature is as large."""
    def logits(gen, shape):
        z = torch.randn(shape, generator=gen, device="cuda")
        z[..., ::3] = -math.inf
        z[..., 1::3] = torch.finfo(dtype).min
        z[::2, :, 2::6] = 1e37
        return z

    _walks(3, dtype, 3001, T, logits)
