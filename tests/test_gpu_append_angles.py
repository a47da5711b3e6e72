"""Cosines and sines of rotated appends are fp32 numbers as near as fp32 has them: where x cos a and y sin a cancel, what is left shows their
last bits."""
import numpy as np
import pytest
import torch

from test_gpu_verifier import BF, _cache, _graft, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,far", [(1, 8), (3, 8), (97, 4096), (1000, 100000)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_what_is_left_of_numbers_that_cancel(P, far, interleaved):
    """Angles close to pi / 4 and a whole number of turns: pairs (1, 1) and (1, -1).  Half a step of a cosine, half a step of a sine (2^-25 each, both
    are below 1), their sum is exact; the result's own rounding to bf16."""
    from paper_2608_20375_b200 import Rope
    rows, D = 200, 128
    rng = np.random.default_rng(P)
    freq = ((np.pi / 4 + 2 * np.pi * np.arange(64)) / P).astype(np.float32)
    pos = P * (8 * rng.integers(0, far, rows) + 1)
    g = _graft(2, 1)
    c = _cache(torch.Generator(device="cuda").manual_seed(0), (1, 14, 1, 16, D), BF, garbage=False)
    q = torch.ones((1, rows, 2, D), dtype=BF, device="cuda")
    q[:, :, 1, slice(1, None, 2) if interleaved else slice(64, None)] = -1
    kv, out = q[:, :, :1].contiguous(), torch.zeros_like(q)
    g.cache_append(c, 0, _i32([list(range(14))]), _i32([1]), _i32([rows]), Rope(torch.from_numpy(freq[None]).cuda(), interleaved), q, kv, kv, out,
                   position=_i32(pos[None]))
    got = out[0].cpu().double().numpy()
    a = pos.astype(np.longdouble)[:, None] * freq.astype(np.longdouble)
    s, co = np.sin(a), np.cos(a)
    # (the angle in fp64: its product, the turns and what is left of them are rounded)
    far_off = np.float64(np.abs(a) * 2.0 ** -51 + 2.0 ** -50)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, 64), slice(64, None))
    for h, y in ((0, 1), (1, -1)):
        for part, want in ((first, co - y * s), (second, s + y * co)):
            want = np.float64(want)
            tol = 2.0 ** -24 * (1 + 2.0 ** -20) + 2 * far_off
            off = np.abs(got[:, h, part] - want) / (tol + 2.0 ** -8 * (np.abs(want) + tol))
            assert off.max() <= 1, (h, off.max(), (off > 1).mean())
