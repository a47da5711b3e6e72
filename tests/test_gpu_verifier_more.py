"""More of the verifier's operators on the GPU against plain fp64 forms: few rows a sequence, many sequences with long prefixes, scales at both
ends, entries that are not numbers."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
from test_gpu_verifier import BF, Q8, _attend, _cache, _graft, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,mask", [
    (1, 8, 1, 1, 64, 16, [1], [8], "tree"),                                       # eight rows, nothing before them
    (3, 1, 7, 1, 128, 64, [1, 17, 2000], [1, 1, 1], None),                        # seven rows
    (2, 2, 4, 1, 64, 1024, [1023, 15], [2, 1], "random"),
    (4, 4, 4, 2, 128, 16, [15, 16, 17, 400], [4, 0, 3, 1], "tree"),
    (2, 8, 2, 2, 64, 32, [33, 130], [8, 7], "random"),
    (2, 3, 2, 1, 128, 128, [1, 140], [3, 2], "empty"),
    (1, 1, 2, 1, 128, 64, [20000], [1], None),                                    # one sequence over all SMs
    (3, 3, 3, 1, 64, 64, [100, 1, 300], [3, 3, 2], "tree"),                       # nine rows: not few
])
def test_few_rows(dtype, B, rows, Hq, Hk, D, page, lens, counts, mask):
    _attend(11 * rows + B, B, rows, Hq, Hk, D, page, lens, counts, dtype, mask)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows", [1, 20])
def test_many_sequences_with_long_prefixes(dtype, rows):
    """More bytes of K and V than one wave of copies: rings go round many times and copies arrive out of order."""
    B = 48
    rng = np.random.default_rng(rows)
    _attend(rows, B, rows, 16, 4, 128, 64, rng.integers(1500, 2600, B).tolist(), [rows] * B, dtype, None)


@pytest.mark.parametrize("B,rows", [(33, 1), (257, 20), (600, 1), (600, 17)])
def test_many_sequences(B, rows):
    """More sequences than a warp, a block or the plan's shared memory has places for."""
    rng = np.random.default_rng(B)
    _attend(B, B, rows, 2, 1, 64, 16, rng.integers(1, 90, B).tolist(), rng.integers(0, rows + 1, B).tolist(), BF, "tree")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows", [4, 8, 40])
def test_scales_at_both_ends(rows, dtype, D):
    """Entries from 2^-100 to 2^100: of e4m3 rows, scales on both sides of those that one factor in bf16 holds."""
    def spread(key, value):
        key[:, ::7] *= 2.0 ** -100
        value[:, ::5] *= 2.0 ** 100
        value[:, 1::5] *= 2.0 ** -100
        value[:, 2::5] *= 2.0 ** 12

    _attend(5, 2, rows, 2, 2, D, 16, [150, 40], [rows, rows - 1], dtype, "tree", spoil=spread)

    def large(key, value):
        key[:, ::7] *= 2.0 ** 10
        value *= 2.0 ** -110

    _attend(6, 2, rows, 2, 2, D, 16, [150, 40], [rows, rows - 1], dtype, "tree", spoil=large, scale=2.0 ** -10)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk", [(8, 2, 2), (4, 4, 2)])
def test_few_rows_that_do_not_see_what_is_not_a_number(rows, Hq, Hk, dtype, D):
    lens = [90, 121]

    def spoil(key, value):
        for b, n in enumerate(lens):
            value[b, n - 1 + 1] = math.nan
            value[b, n - 1 + 2, :, 3] = math.inf
            value[b, n - 1 + 3:n - 1 + 4, 0, 5] = math.nan  # (the second sequence of four rows has three)

    out = _attend(rows, 2, rows, Hq, Hk, D, 16, lens, [rows, rows - 1], dtype, "tree", spoil=spoil)
    assert torch.isnan(out).any() and torch.isfinite(out[0, 0]).all()


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows", [2, 20])
def test_rows_of_q_with_a_stride(dtype, rows):
    """Q taken where it stands in a fused projection: the same bits as from a copy."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    B, Hq, Hk, D, page = 3, 4, 2, 128, 16
    g = _graft(max(2, rows), B)
    table, n_pages = ref.page_table(np.random.default_rng(1), B, 12)
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype)
    x = torch.randn((B, 150 + rows, Hq + 2 * Hk, D), generator=gen, device="cuda").to(BF)
    q, key, value = x[:, -rows:, :Hq], x[:, :, Hq:Hq + Hk], x[:, :, Hq + Hk:]
    g.cache_write(c, 0, _i32(table), _i32([1] * B), _i32([150 + rows] * B), key, value)
    outs = []
    for qq in (q.contiguous(), x[:, -rows:].contiguous()[:, :, :Hq]):
        out = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
        g.tree_attention(c, 0, _i32(table), qq, _i32([151] * B), _i32([rows] * B), None, out)
        outs.append(out)
    assert torch.equal(*outs) and outs[0].abs().sum() > 0
