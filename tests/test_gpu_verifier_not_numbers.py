"""Entries that are not numbers, in places that rows of the verifier's attention see, on the GPU against plain fp64 forms."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
from test_gpu_verifier import BF, Q8, _attend, _cache, _graft, _i32

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


def _expect(q, k, v, seen, scale):
    """One sequence, as ref.attention, but keys count as they are: a row that sees a score of NaN or +inf is NaN, one of -inf weighs nothing."""
    n, Hq, D = q.shape
    group = Hq // k.shape[1]
    parts = []
    for h in range(Hq):
        kh, vh = k[:, h // group], v[:, h // group:h // group + 1]
        with np.errstate(invalid="ignore"):
            s = np.where(seen, scale * (q[:, h] @ kh.T), -math.inf)  # (a sum with an infinity and a zero in its place: NaN)
        lost = (np.isnan(s) | (s == math.inf)).any(1)
        kept = np.where(np.isfinite(kh).all(1)[:, None], kh, 0.0)[:, None]
        out, lse, tol, ltol = ref.attention(q[:, h:h + 1], kept, vh, seen & np.isfinite(s), scale)
        out[lost], lse[lost] = math.nan, math.nan
        parts.append((out, lse, tol, ltol))
    return [np.concatenate(x, 1) for x in zip(*parts)]


def _keys(dtype, rows, Hq, Hk, D, lens, spoil, shared=0, page=16):
    """Chains of `rows` rows behind lens - 1 slots, key entries as spoil left them: out and lse against the definition's."""
    B = len(lens)
    rng, gen = np.random.default_rng(rows), torch.Generator(device="cuda").manual_seed(rows)
    g = _graft(max(2, rows), B)
    table, n_pages = ref.page_table(rng, B, -(-(max(lens) - 1 + rows) // page), shared_pages=shared // page)
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype)
    tb, pl, cnt = _i32(table), _i32(lens), _i32([rows] * B)
    total = max(lens) - 1 + rows
    key, value = (torch.randn((B, total, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    if shared:
        key[:, :shared], value[:, :shared] = key[:1, :shared], value[:1, :shared]
    spoil(key)
    g.cache_write(c, 0, tb, _i32([1] * B), _i32([n - 1 + rows for n in lens]), key, value)
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    out, lse = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda"), torch.zeros((B, rows, Hq), device="cuda")
    g.tree_attention(c, 0, tb, q, pl, cnt, None, out, lse, shared=shared)
    torch.cuda.synchronize()
    o, ls, qq = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.cpu().double().numpy()
    ke, ve = (None, None) if dtype is BF else (c.k_exp[0].cpu(), c.v_exp[0].cpu())
    k0, v0 = c.k[0].cpu(), c.v[0].cpu()
    spoilt = 0
    for b in range(B):
        slots = np.arange(lens[b] - 1 + rows)
        seen = slots[None, :] <= lens[b] - 1 + np.arange(rows)[:, None]
        wo, wl, tol, ltol = _expect(qq[b], ref.entries(k0, ke, table[b], slots), ref.entries(v0, ve, table[b], slots), seen, D ** -0.5)
        assert np.array_equal(np.isnan(o[b]), np.isnan(wo)), (b, np.argwhere(np.isnan(o[b]) != np.isnan(wo))[:5])
        assert np.array_equal(np.isnan(ls[b]), np.isnan(wl)) and np.array_equal(np.isinf(ls[b]), np.isinf(wl))
        fin, lfin = np.isfinite(wo), np.isfinite(wl)
        assert (np.abs(o[b] - wo)[fin] <= tol[fin]).all() and (np.abs(ls[b] - wl)[lfin] <= ltol[lfin]).all()
        spoilt += np.isnan(wl).any()
    return spoilt


KINDS = [(1, 4, 2, 128), (2, 4, 1, 64), (20, 8, 2, 128), (20, 4, 2, 64), (40, 8, 2, 128), (70, 4, 1, 64)]  # few rows, one and two row tiles


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk,D", KINDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("first,prefix", [(64, 91), (192, 300), (1500, 1700)])  # in either stream's tiles, in units that are cut
def test_a_key_of_the_prefix_that_is_not_a_number_reaches_every_row(first, prefix, bad, rows, Hq, Hk, D, dtype):
    """Sequence b has it b slots behind the first: each place that a slot may have in its group of eight."""
    def spoil(key):
        for b in range(8):
            key[b, first + b, b % Hk, 3] = bad

    # (an infinite number in bf16 gives scores of both signs, row by row; in e4m3 its row is NaN)
    assert _keys(dtype, rows, Hq, Hk, D, [prefix] * 8, spoil) >= (8 if dtype is Q8 or math.isnan(bad) or rows > 2 else 1)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk,D", [(8, 1, 1, 128), (8, 2, 2, 64)] + KINDS[2:])
@pytest.mark.parametrize("prefix", [1, 91, 129])
def test_a_new_key_that_is_not_a_number_reaches_the_rows_that_see_it(prefix, rows, Hq, Hk, D, dtype):
    """Without a prefix the first row may see nothing else."""
    def spoil(key):
        for b in range(8):
            key[b, prefix - 1 + b, 0, 1] = math.nan

    assert _keys(dtype, rows, Hq, Hk, D, [prefix] * 8, spoil) == 8


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("place", range(8))
def test_a_key_of_a_shared_prefix_that_is_not_a_number_reaches_all_sequences(place, dtype):
    def spoil(key):
        key[:, 24 + place, 1, 7] = math.nan

    assert _keys(dtype, 20, 8, 2, 128, [81, 90, 200, 400], spoil, shared=64) == 4


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk,D", [(8, 1, 1, 64), (4, 4, 2, 128), (20, 4, 2, 64), (40, 8, 2, 128)])
@pytest.mark.parametrize("where", [-50, 1])  # in the prefix, the second new row
def test_a_value_that_is_not_a_number_behind_the_smallest_weight(where, rows, Hq, Hk, D, dtype):
    """A weight below fp32's smallest number is 0 there, not in the definition: infinity in its slot's value reaches the rows that see it."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    base, page = 90, 16
    g = _graft(max(2, rows), 1)
    table, n_pages = ref.page_table(np.random.default_rng(1), 1, 10)
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype)
    key, value = (torch.randn((1, base + rows, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    key[:, base + where], value[:, base + where, :, 3] = -60.0, math.inf  # (scores of -200 and less)
    q = torch.randn((1, rows, Hq, D), generator=gen, device="cuda").abs().to(BF)
    tb, out = _i32(table), torch.zeros((1, rows, Hq, D), dtype=BF, device="cuda")
    g.cache_write(c, 0, tb, _i32([1]), _i32([base + rows]), key, value)
    g.tree_attention(c, 0, tb, q, _i32([base + 1]), _i32([rows]), None, out)
    assert ((q.float().sum(3) * -60.0 * D ** -0.5) < -200).all()
    first = max(where, 0)
    assert not torch.isfinite(out[0, first:, :, 3]).any() and torch.isfinite(out[0, :first]).all()
    if dtype is BF:  # (a row of e4m3 numbers is NaN as a whole)
        assert torch.isfinite(out[..., 4:]).all()
