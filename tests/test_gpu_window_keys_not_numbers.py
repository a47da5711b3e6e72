"""Keys that are not numbers at a window's border, among sinks and new rows: rows that see their slot are NaN, the others as if it held a number."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
import window_ref as win
from test_gpu_verifier import BF, Q8, _cache, _graft, _i32
from test_gpu_verifier_not_numbers import _expect

pytestmark = pytest.mark.gpu


def _keys(dtype, rows, Hq, Hk, D, page, mask, bad, places, seed):
    """Sequence b has a key that is `bad` in slot places[b] alone: out and lse against the definition's; rows that are NaN."""
    prefix, window, sinks = 400, 130, 5
    B = len(places)
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    g = _graft(max(2, rows), B)
    table, n_pages = ref.page_table(rng, B, -(-(prefix + rows) // page))
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype)
    key, value = (torch.randn((B, prefix + rows, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    for b, s in enumerate(places):
        key[b, s, b % Hk, 3 + b] = bad
    g.cache_write(c, 0, _i32(table), _i32([1] * B), _i32([prefix + rows] * B), key, value)
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    m = pos = None
    if mask:
        trees = [ref.tree(rng, rows, g.nmax) for _ in range(B)]
        m, pos = np.stack([t[2] for t in trees]), np.stack([np.where(t[1] < 0, -1, prefix + t[1]) for t in trees])
    out, lse = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda"), torch.zeros((B, rows, Hq), device="cuda")
    g.window_attention(c, 0, _i32(table), q, _i32([prefix + 1] * B), _i32([rows] * B), None if m is None else _i32(m), None if pos is None else _i32(pos),
                       window, sinks, out, lse=lse)
    torch.cuda.synchronize()
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    ke, ve = (None, None) if dtype is BF else (c.k_exp[0].cpu(), c.v_exp[0].cpu())
    lost = []
    for b in range(B):
        slots = np.arange(prefix + rows)
        seen = np.stack([win.sees(i, slots, prefix, rows, None if pos is None else pos[b], None if m is None else ref.bits(m[b], g.nmax)[i], window, sinks)
                         for i in range(rows)])
        wo, wl, tol, ltol = _expect(f64(q[b]), ref.entries(c.k[0].cpu(), ke, table[b], slots), ref.entries(c.v[0].cpu(), ve, table[b], slots), seen,
                                    D ** -0.5)
        o, ls = f64(out[b]), f64(lse[b])
        assert np.array_equal(np.isnan(o), np.isnan(wo)), (b, places[b], np.argwhere(np.isnan(o) != np.isnan(wo))[:5])
        assert np.array_equal(np.isnan(ls), np.isnan(wl)) and np.array_equal(np.isinf(ls), np.isinf(wl))
        fin, lfin = np.isfinite(wo), np.isfinite(wl)
        assert (np.abs(o - wo)[fin] <= tol[fin]).all() and (np.abs(ls - wl)[lfin] <= ltol[lfin]).all()
        group = Hq // Hk
        if math.isnan(bad) or dtype is Q8:  # exactly the rows that see the slot, of its key head
            heads = slice(b % Hk * group, (b % Hk + 1) * group)
            assert np.array_equal(np.isnan(ls[:, heads]), np.broadcast_to(seen[:, places[b], None], (rows, group)))
        lost.append(np.isnan(ls).any())
    return lost


# Slots: a sink, the last one, the first behind them (nobody's), the last that no row sees, and those from the first row's border on.
PLACES = [0, 4, 5, 270, 271, 272, 278, 300, 399, 400]


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rows,Hq,Hk,D,page,mask", [
    (1, 4, 2, 128, 64, False), (1, 8, 1, 64, 16, False), (4, 2, 1, 128, 16, True), (8, 1, 1, 64, 32, False),          # few rows
    (20, 8, 2, 128, 16, True), (30, 4, 1, 64, 64, False), (64, 4, 2, 64, 16, True), (90, 4, 1, 128, 32, False),      # one row tile and two
])
def test_keys_at_the_border_among_sinks_and_new_rows(rows, Hq, Hk, D, page, mask, bad, dtype):
    places = PLACES + [400 + rows // 2, 399 + rows, min(271 + rows // 2, 399)]
    lost = _keys(dtype, rows, Hq, Hk, D, page, mask, bad, places, rows)
    if math.isnan(bad) or dtype is Q8:
        assert lost[0] and lost[1] and not lost[2] and not lost[3]
