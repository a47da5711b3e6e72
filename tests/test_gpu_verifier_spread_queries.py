"""Queries whose numbers are of very unlike size: what is small in a row counts where the keys have nothing in the large ones' places.  On the
GPU against the plain fp64 form."""
import numpy as np
import pytest
import torch

import verifier_ref as ref
import window_ref as win
from test_gpu_verifier import BF, Q8, _cache, _graft, _i32

pytestmark = pytest.mark.gpu


def _compare(call, dtype, rows, Hq, Hk, D, change, seed=0):
    """One call of chains behind 130 and 300 slots; the queries and keys as `change` left them (places 0 and D - 9 of a key are zero)."""
    lens, page, window, sinks = [131, 301], 16, 90, 5
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    g = _graft(max(2, rows), 2)
    table, n_pages = ref.page_table(rng, 2, -(-(max(lens) + rows) // page))
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype)
    total = max(lens) - 1 + rows
    key, value = (torch.randn((2, total, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    key[..., [0, D - 9]] = 0
    q = torch.randn((2, rows, Hq, D), generator=gen, device="cuda").to(BF)
    change(q, key)
    g.cache_write(c, 0, _i32(table), _i32([1, 1]), _i32([n - 1 + rows for n in lens]), key, value)
    out, lse = torch.zeros((2, rows, Hq, D), dtype=BF, device="cuda"), torch.zeros((2, rows, Hq), device="cuda")
    args = c, 0, _i32(table), q, _i32(lens), _i32([rows, rows])
    if call == "window":
        g.window_attention(*args, None, None, window, sinks, out, lse=lse)
    else:
        g.tree_attention(*args, None, out, lse=lse)
    torch.cuda.synchronize()
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    ke, ve = (None, None) if dtype is BF else (c.k_exp[0].cpu(), c.v_exp[0].cpu())
    for b, n in enumerate(lens):
        slots = np.arange(n - 1 + rows)
        seen = np.stack([win.sees(i, slots, n - 1, rows, None, None, window if call == "window" else 2 ** 30, sinks) for i in range(rows)])
        o, l, tol, ltol = ref.attention(f64(q[b]), ref.entries(c.k[0].cpu(), ke, table[b], slots), ref.entries(c.v[0].cpu(), ve, table[b], slots), seen,
                                        D ** -0.5)
        off, loff = np.abs(f64(out[b]) - o) / tol, np.abs(f64(lse[b]) - l) / ltol
        assert off.max() <= 1 and loff.max() <= 1, (b, off.max(), loff.max())


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("call", ["tree", "window"])
@pytest.mark.parametrize("rows,Hq,Hk,D", [(1, 8, 1, 128), (1, 4, 2, 64), (8, 1, 1, 128), (3, 4, 2, 64), (20, 4, 1, 128)])  # (the last: tiles)
@pytest.mark.parametrize("top", [20, 28, 33, 40, 70, 120])
def test_small_numbers_beside_large_ones(top, rows, Hq, Hk, D, call, dtype):
    """In one row of several, in every second one, in all of them."""
    def one(q, key):
        q[:, -1, -1, 0] = 2.0 ** top

    def some(q, key):
        q[:, :, ::2, D - 9] = -1.5 * 2.0 ** top

    def every(q, key):
        q[..., 0], q[..., D - 9] = 2.0 ** top, 2.0 ** (top - 3)

    for seed, change in enumerate((one, some, every)):
        _compare(call, dtype, rows, Hq, Hk, D, change, seed)


@pytest.mark.parametrize("call", ["tree", "window"])
@pytest.mark.parametrize("rows,Hq,Hk,D", [(1, 8, 1, 128), (3, 4, 2, 64)])
@pytest.mark.parametrize("down", [100, -60])
def test_small_numbers_whose_keys_are_of_another_size(down, rows, Hq, Hk, D, call):
    """The same with the small numbers 2^-down times their size, and keys that bring them back (e4m3 rows' powers of two are far from 1)."""
    def change(q, key):
        q *= 2.0 ** -down
        key *= 2.0 ** down
        q[:, :, ::3, 0] = 2.0 ** (60 if down < 0 else -20)

    _compare(call, Q8, rows, Hq, Hk, D, change)


@pytest.mark.parametrize("rows,Hq,D", [(1, 8, 128), (4, 2, 64)])
def test_rows_beside_one_with_unlike_numbers_keep_their_results(rows, Hq, D):
    """Rows of a call that have no such numbers: within what fp32 sums may differ by, whatever another row of theirs holds."""
    results = []
    for top in (0, 50):
        gen = torch.Generator(device="cuda").manual_seed(5)
        g = _graft(2, 1)
        c = _cache(gen, (1, 8, 1, 64, D), Q8, garbage=False)
        key, value = (torch.randn((1, 400, 1, D), generator=gen, device="cuda").to(BF) for _ in range(2))
        key[..., 0] = 0
        tb = _i32([list(range(8))])
        g.cache_write(c, 0, tb, _i32([1]), _i32([400]), key, value)
        q = torch.randn((1, rows, Hq, D), generator=gen, device="cuda").to(BF)
        q[0, -1, -1, 0] = 2.0 ** top
        out = torch.zeros_like(q)
        g.tree_attention(c, 0, tb, q, _i32([401 - rows]), _i32([rows]), None, out)
        results.append(out.float().flatten(1, 2)[0])
    # (two bf16 results of numbers whose weights differ by a few roundings of a score in fp32: a step of bf16 at most)
    assert ((results[0] - results[1]).abs() <= 2.0 ** -7 * results[0].abs() + 2.0 ** -14)[:-1].all()
