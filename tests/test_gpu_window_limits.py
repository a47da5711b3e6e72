"""Rotated appends and attention with a window where their plans and addresses change form: many sequences, many blocks of rows, caches
beyond 32 bits of bytes, graphs that share a context, windows beyond 32 bits."""
import numpy as np
import pytest
import torch

import verifier_ref as ref
from test_gpu_verifier import BF, Q8, _cache, _graft, _i32
from test_gpu_window import BAD_CACHE, _append, _attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B", [191, 192, 193, 256, 257, 600])  # with a launch for their plan from 193 on, that is not held on the chip from 513 on
def test_many_single_tokens(dtype, B):
    lens, counts = [1 + 7 * i % 190 for i in range(B)], [int(i % 11 != 3) for i in range(B)]
    _attend(B, dtype, B, 1, 2, 1, 64, 16, lens, counts, 50, 3, None, calls=2)


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_many_sequences_with_trees(dtype):
    B = 600
    lens, counts = [1 + 7 * i % 190 for i in range(B)], [i % 13 for i in range(B)]
    _attend(B, dtype, B, 12, 2, 1, 64, 16, lens, counts, 50, 3, "tree", calls=2)


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_more_blocks_of_rows_than_a_plan_holds(dtype):
    """64 heads on a key head: blocks of four rows, 275 a sequence; 85 heads: of three, and some sequences without any."""
    _attend(1, dtype, 2, 1100, 64, 1, 64, 16, [1, 40], [1100, 1099], 33, 2, None, calls=2)
    _attend(2, dtype, 70, 25, 85, 1, 64, 16, [1 + i for i in range(70)], [25 * (i % 3) // 2 for i in range(70)], 17, 0, None, calls=2)


def test_many_sequences_appended():
    lens, counts = [1 + 5 * i % 90 for i in range(700)], [i % 4 for i in range(700)]
    for dtype in (BF, Q8):
        _append(1, dtype, 700, 3, 2, 1, 64, 16, lens, counts, rot=64, shift=9)


@pytest.mark.parametrize("B", [3, 300])
@pytest.mark.parametrize("rows", [1, 20])
def test_sequences_left_out_among_many(B, rows):
    """A page that is not there and a length of zero, in both forms of the plan: the others are as without them."""
    gen = torch.Generator(device="cuda").manual_seed(B)
    g = _graft(2, B)
    c = _cache(gen, (1, 5 * B, 1, 16, 64), BF, garbage=False)
    for t in (c.k, c.v):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    table = np.arange(5 * B).reshape(B, 5).astype(np.int32)
    lens = np.array([40 + i % 20 for i in range(B)])
    q = torch.randn((B, rows, 4, 64), generator=gen, device="cuda").to(BF)

    def call(table, lens):
        out, st = torch.full_like(q, 7.0), torch.full((B,), -1, dtype=torch.int32, device="cuda")
        for _ in range(2):
            g.window_attention(c, 0, _i32(table), q, _i32(lens), _i32([rows] * B), None, None, 30, 2, out, status=st)
        return out, st.tolist()

    want, st = call(table, lens)
    assert not any(st)
    table[1, 2], lens[2] = 5 * B, 0
    out, st = call(table, lens)
    assert [b for b in range(B) if st[b]] == [1, 2] and st[1] == st[2] == BAD_CACHE
    assert (out[1:3] == 7.0).all() and torch.equal(out[0], want[0]) and torch.equal(out[3:], want[3:])


@pytest.mark.parametrize("rows", [1, 5, 40])
def test_slots_beyond_32_bits_of_bytes(rows):
    """A cache of over 4 GB, its last pages in use: appends and attention as in a small one."""
    from paper_2608_20375_b200 import KVCache, Rope
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, Hq, Hk, D, page, n_pages = 1, 8, 8, 128, 64, 33000
    g = _graft(2, B)
    shape = (1, n_pages, Hk, page, D)
    large = KVCache(torch.empty(shape, dtype=BF, device="cuda"), torch.empty(shape, dtype=BF, device="cuda"))
    small = KVCache.alloc(1, 4, Hk, page, D)
    key, value = (torch.randn((B, 150, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    outs = []
    for cache, table in ((small, [[0, 1, 2]]), (large, [[n_pages - 1, n_pages - 3, n_pages - 2]])):
        out = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
        g.cache_append(cache, 0, _i32(table), _i32([1]), _i32([150]), Rope.of(D), None, key, value)
        g.window_attention(cache, 0, _i32(table), q, _i32([151 - rows]), _i32([rows]), None, None, 70, 4, out)
        outs.append(out)
    assert torch.equal(*outs) and outs[0].abs().sum() > 0


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_two_graphs_of_one_context_by_turns(dtype):
    """Graphs of few rows whose units are cut at other places, replayed one after another."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    B, Hq, Hk, D, page = 2, 8, 2, 128, 64
    g = _graft(2, B)
    c = _cache(gen, (1, 200, Hk, page, D), dtype, garbage=False)
    tb = torch.arange(200, dtype=torch.int32, device="cuda").view(B, 100)
    key, value = (torch.randn((B, 6000, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    g.cache_write(c, 0, tb, _i32([1] * B), _i32([6000] * B), key, value)
    graphs, outs, wants, kept = [], [], [], []
    for lens, rows in (([6000, 5000], 1), ([70, 5990], 2)):
        q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
        out = torch.zeros_like(q)
        args = (c, 0, tb, q, _i32(lens), _i32([rows] * B), None, None, 3500, 4, out)
        g.window_attention(*args)
        torch.cuda.synchronize()
        wants.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            g.window_attention(*args)
        graphs.append(graph)
        outs.append(out)
        kept.append(args)  # (a graph reads its inputs where they were)
    for _ in range(3):
        for graph, out, want in zip(graphs, outs, wants):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_windows_and_sinks_beyond_32_bits():
    """More than any cache holds is all of it, and does not come round to a small number."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = _graft(2, 1)
    c = _cache(gen, (1, 8, 1, 64, 64), BF, garbage=False)
    for t in (c.k, c.v):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    tb = _i32([list(range(8))])
    from paper_2608_20375_b200 import GraftError
    for rows in (1, 40):
        q = torch.randn((1, rows, 2, 64), generator=gen, device="cuda").to(BF)
        outs = []
        for window, sinks in ((500, 0), (2 ** 32 + 5, 0), (5, 2 ** 32 + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
            out = torch.zeros_like(q)
            g.window_attention(c, 0, tb, q, _i32([400]), _i32([rows]), None, None, window, sinks, out)
            outs.append(out)
        assert all(torch.allclose(outs[0].float(), o.float(), atol=2.0 ** -7) for o in outs[1:])  # (other cuts of the sums: a step of bf16 at 1)
        for window, sinks in ((0, 0), (-2 ** 32 + 5, 0), (5, -1), (5, -2 ** 32)):
            with pytest.raises(GraftError):
                g.window_attention(c, 0, tb, q, _i32([400]), _i32([rows]), None, None, window, sinks, out)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,heads", [(1, 8), (4, 2), (40, 4)])
def test_powers_of_two_go_through(dtype, rows, heads):
    """Queries times 2^a, keys times 2^-a and values times 2^b: the same scores, and the same result times 2^b, bit for bit."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    g = _graft(2, 2)
    n, D = 300, 128
    tb = torch.arange(2 * 6, dtype=torch.int32, device="cuda").view(2, 6)
    key, value = (torch.randn((2, n, 1, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    q = torch.randn((2, rows, heads, D), generator=gen, device="cuda").to(BF)
    q[:, 0, 0, 1:] *= 2.0 ** -20  # (numbers far below a row's largest)
    want = None
    for a, b in ((0, 0), (5, 9), (40, 20), (-40, 100), (75, -60), (-75, 7), (100, -100), (-100, 8)):
        c = _cache(gen, (1, 12, 1, 64, D), dtype, garbage=False)
        g.cache_write(c, 0, tb, _i32([1, 1]), _i32([n, n]), (key.float() * 2.0 ** -a).to(BF), (value.float() * 2.0 ** b).to(BF))
        out, lse = torch.zeros_like(q), torch.zeros((2, rows, heads), device="cuda")
        for call in ("window", "tree"):
            args = c, 0, tb, (q.float() * 2.0 ** a).to(BF), _i32([n + 1 - rows, 100]), _i32([rows, rows])
            if call == "window":
                g.window_attention(*args, None, None, 200, 4, out, lse=lse)
            else:
                g.tree_attention(*args, None, out, lse=lse)
            got = out.float() * 2.0 ** -b, lse.clone()
            if (a, b) == (0, 0):
                want = {**(want or {}), call: got}
            assert torch.equal(got[0], want[call][0]) and torch.equal(got[1], want[call][1]), (call, a, b)
    assert want["window"][0].abs().sum() > 0


@pytest.mark.parametrize("rows,heads", [(1, 8), (4, 2)])
def test_rows_of_queries_that_are_not_numbers(rows, heads):
    """Over e4m3 slots: a query with an infinity or NaN makes its own row NaN and no other; a row of zeros weighs all alike."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    g = _graft(2, 1)
    D, n = 64, 200
    tb = _i32([list(range(4))])
    c = _cache(gen, (1, 4, 1, 64, D), Q8, garbage=False)
    key, value = (torch.randn((1, n, 1, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    g.cache_write(c, 0, tb, _i32([1]), _i32([n]), key, value)
    q = torch.randn((1, rows, heads, D), generator=gen, device="cuda").to(BF)

    def call(q):
        out = torch.zeros_like(q)
        g.window_attention(c, 0, tb, q, _i32([n + 1 - rows]), _i32([rows]), None, None, 90, 3, out)
        return out.flatten(1, 2)[0]

    want = call(q)
    assert torch.isfinite(want).all()
    bad = q.clone().flatten(1, 2)
    bad[0, 1, 5], bad[0, 3, 7], bad[0, 5] = float("inf"), float("nan"), 0.0
    got = call(bad.view_as(q))
    assert got[1].isnan().all() and got[3].isnan().all()
    others = [i for i in range(8) if i not in (1, 3, 5)]
    assert torch.equal(got[others], want[others]) and torch.isfinite(got[5]).all()
