"""Rotated appends to the paged cache and attention with a window, on the GPU against plain fp64 forms."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
import window_ref as win
from test_gpu_verifier import BF, Q8, _cache, _graft, _i32

pytestmark = pytest.mark.gpu
BAD_CACHE = 16


def _f64(t):
    return t.detach().cpu().double().numpy()


# ---- appends -------------------------------------------------------------------------------------------------------
def _append(seed, dtype, B, rows, Hq, Hk, D, page, lens, counts, rot, axes=1, interleaved=False, gain=1.0, position=None, shift=None,
            fused=True, in_place=False, base=10000.0):
    from paper_2608_20375_b200 import Rope
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    g = _graft(max(2, min(rows, 1024)), B)
    width = (max(lens) + rows) // page + 1
    table, n_pages = ref.page_table(rng, B, width)
    c = _cache(gen, (2, n_pages, Hk, page, D), dtype)
    before = [None if t is None else t.clone() for t in (c.k, c.v, c.k_exp, c.v_exp)]
    qkv = torch.randn((B, rows, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(BF)
    q, key, value = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
    if not fused:
        q, key, value = q.contiguous(), key.contiguous(), value.contiguous()
    pairs = rot // 2
    freq = base ** -(np.arange(pairs) / pairs)
    axis = np.arange(pairs) * axes // pairs
    freq = np.where(axis[None] == np.arange(axes)[:, None], freq, 0.0).astype(np.float32)
    pos = None
    if position == "tree":
        pos = rng.integers(0, 3, (B, rows)).cumsum(1) + np.array(lens)[:, None] - 1
    elif position == "axes":
        pos = rng.integers(-5, 100000, (B, rows + 3, axes))
    elif position == "far":
        pos = rng.integers(2 ** 30, 2 ** 31, (B, rows))
    sh = None if shift is None else rng.integers(-shift, shift + 1, B)
    rope = Rope(torch.from_numpy(freq).cuda(), interleaved, gain, None if sh is None else _i32(sh))
    was = qkv.clone()
    out = q if in_place else torch.full((B, rows, Hq, D), 7.0, dtype=BF, device="cuda")
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    g.cache_append(c, 1, _i32(table), _i32(lens), _i32(counts), rope, q, key, value, None if in_place else out,
                   None if pos is None else _i32(pos), st)
    torch.cuda.synchronize()
    assert not st.any()
    x = _f64(was).reshape(B, rows, Hq + 2 * Hk, D)
    touched = np.zeros((n_pages, Hk, page), bool)
    for b in range(B):
        n, at = counts[b], lens[b] - 1 + np.arange(counts[b])
        touched[table[b][at // page], :, at % page] = True
        p = (at[:, None] if pos is None else pos[b, :n].reshape(n, pos[b, 0].size)) + (0 if sh is None else sh[b])
        p = np.broadcast_to(p, (n, axes)) if p.shape[1] == 1 else p
        y, tol = win.turned(x[b, :n, :Hq + Hk], p, freq, interleaved, gain)
        bf = lambda got, want, t: np.all(np.abs(got - want) <= t + 2.0 ** -8 * (np.abs(want) + t))  # noqa: E731
        assert bf(_f64(out)[b, :n], y[:, :Hq], tol[:, :Hq])
        dead = _f64(out)[b, n:]
        assert np.array_equal(dead, x[b, n:, :Hq]) if in_place else (dead == 7.0).all()
        for e, exps, want, t in ((c.k, c.k_exp, y[:, Hq:], tol[:, Hq:]), (c.v, c.v_exp, x[b, :n, Hq + Hk:], np.zeros((n, Hk, D)))):
            got = ref.entries(e[1].cpu(), None if exps is None else exps[1].cpu(), table[b], at)
            if dtype is Q8:
                pg, sl = torch.from_numpy(table[b][at // page]).long(), torch.from_numpy(at % page).long()
                assert win.held_ok(got, exps[1].cpu()[pg, :, sl].numpy(), want, t)
            else:
                assert bf(got, want, t)
                if e is c.v:
                    assert np.array_equal(got, want)
    if not in_place:
        assert torch.equal(qkv, was)
    for t, old in zip((c.k, c.v, c.k_exp, c.v_exp), before):  # everything else is as it was
        if t is not None:
            t, old = (z.view(torch.uint8).cpu().numpy() for z in (t, old))
            assert np.array_equal(t[0], old[0]) and np.array_equal(t[1][~touched], old[1][~touched])


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,kw", [
    (1, 1, 1, 1, 64, 16, [1], [1], dict(rot=64)),
    (1, 1, 32, 8, 128, 64, [5000], [1], dict(rot=128, interleaved=True)),
    (3, 5, 4, 2, 128, 16, [1, 16, 40], [5, 0, 3], dict(rot=64, position="tree")),
    (2, 70, 3, 3, 64, 32, [33, 2], [70, 69], dict(rot=16, axes=2, position="axes", gain=1.25)),
    (2, 130, 8, 8, 128, 128, [127, 1], [130, 1], dict(rot=96, axes=3, position="axes", interleaved=True, shift=1000)),
    (1, 300, 5, 5, 128, 1024, [900], [300], dict(rot=128, shift=7, in_place=True)),
    (2, 33, 7, 1, 64, 16, [1, 9], [33, 20], dict(rot=32, interleaved=True, fused=False, in_place=True)),
    (1, 40, 4, 2, 128, 16, [10], [40], dict(rot=128, position="far")),
    (1, 40, 4, 2, 64, 16, [10], [40], dict(rot=64, position="tree", gain=-0.5, shift=100000)),
    (70, 9, 2, 1, 128, 16, [1 + 3 * i for i in range(70)], [i % 10 for i in range(70)], dict(rot=128)),
])
def test_rows_are_turned_and_written(dtype, B, rows, Hq, Hk, D, page, lens, counts, kw):
    _append(rows + B, dtype, B, rows, Hq, Hk, D, page, lens, counts, **kw)


def test_keys_without_queries_and_position_zero():
    """At position 0 nothing is turned, bit for bit, and the cache is what cache_write makes of the rows; but for the partner of an
    infinity, which is x - inf sin 0 = x - inf 0, not a number."""
    from paper_2608_20375_b200 import Rope
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, rows, Hk, D, page = 2, 21, 3, 128, 16
    g = _graft(2, B)
    key, value = (torch.randn((B, rows, Hk, D), generator=gen, device="cuda").to(BF) * 3 for _ in range(2))
    value[0, 3, 1, 5], value[0, 4, 0, 100], key[1, 2, 2, 127], key[1, 3] = math.nan, math.inf, -math.inf, 0
    tb, pl, cnt = _i32([[3, 0, 1], [5, 2, 4]]), _i32([2, 9]), _i32([21, 17])
    zero = torch.zeros((B, rows), dtype=torch.int32, device="cuda")
    turned = key.clone()
    turned[1, 2, 2, 63] = math.nan
    for dtype in (BF, Q8):
        a, b = (_cache(gen, (1, 6, Hk, page, D), dtype, garbage=False) for _ in range(2))
        g.cache_append(a, 0, tb, pl, cnt, Rope.of(128), None, key, value, position=zero)
        g.cache_write(b, 0, tb, pl, cnt, turned, value)
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k_exp, b.k_exp), (a.v_exp, b.v_exp)):
            if x is not None and x.dtype is BF:
                assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x[~x.isnan()].view(torch.int16), y[~y.isnan()].view(torch.int16))
            else:
                assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_what_is_not_a_number_when_turned():
    """Infinities and NaN reach their pair alone; an e4m3 row with one of them reads back as NaN."""
    from paper_2608_20375_b200 import Rope
    g = _graft(2, 1)
    x = torch.ones((1, 4, 2, 64), dtype=BF, device="cuda")
    x[0, 1, 0, 3], x[0, 2, 1, 40] = math.nan, math.inf
    for dtype in (BF, Q8):
        c = _cache(torch.Generator(device="cuda").manual_seed(0), (1, 1, 2, 16, 64), dtype, garbage=False)
        q = torch.zeros_like(x)
        tb, pl, cnt = _i32([[0]]), _i32([5]), _i32([4])
        g.cache_append(c, 0, tb, pl, cnt, Rope.of(64), x, x, x, q)
        kb, vb = torch.zeros_like(x), torch.zeros_like(x)
        g.cache_read(c, 0, tb, pl, cnt, kb, vb)
        bad = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
        bad[0, 1, 0, [3, 35]] = bad[0, 2, 1, [8, 40]] = True
        assert torch.equal(~torch.isfinite(q), bad)
        rows = bad if dtype is BF else bad.any(-1, keepdim=True).expand(x.shape)
        assert torch.equal(~torch.isfinite(kb), rows)


# ---- attention -----------------------------------------------------------------------------------------------------
def _attend(seed, dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, mask=None, scale=None, spoil=None, want_lse=True, nmax=None,
            positions=None, calls=1):
    """One call against the plain form.  What no row sees is garbage: pages that hold nothing else are not in the table."""
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    nmax = max(2, rows) if nmax is None else nmax
    g = _graft(nmax if mask is not None else 2, B)
    width = -(-(max(lens) - 1 + rows) // page) + 1
    table, n_pages = ref.page_table(rng, B, width)
    c = _cache(gen, (2, n_pages, Hk, page, D), dtype)
    total = [lens[b] - 1 + counts[b] for b in range(B)]
    most = max(1, max(total))
    k = torch.randn((B, most, Hk, D), generator=gen, device="cuda").to(BF)
    v = torch.randn((B, most, Hk, D), generator=gen, device="cuda").to(BF)
    if spoil is not None:
        spoil(k, v)
    g.cache_write(c, 1, _i32(table), _i32([1] * B), _i32(total), k, v)
    layer = [None if t is None else t[1].cpu() for t in (c.k, c.v, c.k_exp, c.v_exp)]
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    m = pos = None
    if mask is not None:
        W = (nmax + 31) // 32
        m, pos = np.zeros((B, nmax, W), np.int32), np.full((B, nmax), -1, np.int32)
        for b in range(B):
            depth, bits = ref.tree(rng, counts[b], nmax)[1:]
            m[b] = bits
            pos[b] = np.where(depth < 0, -1, lens[b] - 1 + depth)
            if mask == "random":
                m[b] = rng.integers(-2 ** 31, 2 ** 31, (nmax, W)) & rng.integers(-2 ** 31, 2 ** 31, (nmax, W))
            if mask == "empty":
                m[b] = 0
            if positions == "junk":
                pos[b] = rng.integers(-2 ** 31, 2 ** 31, nmax)
            elif positions == "chain":  # (a tree that is one long path)
                m[b] = 0
                for i in range(counts[b]):
                    for j in range(i + 1):
                        m[b, i].view(np.uint32)[j // 32] |= np.uint32(1 << (j % 32))
                pos[b] = lens[b] - 1 + np.arange(nmax)
    # what the call may look at
    tb = table.copy()
    for b in range(B):
        base, end = lens[b] - 1, total[b]
        lo = max(0, base - window + 1)
        for i in range(width):
            s = np.arange(i * page, (i + 1) * page)
            live = (s < end) & ((s < sinks) | (s >= lo)) if counts[b] else np.zeros(page, bool)
            if not live.any():
                tb[b, i] = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31])
            dead = torch.from_numpy(np.nonzero(~live)[0]).cuda()
            for t in (c.k, c.v, c.k_exp, c.v_exp):
                if t is not None:
                    t[1, int(table[b, i])][:, dead] = torch.full((), 0xFF, dtype=torch.uint8, device="cuda") if t.dtype is torch.uint8 else math.nan
    out = torch.full((B, rows, Hq, D), 7.0, dtype=BF, device="cuda")
    lse = torch.full((B, rows, Hq), 7.0, device="cuda") if want_lse else None
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    args = (c, 1, _i32(tb), q, _i32(lens), _i32(counts), None if m is None else _i32(m), None if pos is None else _i32(pos), window, sinks)
    first = None
    for _ in range(calls):
        g.window_attention(*args, out, lse=lse, scale=scale, status=st)
        torch.cuda.synchronize()
        assert not st.any()
        assert first is None or torch.equal(first.view(torch.int16), out.view(torch.int16))  # (NaN among it: bit for bit)
        first = out.clone()
    scale = D ** -0.5 if scale is None else scale
    for b in range(B):
        n, base = counts[b], lens[b] - 1
        lo = max(0, base - window + 1)
        assert (out[b, n:] == 7.0).all() and (lse is None or (lse[b, n:] == 7.0).all())
        if not n:
            continue
        slots = np.concatenate([np.arange(min(sinks, lo)), np.arange(lo, total[b])])
        ke = ref.entries(layer[0], layer[2], table[b], slots)
        ve = ref.entries(layer[1], layer[3], table[b], slots)
        seen = np.stack([win.sees(i, slots, base, n, None if pos is None else pos[b], None if m is None else ref.bits(m[b], nmax)[i], window, sinks)
                         for i in range(n)])
        o, l, tol, ltol = ref.attention(_f64(q[b, :n]), ke, ve, seen, scale)
        got = _f64(out[b, :n])
        assert np.array_equal(np.isnan(got), np.isnan(o)), f"sequence {b}: NaN elsewhere"
        fine = np.isfinite(o)
        off = np.abs(got - o)[fine] / tol[fine]
        assert fine.sum() == 0 or off.max() <= 1, f"sequence {b}: {off.max()} of the tolerance"
        assert np.array_equal(got[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)])
        if lse is not None:
            gl = _f64(lse[b, :n])
            ok = np.isfinite(l)
            assert np.array_equal(gl[~ok], l[~ok]) and (np.abs(gl - l)[ok] <= ltol[ok]).all()


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,window,sinks,mask", [
    (1, 1, 1, 1, 64, 16, [1], [1], 1, 0, None),               # one token sees itself
    (1, 1, 4, 1, 128, 16, [200], [1], 16, 4, None),
    (1, 1, 8, 1, 128, 64, [3000], [1], 1000, 4, None),
    (4, 1, 8, 2, 128, 64, [1, 100, 900, 5000], [1, 1, 0, 1], 257, 20, None),
    (3, 1, 4, 4, 64, 128, [10, 129, 700], [1, 1, 1], 100, 300, None),  # sinks beyond the window, and beyond the prefix
    (2, 1, 7, 1, 128, 1024, [2050, 5], [1, 1], 1000, 1, None),
    (2, 2, 8, 2, 64, 32, [77, 300], [2, 1], 40, 33, "tree"),
    (3, 8, 2, 2, 128, 16, [1, 50, 333], [8, 5, 0], 3, 2, "tree"),      # a window shorter than the trees are deep
    (2, 8, 8, 8, 64, 16, [1, 50], [8, 8], 5, 0, None),
])
def test_few_rows(dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, mask):
    _attend(B + rows + window, dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, mask, calls=2)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,window,sinks,mask", [
    (1, 65, 4, 1, 128, 64, [1500], [65], 512, 4, "tree"),
    (3, 40, 8, 2, 128, 16, [1, 100, 700], [40, 17, 40], 100, 4, "tree"),
    (2, 30, 4, 4, 64, 32, [500, 20], [30, 30], 2, 1, "tree"),          # shorter than the trees are deep
    (2, 200, 2, 1, 128, 128, [300, 2000], [200, 111], 700, 130, "tree"),
    (2, 150, 8, 2, 64, 64, [300, 900], [150, 64], 64, 0, "tree"),
    (4, 33, 5, 1, 128, 16, [1, 2, 64, 3000], [33, 0, 32, 33], 1024, 4, "random"),
    (2, 70, 4, 2, 128, 16, [50, 400], [70, 70], 30, 0, "random"),
    (2, 400, 4, 4, 64, 64, [900, 1], [400, 399], 300, 7, "random"),
])
def test_trees(dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, mask):
    _attend(B + rows + window, dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, mask, calls=2)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,window,sinks", [
    (1, 300, 4, 1, 128, 64, [1], [300], 64, 4),
    (2, 300, 8, 2, 64, 16, [1, 1000], [300, 257], 100, 0),
    (3, 700, 7, 1, 128, 32, [1, 40, 300], [700, 1, 0], 257, 5),        # blocks of 36 rows
    (2, 200, 3, 3, 128, 128, [1, 129], [200, 130], 1, 0),              # every row sees itself alone
    (1, 200, 2, 1, 64, 64, [700], [200], 1, 3),
    (2, 100, 4, 4, 128, 64, [513, 100], [100, 100], 4096, 4),          # a window beyond all there is
    (1, 3, 300, 1, 64, 16, [90], [3], 33, 2),                          # more heads on a key head than a unit has rows
    (1, 600, 1, 1, 128, 1024, [1500], [600], 400, 129),
    (1, 1100, 4, 2, 64, 16, [10], [1100], 33, 17),
])
def test_chunks_of_prompts(dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks):
    _attend(B + rows + window, dtype, B, rows, Hq, Hk, D, page, lens, counts, window, sinks, None, calls=2)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk", [(4, 2, 2), (60, 4, 2), (200, 4, 2)])
def test_rows_that_see_nothing_and_positions_that_no_tree_has(dtype, rows, Hq, Hk):
    """Masks that are empty with a window that leaves nothing of the prefix; positions that are held to what a tree can have."""
    _attend(3, dtype, 2, rows, Hq, Hk, 64, 16, [40, 300], [rows, rows - 1], 1, 0, "empty")
    _attend(4, dtype, 2, rows, Hq, Hk, 64, 16, [40, 300], [rows, rows - 1], 50, 2, "empty")
    _attend(5, dtype, 2, rows, Hq, Hk, 128, 32, [40, 300], [rows, rows - 1], 90, 4, "random", positions="junk")
    _attend(6, dtype, 2, rows, Hq, Hk, 64, 16, [1, 200], [rows, rows // 2], 3, 0, "tree", positions="chain")
    _attend(7, dtype, 2, rows, Hq, Hk, 64, 16, [1, 200], [rows, rows // 2], 20, 8, "tree", positions="chain")


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,Hq,Hk,mask", [(1, 8, 2, None), (4, 2, 1, "tree"), (30, 8, 2, "tree"), (200, 4, 2, "tree"), (300, 4, 2, None)])
def test_what_is_not_a_number_reaches_those_that_see_it(dtype, rows, Hq, Hk, mask):
    """V (and K) at the window's border, among sinks and new rows: rows that see it get it, the others do not."""
    lens, window, sinks = [500, 90], 130, 5

    def spoil(k, v):
        for s in (2, 4, 371, 372, 499, 88, 95, 380):
            if s < v.shape[1]:
                v[:, s, 0, s % 7] = math.nan if s % 2 else math.inf

    _attend(11, dtype, 2, rows, Hq, Hk, 64, 16, lens, [rows, max(1, rows - 1)], window, sinks, mask, spoil=spoil)
    _attend(12, dtype, 2, rows, Hq, Hk, 128, 64, lens, [rows, max(1, rows - 1)], window, sinks, mask, spoil=spoil)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows", [1, 50])
def test_other_scales_and_no_lse(dtype, rows):
    for scale in (0.0, -0.2, 1.5):
        _attend(21, dtype, 2, rows, 4, 2, 64, 16, [300, 40], [rows, rows], 100, 4, "tree" if rows > 1 else None, scale=scale, want_lse=scale > 0)


def test_a_window_without_an_end_is_tree_attention():
    gen = torch.Generator(device="cuda").manual_seed(3)
    for B, rows, mask in ((3, 1, False), (3, 40, True), (2, 300, False)):
        g = _graft(max(2, rows), B)
        c = _cache(gen, (1, 64 * B, 2, 16, 64), BF, garbage=False)
        c.k.copy_(torch.randn(c.k.shape, generator=gen, device="cuda")), c.v.copy_(torch.randn(c.v.shape, generator=gen, device="cuda"))
        tb = torch.arange(64 * B, dtype=torch.int32, device="cuda").view(B, 64)
        lens, counts = [700, 30, 5][:B], [rows, max(1, rows - 3), rows][:B]
        q = torch.randn((B, rows, 4, 64), generator=gen, device="cuda").to(BF)
        m = pos = None
        if mask:
            t = [ref.tree(np.random.default_rng(b), counts[b], g.nmax) for b in range(B)]
            m = _i32(np.stack([x[2] for x in t]))
            pos = _i32(np.stack([x[1] for x in t]) + np.array(lens)[:, None] - 1)
        a, b, la, lb = (torch.zeros((B, rows, 4, 64), dtype=BF, device="cuda") for _ in range(2)), None, None, None
        a, b = a
        la, lb = (torch.zeros((B, rows, 4), device="cuda") for _ in range(2))
        g.tree_attention(c, 0, tb, q, _i32(lens), _i32(counts), m, a, lse=la)
        g.window_attention(c, 0, tb, q, _i32(lens), _i32(counts), m, pos, 2 ** 31 - 1, 0, b, lse=lb)
        # each is within its own roundings of the same numbers: a weight's and the result's
        assert ((a.float() - b.float()).abs() <= 2.0 ** -6 * (a.float().abs() + 0.25)).all()
        assert ((la - lb).abs() <= 1e-5 * (1 + la.abs())).all()


def test_bad_pages_and_counts_leave_a_sequence_out():
    """Host numbers that the kernels look at before they use them; pages that nothing sees are not looked at."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    from paper_2608_20375_b200 import Rope
    B, Hk, D, page, rows = 7, 2, 64, 16, 6
    for dtype in (BF, Q8):
        for r, heads in ((rows, 2), (rows, 16)):
            g = _graft(rows, B)
            c = _cache(gen, (1, 40, Hk, page, D), dtype, garbage=False)
            table = np.arange(40)[: B * 5].reshape(B, 5).astype(np.int32)
            table[0, 1] = -1           # between the sinks and the window
            table[1, 0] = 40           # the sinks' page
            table[2, 3] = -1           # the window's
            table[3, 4] = 99           # behind the rows
            lens, counts = [60, 60, 60, 50, 0, 60, 78], [6, 6, 6, 6, 1, 7, 6]
            want = [0, BAD_CACHE, BAD_CACHE, 0, BAD_CACHE, BAD_CACHE, BAD_CACHE]
            q = torch.randn((B, r, heads, D), generator=gen, device="cuda").to(BF)
            out, st = torch.full_like(q, 7.0), torch.full((B,), -1, dtype=torch.int32, device="cuda")
            g.window_attention(c, 0, _i32(table), q, _i32(lens), _i32(counts), None, None, 20, 3, out, status=st)
            assert st.tolist() == want
            assert [bool((out[b] == 7.0).all()) for b in range(B)] == [w != 0 for w in want]
            # of an append, only the new rows' pages
            key = torch.randn((B, r, Hk, D), generator=gen, device="cuda").to(BF)
            qo = torch.full_like(q, 7.0)
            k0 = c.k.clone()
            g.cache_append(c, 0, _i32(table), _i32(lens), _i32(counts), Rope.of(64), q, key, key, qo, status=st)
            want = [0, 0, BAD_CACHE, 0, BAD_CACHE, BAD_CACHE, BAD_CACHE]
            assert st.tolist() == want
            assert [bool((qo[b] == 7.0).all()) for b in range(B)] == [w != 0 for w in want]
            for b in range(B):
                pages = torch.tensor([x for x in table[b] if 0 <= x < 40], device="cuda")
                same = torch.equal(c.k[0, pages].view(torch.uint8), k0[0, pages].view(torch.uint8))
                assert same == (want[b] != 0)


def test_captured_and_on_another_stream():
    """A layer captured into a graph and replayed with other inputs in its buffers; calls of other shapes between, on the same context."""
    from paper_2608_20375_b200 import Rope
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, rows, Hq, Hk, D, page = 3, 20, 8, 2, 64, 16
    for dtype in (BF, Q8):
        g = _graft(rows, B)
        c = _cache(gen, (1, 200, Hk, page, D), dtype, garbage=False)
        tb = torch.arange(200, dtype=torch.int32, device="cuda")[:B * 60].view(B, 60)
        rope = Rope.of(64)
        t = [ref.tree(np.random.default_rng(b), rows, g.nmax) for b in range(B)]
        m, depth = _i32(np.stack([x[2] for x in t])), _i32(np.stack([x[1] for x in t]))
        lens, cnt = _i32([300, 7, 800]), _i32([20, 20, 11])
        q, key, value = (torch.randn((B, rows, h, D), generator=gen, device="cuda").to(BF) for h in (Hq, Hk, Hk))
        pos = depth + lens[:, None] - 1
        qr, out = torch.zeros_like(q), torch.zeros_like(q)

        def layer(qr, out):
            g.cache_append(c, 0, tb, lens, cnt, rope, q, key, value, qr, position=pos)
            g.window_attention(c, 0, tb, qr, lens, cnt, m, pos, 100, 4, out)

        def other():  # more scratch than the captured call needed
            x = torch.zeros((B, 300, Hq, D), dtype=BF, device="cuda")
            g.window_attention(c, 0, tb, x, _i32([1, 1, 1]), _i32([300, 300, 300]), None, None, 64, 0, torch.empty_like(x))

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            layer(qr, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(qr, out)
        for _ in range(3):
            for x in (q, key, value):
                x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            other()
            qr.zero_(), out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            a, b = torch.zeros_like(q), torch.zeros_like(q)
            got = qr.clone(), out.clone()
            layer(a, b)
            torch.cuda.synchronize()
            assert torch.equal(got[0], a) and torch.equal(got[1], b)
