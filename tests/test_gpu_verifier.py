"""The verifier's operators on the GPU against plain fp64 forms: the paged cache, attention of trees over it, the sampled walk, the move of
accepted entries, and a round of them together."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref

pytestmark = pytest.mark.gpu

BF, Q8 = torch.bfloat16, torch.float8_e4m3fn


def _graft(nmax=2, batch=8, V=64, L=16):
    from paper_2608_20375_b200 import Graft
    return Graft(V, L, 4, 16, 8, batch, 1, max(1, nmax - 1), 1, 0.0)


def _cache(gen, shape, dtype, garbage=True):
    """A cache full of what an earlier owner of its memory left (NaN among it), or of numbers."""
    from paper_2608_20375_b200 import BF16, E4M3, KVCache
    c = KVCache.alloc(*shape, E4M3 if dtype is Q8 else BF16)
    for t in (c.k, c.v):
        if garbage:
            t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=gen, device="cuda", dtype=torch.uint8))
    if garbage and dtype is Q8:
        for t in (c.k_exp, c.v_exp):
            t.copy_(torch.randint(0, 256, t.shape, generator=gen, device="cuda", dtype=torch.uint8))
    return c


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ---- the cache -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hk,D,page,lens,counts", [
    (1, 1, 1, 64, 16, [1], [1]),
    (3, 5, 2, 128, 16, [1, 16, 40], [5, 0, 3]),
    (2, 70, 3, 64, 32, [33, 2], [70, 69]),
    (2, 130, 8, 128, 128, [127, 1], [130, 1]),
    (1, 300, 5, 128, 1024, [900], [300]),
])
def test_cache_rows_are_written_and_read_back(dtype, B, rows, Hk, D, page, lens, counts):
    rng, gen = np.random.default_rng(rows), torch.Generator(device="cuda").manual_seed(rows)
    g = _graft(batch=B)
    width = (max(lens) + rows) // page + 1
    table, n_pages = ref.page_table(rng, B, width)
    c = _cache(gen, (2, n_pages, Hk, page, D), dtype)
    before = [None if t is None else t.clone() for t in (c.k, c.v, c.k_exp, c.v_exp)]
    # numbers of all sizes, rows of zeros, rows with one NaN or infinity
    key = torch.randn((B, rows, Hk, D), generator=gen, device="cuda") * torch.logspace(-38, 37, rows * Hk, device="cuda").view(rows, Hk, 1)
    value = torch.randn((B, rows, Hk, D), generator=gen, device="cuda")
    key, value = key.to(BF), value.to(BF)
    if rows > 3:
        value[0, 1], value[0, 2, 0, 7], value[0, 3, -1, 5] = 0, math.nan, -math.inf
    tb, pl, cnt, st = _i32(table), _i32(lens), _i32(counts), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    g.cache_write(c, 1, tb, pl, cnt, key, value, st)
    kb, vb = torch.full_like(key, 7.0), torch.full_like(value, 7.0)
    st2 = torch.full_like(st, -1)
    g.cache_read(c, 1, tb, pl, cnt, kb, vb, st2)
    torch.cuda.synchronize()
    assert not st.any() and not st2.any()
    alive = np.arange(rows)[None, :] < np.array(counts)[:, None]
    touched = np.zeros((n_pages, Hk, page), bool)
    for b in range(B):
        s = lens[b] - 1 + np.arange(counts[b])
        touched[table[b][s // page], :, s % page] = True
    for x, back in ((key, kb), (value, vb)):
        x, back = x.cpu().double().numpy(), back.cpu().double().numpy()
        want = ref.quantise_rows(x)[0] if dtype is Q8 else x
        with np.errstate(over="ignore"):
            want = torch.from_numpy(want).to(BF).double().numpy()  # (above bf16's largest: infinity, on both sides)
        assert np.array_equal(back[alive], want[alive], equal_nan=True)
        assert (back[~alive] == 7.0).all()
    for t, old in zip((c.k, c.v, c.k_exp, c.v_exp), before):  # everything else is as it was
        if t is not None:
            t, old = (x.view(torch.uint8).cpu().numpy() for x in (t, old))
            assert np.array_equal(t[0], old[0]) and np.array_equal(t[1][~touched], old[1][~touched])


def test_rows_of_a_fused_projection_are_taken_where_they_stand():
    gen = torch.Generator(device="cuda").manual_seed(5)
    B, rows, Hq, Hk, D, page = 2, 9, 6, 2, 64, 16
    g = _graft(rows, B)
    qkv = torch.randn((B, rows, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(BF)
    q, key, value = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
    out = []
    for dense in (False, True):
        c = _cache(gen, (1, 8, Hk, page, D), BF)
        tb, pl, cnt = _i32([[0, 1], [2, 3]]), _i32([1, 7]), _i32([9, 4])
        o = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
        a = (lambda t: t.contiguous()) if dense else (lambda t: t)
        c.k.fill_(0.5), c.v.fill_(0.25)
        g.cache_write(c, 0, tb, pl, cnt, a(key), a(value))
        g.tree_attention(c, 0, tb, a(q), pl, cnt, None, o)
        out.append((c.k.clone(), c.v.clone(), o))
    for x, y in zip(*out):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,layers,Hk,D,page,in_place", [(1, 1, 1, 64, 16, False), (5, 3, 4, 128, 64, True), (40, 2, 2, 64, 16, True)])
def test_accepted_entries_move_up(dtype, B, layers, Hk, D, page, in_place):
    rng, gen = np.random.default_rng(B), torch.Generator(device="cuda").manual_seed(B)
    L, nodes = 16, 50
    g = _graft(nodes, B, L=L)
    lens = rng.integers(1, 60, B)
    width = (60 + nodes) // page + 1
    table, n_pages = ref.page_table(rng, B, width)
    c = _cache(gen, (layers, n_pages, Hk, page, D), dtype)
    alen = rng.integers(0, L + 1, B)
    alen[0] = L
    path = np.full((B, L), -1, np.int32)
    for b in range(B):
        path[b, :alen[b]] = np.sort(rng.choice(np.arange(1, nodes), alen[b], replace=False))
    path[0] = np.arange(2, L + 2)  # every entry moves into the one before it
    want = [None if t is None else t.clone().cpu().view(torch.uint8).numpy() for t in (c.k, c.v, c.k_exp, c.v_exp)]
    for b in range(B):
        src, dst = lens[b] - 1 + path[b, :alen[b]], lens[b] + np.arange(alen[b])
        for t in want:
            if t is not None:
                t[:, table[b][dst // page], :, dst % page] = t[:, table[b][src // page], :, src % page]
    pl, st = _i32(lens), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    nxt = pl if in_place else torch.zeros_like(pl)
    g.cache_keep(c, _i32(table), pl, _i32(alen), _i32(path), nxt, st)
    torch.cuda.synchronize()
    assert not st.any() and np.array_equal(nxt.cpu().numpy(), lens + alen + 1)
    for t, w in zip((c.k, c.v, c.k_exp, c.v_exp), want):
        if t is not None:
            assert np.array_equal(t.view(torch.uint8).cpu().numpy(), w)


def test_bad_pages_and_counts_leave_a_sequence_out():
    """Table entries outside the cache, slots behind the table, counts and lengths out of range: host numbers that the kernels look at before
    they use them.  The sequence is reported and left alone; the others are served."""
    rng, gen = np.random.default_rng(2), torch.Generator(device="cuda").manual_seed(2)
    B, rows, Hq, Hk, D, page, width, L = 9, 20, 4, 2, 64, 16, 4, 16
    g = _graft(rows, B, L=L)
    table, n_pages = ref.page_table(rng, B, width)
    lens, counts = np.full(B, 30), np.full(B, 17)
    table[1, 2] = n_pages      # page behind the cache, in use
    table[2, 1] = -1           # page in front of it
    lens[3] = 49               # slots 48 .. 64, the last behind the table
    lens[4] = 0                # no root
    counts[5] = rows + 1
    counts[6] = -1
    table[7, 3] = 1 << 30      # not in use: fine
    bad = np.isin(np.arange(B), [1, 2, 3, 4, 5, 6])
    c = _cache(gen, (1, n_pages, Hk, page, D), BF, garbage=False)
    tb, pl, cnt = _i32(table), _i32(lens), _i32(counts)
    key, value = (torch.randn((B, rows, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    want_st = np.where(bad, 16, 0)
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    g.cache_write(c, 0, tb, pl, cnt, key, value, st)
    assert np.array_equal(st.cpu().numpy(), want_st)
    kb, vb = torch.full_like(key, 7.0), torch.full_like(value, 7.0)
    g.cache_read(c, 0, tb, pl, cnt, kb, vb, st)
    assert np.array_equal(st.cpu().numpy(), want_st)
    assert torch.equal(kb[~torch.from_numpy(bad)][:, :17], key[~torch.from_numpy(bad)][:, :17]) and (kb[torch.from_numpy(bad)] == 7.0).all()
    out = torch.full((B, rows, Hq, D), 7.0, dtype=BF, device="cuda")
    lse = torch.full((B, rows, Hq), 7.0, device="cuda")
    g.tree_attention(c, 0, tb, q, pl, cnt, None, out, lse, status=st)
    assert np.array_equal(st.cpu().numpy(), want_st)
    assert (out.cpu()[torch.from_numpy(bad)] == 7.0).all() and (lse.cpu()[torch.from_numpy(bad)] == 7.0).all()
    assert torch.isfinite(out).all() and (lse.cpu()[torch.from_numpy(~bad)][:, :17] != 7.0).all()
    # moves: a page outside, an accepted length out of range, a node in front of the root, a path that ends behind the table
    path = np.tile(np.arange(1, L + 1, dtype=np.int32), (B, 1))
    alen = np.full(B, 2)
    table2 = table.copy()
    table2[7, 3] = 0
    path[0, 1] = -1
    alen[7], alen[8] = L + 1, -1
    path[3, 1] = 16
    kept = c.k.clone()
    nxt = torch.zeros_like(pl)
    g.cache_keep(c, _i32(table2), pl, _i32(alen), _i32(path), nxt, st)
    bad2 = np.isin(np.arange(B), [0, 2, 3, 4, 7, 8])  # (1: its bad page holds none of the slots that move)
    assert np.array_equal(st.cpu().numpy(), np.where(bad2, 16, 0))
    assert np.array_equal(nxt.cpu().numpy(), np.where(bad2, lens, lens + alen + 1))
    assert torch.equal(c.k, kept)  # (nodes 1 and 2 stand where they belong)


# ---- attention -----------------------------------------------------------------------------------------------------
def _attend(seed, B, rows, Hq, Hk, D, page, lens, counts, dtype, mask="tree", shared=0, scale=None, spoil=None, nmax=None, want_lse=True):
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    nmax = nmax or max(2, rows)
    g = _graft(nmax, B)
    width = -(-(max(lens) - 1 + rows) // page)
    table, n_pages = ref.page_table(rng, B, width, shared_pages=shared // page)
    c = _cache(gen, (2, n_pages, Hk, page, D), dtype)  # garbage wherever no sequence has an entry
    tb, cnt = _i32(table), _i32(counts)
    # the whole sequence goes in as a prompt: prefix and new rows
    total = max(n + s - 1 for n, s in zip(counts, lens))
    if total:
        key = torch.randn((B, total, Hk, D), generator=gen, device="cuda").to(BF)
        value = torch.randn((B, total, Hk, D), generator=gen, device="cuda").to(BF)
        if shared:
            key[:, :shared], value[:, :shared] = key[:1, :shared], value[:1, :shared]
        if spoil:
            spoil(key, value)
        ends = _i32([n + s - 1 for n, s in zip(counts, lens)])
        g.cache_write(c, 1, tb, _i32([1] * B), ends, key, value)
    pl = _i32(lens)
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    m = None
    if mask is not None:
        W = g.mask_words
        m = np.zeros((B, nmax, W), np.int32)
        for b in range(B):
            if mask == "tree":
                m[b] = ref.tree(rng, counts[b], nmax)[2]
            elif mask == "random":
                m[b] = rng.integers(-2 ** 31, 2 ** 31, (nmax, W))  # bits of rows behind the count too
                m[b, ::3] = 0
            else:
                assert mask == "empty"
    out = torch.full((B, rows, Hq, D), 7.0, dtype=BF, device="cuda")
    lse = torch.full((B, rows, Hq), 7.0, device="cuda") if want_lse else None
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    g.tree_attention(c, 1, tb, q, pl, cnt, None if m is None else _i32(m), out, lse, scale=scale, shared=shared, status=st)
    torch.cuda.synchronize()
    assert not st.any()
    o, ls = out.cpu().double().numpy(), None if lse is None else lse.cpu().double().numpy()
    k1, v1 = c.k[1].cpu(), c.v[1].cpu()
    ke, ve = (None, None) if dtype is BF else (c.k_exp[1].cpu(), c.v_exp[1].cpu())
    for b in range(B):
        n, base = counts[b], lens[b] - 1
        assert (o[b, n:] == 7.0).all() and (ls is None or (ls[b, n:] == 7.0).all())
        if n == 0:
            continue
        slots = np.arange(base + n)
        k, v = ref.entries(k1, ke, table[b], slots), ref.entries(v1, ve, table[b], slots)
        seen = np.ones((n, base + n), bool)
        seen[:, base:] = np.tril(np.ones((n, n), bool)) if m is None else ref.bits(m[b, :n], nmax)[:, :n]
        wo, wl, tol, ltol = ref.attention(q[b, :n].cpu().double().numpy(), k, v, seen, D ** -0.5 if scale is None else scale)
        fin = np.isfinite(wo)
        assert np.array_equal(np.isnan(wo), np.isnan(o[b, :n])) and np.array_equal(wo[~fin & ~np.isnan(wo)], o[b, :n][~fin & ~np.isnan(wo)])
        off = np.abs(o[b, :n] - wo)[fin] - tol[fin]
        assert off.max(initial=-1) <= 0, (b, off.max(), np.argwhere(np.abs(o[b, :n] - wo) > tol)[:5])
        if ls is not None:
            inf = np.isinf(wl)
            assert np.array_equal(np.isinf(ls[b, :n]), inf)
            assert (np.abs(ls[b, :n] - wl)[~inf] <= ltol[~inf]).all(), np.abs(ls[b, :n] - wl)[~inf].max()
    return out


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,lens,counts,mask", [
    (1, 1, 1, 1, 64, 16, [1], [1], None),                                  # one token, nothing before it
    (1, 1, 8, 2, 128, 64, [700], [1], None),                               # one token
    (4, 1, 32, 8, 128, 64, [1, 128, 129, 1000], [1, 1, 1, 1], None),       # the last slot ends, begins a tile
    (2, 3, 4, 4, 64, 16, [127, 126], [3, 2], "tree"),
    (3, 65, 32, 8, 128, 64, [300, 1, 64], [65, 65, 40], "tree"),
    (3, 40, 28, 4, 64, 16, [513, 77, 1], [0, 40, 39], "tree"),             # a group of seven, a sequence without rows
    (2, 40, 5, 1, 128, 32, [250, 90], [40, 33], "random"),                 # groups of five, bits of slots that are not there
    (2, 37, 4, 1, 128, 128, [1, 200], [37, 30], "empty"),                  # a sequence whose rows see nothing
    (2, 300, 8, 2, 128, 64, [400, 129], [300, 257], "tree"),               # several row tiles
    (1, 513, 4, 2, 64, 1024, [900], [513], "tree"),
    (2, 260, 2, 2, 128, 16, [1, 100], [260, 200], None),                   # a prompt, a chunk of one
    (1, 7, 16, 1, 128, 64, [3000], [7], "tree"),                           # few rows, long prefix: split and joined
    (9, 20, 8, 8, 128, 16, [16, 17, 31, 32, 33, 255, 256, 257, 511], [20, 1, 2, 3, 16, 17, 18, 19, 20], "tree"),
])
def test_attention(dtype, B, rows, Hq, Hk, D, page, lens, counts, mask):
    _attend(7 * rows + B, B, rows, Hq, Hk, D, page, lens, counts, dtype, mask)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("B,rows,Hq,Hk,D,page,shared,lens,counts,mask", [
    (3, 1, 8, 2, 128, 64, 256, [257, 300, 500], [1, 1, 1], None),
    (5, 17, 32, 4, 128, 64, 128, [129, 140, 129, 400, 200], [17, 1, 0, 16, 9], "tree"),
    (2, 70, 7, 1, 64, 16, 48, [49, 80], [70, 61], "tree"),
    (40, 9, 4, 2, 64, 32, 320, [321 + i for i in range(40)], [1 + i % 9 for i in range(40)], "random"),
    (4, 200, 4, 2, 128, 64, 512, [513, 600, 700, 513], [200, 150, 0, 3], None),
])
def test_attention_behind_a_shared_prefix(dtype, B, rows, Hq, Hk, D, page, shared, lens, counts, mask):
    _attend(rows + B, B, rows, Hq, Hk, D, page, lens, counts, dtype, mask, shared=shared)


def test_sequences_behind_their_shared_prefix_only():
    """prefix_len must be above `shared`: the sequence that is not is left out, the others are served."""
    B, rows, Hq, Hk, D, page = 3, 4, 2, 1, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = _graft(rows, B)
    c = _cache(gen, (1, 16, Hk, page, D), BF, garbage=False)
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    out, st = torch.full_like(q, 7.0), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    g.tree_attention(c, 0, _i32([[0, 1, 2, 3], [0, 1, 4, 5], [0, 1, 6, 7]]), q, _i32([33, 32, 40]), _i32([4, 4, 4]), None, out, shared=32,
                     status=st)
    assert st.tolist() == [0, 16, 0]
    assert (out[1] == 7.0).all() and (out[0] == 0).all() and (out[2] == 0).all()


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_attention_without_lse_other_scales_and_sharp_scores(dtype):
    _attend(1, 2, 12, 4, 2, 64, 16, [90, 33], [12, 5], dtype, "tree", scale=-0.3, want_lse=False)
    _attend(2, 2, 12, 4, 2, 128, 16, [90, 33], [12, 5], dtype, "tree", scale=0.0)
    _attend(3, 2, 12, 4, 2, 128, 64, [1500, 800], [12, 5], dtype, "tree", scale=4.0)  # one weight takes almost all

    def grow(key, value):  # largest scores that keep growing along the prefix, far apart
        key *= torch.linspace(0.01, 30.0, key.shape[1], device="cuda").view(1, -1, 1, 1).to(BF)

    _attend(4, 2, 12, 4, 2, 128, 64, [1500, 800], [12, 5], dtype, "tree", spoil=grow)


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("rows,lens", [(40, [90, 120]), (200, [300, 1])])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, rows, lens):
    """NaN and infinities among the new entries: only the rows that see them have them; memory behind the last slot holds NaN anyway."""
    def spoil(key, value):
        for b, n in enumerate(lens):
            value[b, n - 1 + 9] = math.nan
            value[b, n - 1 + 20, :, 3] = math.inf
            value[b, n - 1 + 21, :, 3] = -math.inf
            value[b, n - 1 + 30, 0, 5] = math.nan

    out = _attend(rows, 2, rows, 4, 2, 128, 16, lens, [rows, rows - 1], dtype, "tree", spoil=spoil)
    assert torch.isnan(out).any() and torch.isfinite(out[0, 0]).all()


def test_keys_that_are_not_numbers_in_places_not_seen():
    def spoil(key, value):
        key[0, 59 + 5:59 + 9] = math.nan
        key[0, 59 + 11] = math.inf

    rng = np.random.default_rng(0)
    B, rows, Hq, Hk, D, page = 1, 16, 4, 2, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = _graft(rows, B)
    table, n_pages = ref.page_table(rng, B, 5)
    c = _cache(gen, (1, n_pages, Hk, page, D), BF)
    key = torch.randn((B, 75, Hk, D), generator=gen, device="cuda").to(BF)
    value = torch.randn((B, 75, Hk, D), generator=gen, device="cuda").to(BF)
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    m = np.zeros((B, rows, 1), np.int32)
    m[0, :, 0] = 0b1001  # every row sees new rows 0 and 3 alone
    outs = []
    for bad in (False, True):
        if bad:
            spoil(key, value)
        g.cache_write(c, 0, _i32(table), _i32([1]), _i32([75]), key, value)
        out = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
        g.tree_attention(c, 0, _i32(table), q, _i32([60]), _i32([16]), _i32(m), out)
        outs.append(out)
    assert torch.isfinite(outs[1]).all() and torch.equal(*outs)


def test_slots_beyond_32_bits_of_bytes():
    """A cache of over 4 GB, its last pages in use."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, rows, Hq, Hk, D, page = 1, 5, 8, 8, 128, 64
    n_pages = 33000  # 33000 * 8 * 64 * 256 bytes = 4.3 GB of keys
    g = _graft(rows, B)
    from paper_2608_20375_b200 import KVCache
    shape = (1, n_pages, Hk, page, D)
    c = KVCache(torch.empty(shape, dtype=BF, device="cuda"), torch.empty(shape, dtype=BF, device="cuda"))
    small = KVCache.alloc(1, 4, Hk, page, D)
    key, value = (torch.randn((B, 150, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    outs = []
    for cache, table in ((small, [[0, 1, 2]]), (c, [[n_pages - 1, n_pages - 3, n_pages - 2]])):
        out = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
        g.cache_write(cache, 0, _i32(table), _i32([1]), _i32([150]), key, value)
        g.tree_attention(cache, 0, _i32(table), q, _i32([146]), _i32([5]), None, out)
        outs.append(out)
    assert torch.equal(*outs) and outs[0].abs().sum() > 0


def test_attention_twice_captured_and_on_another_stream():
    """The same call again, replayed from a graph with new numbers, and on a stream of its own: the same bits."""
    rng, gen = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(1)
    B, rows, Hq, Hk, D, page = 3, 20, 8, 2, 128, 64
    g = _graft(rows, B)
    table, n_pages = ref.page_table(rng, B, 40)
    c = _cache(gen, (1, n_pages, Hk, page, D), BF, garbage=False)
    c.k.copy_(torch.randn(c.k.shape, generator=gen, device="cuda"))
    c.v.copy_(torch.randn(c.v.shape, generator=gen, device="cuda"))
    m = np.stack([ref.tree(rng, 20, rows)[2] for _ in range(B)])
    tb, mm, q = _i32(table), _i32(m), torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
    pl, cnt = _i32([2500, 100, 1200]), _i32([20, 20, 13])
    call = lambda o: g.tree_attention(c, 0, tb, q, pl, cnt, mm, o)  # noqa: E731
    new = lambda: torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")  # noqa: E731
    a, b, d = new(), new(), new()
    call(a)
    call(b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(d)
    s.synchronize()
    assert torch.equal(a, d)
    graph, e = torch.cuda.CUDAGraph(), new()
    with torch.cuda.graph(graph):
        call(e)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, e)
    q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
    pl.copy_(_i32([700, 2300, 1]))
    graph.replay()
    f = new()
    call(f)
    torch.cuda.synchronize()
    assert torch.equal(e, f) and not torch.equal(a, f)


# ---- the walk ------------------------------------------------------------------------------------------------------
def _trees(rng, B, nmax, counts, V, L):
    parent, depth = np.full((B, nmax), -1, np.int32), np.full((B, nmax), -1, np.int32)
    mask = np.zeros((B, nmax, (nmax + 31) // 32), np.int32)
    token = np.full((B, nmax), -1, np.int32)
    for b in range(B):
        parent[b], depth[b], mask[b] = ref.tree(rng, counts[b], nmax, L)
        for i in range(counts[b]):
            sib = {int(token[b, j]) for j in range(1, i) if i and parent[b, j] == parent[b, i]}
            t = int(rng.integers(0, V))
            while t in sib and len(sib) < V:
                t = (t + 1) % V
            token[b, i] = t
    return parent, depth, mask, token


def _verify(g, B, rows, nmax, counts, parent, token, z, T, u, L, status=True):
    from paper_2608_20375_b200 import TreeOut
    tr = TreeOut(_i32(counts), None, _i32(token), _i32(parent), None, None, None, None, None)
    alen, path, bonus = (torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,)))
    st = torch.full((B,), -9, dtype=torch.int32, device="cuda") if status else None
    g.verify(tr, z, None if T is None else torch.from_numpy(T).cuda(), u, alen, path, bonus, st)
    torch.cuda.synchronize()
    return alen.cpu().numpy(), path.cpu().numpy(), bonus.cpu().numpy(), None if st is None else st.cpu().numpy()


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("B,rows,nmax,V,L,T", [
    (1, 2, 2, 1000, 4, 1.0), (3, 30, 40, 5000, 6, 0.7), (64, 33, 33, 1237, 16, 1.0), (2, 100, 100, 32000, 16, 1.5), (5, 9, 20, 7, 3, 1.0),
    (150, 17, 17, 333, 8, 0.9), (2, 600, 601, 101, 16, 1.0),
])
def test_walk(dtype, B, rows, nmax, V, L, T):
    rng, gen = np.random.default_rng(B + V), torch.Generator(device="cuda").manual_seed(B + V)
    from paper_2608_20375_b200 import Graft
    g = Graft(V, L, min(4, V), 16, 8, B, 1, nmax - 1, 1, 0.0)
    counts = rng.integers(1, rows + 1, B)
    counts[0] = rows
    parent, depth, mask, token = _trees(rng, B, nmax, counts, V, L)
    z = (2.0 * torch.randn((B, rows, V), generator=gen, device="cuda")).to(dtype)
    for b in range(B):  # the target likes what was drafted, often
        for i in range(1, counts[b]):
            if rng.random() < 0.6:
                z[b, parent[b, i], token[b, i]] += 4.0 + math.log(V)
    z[0, 0, ::3] = -math.inf
    if V > 500:
        z[-1, :, 1::2] = torch.finfo(dtype).min
    Ts = np.full(B, T, np.float32)
    Ts[1::4] = 0.0
    u = torch.rand((B, nmax), generator=gen, device="cuda")
    u[::5, 0] = 0.0
    alen, path, bonus, st = _verify(g, B, rows, nmax, counts, parent, token, z, Ts, u, L)
    assert not st.any()
    zc, uc = z.cpu().double().numpy(), u.cpu().double().numpy()
    for b in range(B):
        a, pa, bo = ref.walk(counts[b], parent[b], token[b], lambda i: zc[b, i], Ts[b], uc[b], L)
        assert (alen[b], bonus[b]) == (a, bo) and np.array_equal(path[b], pa), (b, alen[b], a, bonus[b], bo)
    assert B < 50 or alen.max() > 1


def test_greedy_walk_is_accept():
    """Temperature 0 gives what graft_accept gives for the rows' likeliest tokens, ties to the lowest id; the history is kept too."""
    from paper_2608_20375_b200 import Graft, TreeOut
    rng, gen = np.random.default_rng(8), torch.Generator(device="cuda").manual_seed(8)
    B, N, V, L = 6, 50, 40, 8
    g = Graft(V, L, 4, 16, 8, B, 1, N - 1, 1, 0.0)
    counts = np.array([50, 1, 20, 33, 50, 7])
    parent, depth, mask, token = _trees(rng, B, N, counts, V, L)
    z = torch.round(torch.randn((B, N, V), generator=gen, device="cuda") * 2).to(BF)
    nxt = torch.from_numpy(z.cpu().float().numpy().argmax(2).astype(np.int32)).cuda()
    trees = TreeOut(_i32(counts), None, _i32(token), _i32(parent), None, None, None, None, None)
    got = []
    for how in range(2):
        win, cnt, hist = torch.zeros((B, 3), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
        g.set_hist_window(3, win, cnt, hist)
        o = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,))]
        for _ in range(2):
            if how:
                g.verify(trees, z, torch.zeros(B, device="cuda"), torch.rand((B, N), device="cuda"), *o)
            else:
                g.accept(trees, nxt, *o)
        torch.cuda.synchronize()
        got.append([t.cpu().numpy() for t in (*o, win, cnt, hist)])
    for x, y in zip(*got):
        assert np.array_equal(x, y)


def test_comparisons_at_their_border():
    """Uniform numbers that sit on the border between two answers, a rounding of fp32 to either side of it: the sums that decide are fp64's."""
    from paper_2608_20375_b200 import Graft
    rng, gen = np.random.default_rng(4), torch.Generator(device="cuda").manual_seed(4)
    B, N, V, L = 64, 3, 20011, 2
    g = Graft(V, L, 4, 16, 8, B, 1, N - 1, 1, 0.0)
    parent, token = np.tile(np.array([-1, 0, 0], np.int32), (B, 1)), np.tile(np.array([5, 17, 400], np.int32), (B, 1))
    z = (2.0 * torch.randn((B, N, V), generator=gen, device="cuda")).to(torch.float32)
    z[:, 0, 17] = 9.0
    z[:, 0, 400] = 8.0
    zc = z.cpu().double().numpy()
    u = np.zeros((B, N), np.float32)
    for b in range(B):
        w = np.exp(zc[b, 0] - zc[b, 0].max())
        edge = np.float32(w[17] / w.sum())
        u[b, 1] = [np.nextafter(edge, np.float32(0)), edge, np.nextafter(edge, np.float32(1))][b % 3]
        w1 = w.copy()
        w1[17] = 0
        edge = np.float32(w1[400] / w1.sum())
        u[b, 2] = [edge, np.nextafter(edge, np.float32(1))][b % 2]
        w1[400] = 0
        c = np.cumsum(w1)
        edge = np.float32(c[rng.integers(0, V)] / c[-1])
        u[b, 0] = min(edge, np.nextafter(np.float32(1), np.float32(0)))
    alen, path, bonus, st = _verify(g, B, N, N, np.full(B, N), parent, token, z, None, torch.from_numpy(u).cuda(), L)
    for b in range(B):
        a, pa, bo = ref.walk(N, parent[b], token[b], lambda i: zc[b, i], 1.0, u[b].astype(np.float64), L)
        assert (alen[b], bonus[b]) == (a, bo) and np.array_equal(path[b], pa), (b, alen[b], a, bonus[b], bo)
    assert 0 < (alen > 0).sum() < B


def test_walk_reports_bad_rows_and_trees():
    from paper_2608_20375_b200 import Graft
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, N, V, L = 12, 5, 900, 4
    g = Graft(V, L, 4, 16, 8, B, 1, N - 1, 1, 0.0)
    parent = np.tile(np.array([-1, 0, 0, 1, 3], np.int32), (B, 1))
    token = np.tile(np.array([1, 2, 3, 4, 5], np.int32), (B, 1))
    counts = np.full(B, N)
    z = torch.randn((B, N, V), generator=gen, device="cuda").to(BF)
    z[:, 0, 2] = z[:, 1, 4] = z[:, 3, 5] = 60.0  # root -> 1 -> 3 -> 4
    T = np.ones(B, np.float32)
    z[0, 0, 7] = math.nan         # at the root
    z[1, 3, 8] = math.inf         # two steps in
    z[2, 1] = -math.inf           # nothing finite, one step in
    z[3, 2, 9] = math.nan         # a row that is not visited
    T[4], T[5], T[6], T[7] = -1.0, math.nan, math.inf, 0.0
    z[7, 4, 0] = math.nan         # greedy, at the last node
    counts[8], counts[9] = 0, N + 1
    token[10, 1] = V              # no token of the vocabulary: never accepted
    token[11, 2], z[11, 0, 2] = 2, 0.0  # the same token twice among siblings counts once
    u = torch.full((B, N), 0.5, device="cuda")
    alen, path, bonus, st = _verify(g, B, N, N, counts, parent, token, z, T, u, L)
    assert st.tolist() == [1, 1, 1, 0, 1, 1, 1, 1, 32, 32, 0, 0]
    assert alen.tolist()[:10] == [0, 2, 1, 3, 0, 0, 0, 3, 0, 0]
    assert (bonus[[0, 1, 2, 4, 5, 6, 7, 8, 9]] == -1).all() and bonus[3] >= 0
    assert path[1].tolist() == [1, 3, -1, -1] and path[3].tolist() == [1, 3, 4, -1] and (path[[0, 4, 5, 6, 8, 9]] == -1).all()
    zc = z.cpu().double().numpy()
    for b in (3, 10, 11):
        a, pa, bo = ref.walk(N, parent[b], token[b], lambda i: zc[b, i], T[b], np.full(N, 0.5), L)
        assert (alen[b], bonus[b]) == (a, bo) and np.array_equal(path[b], pa)


def test_walk_ends_at_the_block_length_and_where_nothing_is_left():
    from paper_2608_20375_b200 import Graft
    B, V, L = 2, 50, 3
    g = Graft(V, L, 4, 16, 8, B, 1, 7, 1, 0.0)
    parent = np.tile(np.array([-1, 0, 1, 2, 3, 4, 5, 6], np.int32), (B, 1))  # deeper than L: never by graft_build_trees
    token = np.tile(np.arange(8, dtype=np.int32), (B, 1))
    z = torch.full((B, 8, V), -math.inf, device="cuda")
    z[0, torch.arange(8), torch.arange(8) + 1] = 1.0  # all the weight on the next node's token
    z[1, 0, 1] = 0.0
    z[1, 1, 30:33] = 2.0
    u = torch.full((B, 8), float(np.nextafter(np.float32(1), np.float32(0))), device="cuda")
    alen, path, bonus, st = _verify(g, B, 8, 8, np.full(B, 8), parent, token, z, None, u, L)
    assert not st.any() and alen.tolist() == [3, 1] and bonus.tolist() == [4, 32]
    assert path.tolist() == [[1, 2, 3], [1, -1, -1]]


# ---- refusals ------------------------------------------------------------------------------------------------------
def test_refusals():
    from paper_2608_20375_b200 import GraftError, KVCache, TreeOut
    B, rows, Hq, Hk, D, page, L = 2, 4, 4, 2, 64, 16, 16
    g = _graft(rows, B)
    c = KVCache.alloc(2, 6, Hk, page, D)
    tb, pl, cnt = _i32([[0, 1], [2, 3]]), _i32([1, 1]), _i32([1, 1])
    q = torch.zeros((B, rows, Hq, D), dtype=BF, device="cuda")
    kv = torch.zeros((B, rows, Hk, D), dtype=BF, device="cuda")
    out, mask = torch.zeros_like(q), torch.zeros((B, rows, 1), dtype=torch.int32, device="cuda")
    ok = dict(cache=c, layer=0, table=tb, q=q, prefix_len=pl, count=cnt, mask=mask, out=out)
    g.tree_attention(**ok)

    def refuse(match="", **kw):
        with pytest.raises(GraftError, match=match):
            g.tree_attention(**dict(ok, **kw))

    refuse("invalid", layer=2)
    refuse("invalid", layer=-1)
    refuse("invalid", shared=8)
    refuse("invalid", shared=48)
    refuse("invalid", shared=-16)
    refuse("invalid", scale=math.nan)
    refuse("invalid", scale=math.inf)
    refuse("invalid", q=torch.zeros((B, rows, 3, D), dtype=BF, device="cuda"), out=torch.zeros((B, rows, 3, D), dtype=BF, device="cuda"))
    refuse("bfloat16", q=q.float())
    refuse("shape", out=out[:, :2].contiguous())
    refuse("shape", mask=mask[:, :2].contiguous())
    refuse("shape", table=tb[:1])
    refuse("shape", prefix_len=pl[:1])
    refuse("dtype", prefix_len=pl.long())
    refuse("CUDA", count=cnt.cpu())
    refuse("contiguous", out=torch.zeros((B, rows, D, Hq), dtype=BF, device="cuda").transpose(2, 3))
    refuse("strides", q=torch.zeros((B, rows, D, Hq), dtype=BF, device="cuda").transpose(2, 3))
    refuse("strides", q=torch.zeros((B, rows, 2 * Hq, D), dtype=BF, device="cuda")[:, :, ::2])
    refuse("invalid", q=torch.zeros((B, rows, Hq * D + 4), dtype=BF, device="cuda")[:, :, :Hq * D].unflatten(2, (Hq, D)))  # 8 bytes off
    refuse("invalid", q=torch.zeros(B * rows * Hq * D + 1, dtype=BF, device="cuda")[1:].view(B, rows, Hq, D))
    refuse("supported", cache=KVCache.alloc(1, 6, Hk, page, 32), q=q[..., :32].contiguous(), out=out[..., :32].contiguous())
    refuse("supported", cache=KVCache.alloc(1, 6, Hk, 8, D))
    refuse("supported", cache=KVCache.alloc(1, 6, Hk, 24, D))
    refuse("supported", cache=KVCache.alloc(1, 1, Hk, 2048, D))
    refuse("shape", cache=KVCache(c.k, c.v[:1].contiguous()))
    more = torch.zeros((B, rows + 1, Hq, D), dtype=BF, device="cuda")
    refuse("invalid", q=more, out=more.clone())  # masks have room for fewer rows
    big = torch.zeros((B + 1, rows, Hq, D), dtype=BF, device="cuda")
    refuse("invalid", q=big, out=big.clone(), table=_i32([[0, 1]] * 3), prefix_len=_i32([1] * 3), count=_i32([1] * 3), mask=None)
    for call in (lambda **k: g.cache_write(c, 0, tb, pl, cnt, k.get("key", kv), k.get("value", kv), k.get("status")),
                 lambda **k: g.cache_read(c, 0, tb, pl, cnt, k.get("key", kv), k.get("value", kv), k.get("status"))):
        call()
        for kw in (dict(key=kv[..., :32].contiguous()), dict(value=kv[:, :2].contiguous()), dict(key=kv.float()),
                   dict(status=torch.zeros(3, dtype=torch.int32, device="cuda"))):
            with pytest.raises(GraftError):
                call(**kw)
    alen, path = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, L), dtype=torch.int32, device="cuda")
    g.cache_keep(c, tb, pl, alen, path)
    with pytest.raises(GraftError, match="shape"):
        g.cache_keep(c, tb, pl, alen, path[:, :4].contiguous())
    tr = TreeOut(cnt, None, mask[:, :, 0].contiguous(), mask[:, :, 0].contiguous(), None, None, None, None, None)
    z, u, bonus = torch.zeros((B, rows, 64), device="cuda"), torch.zeros((B, rows), device="cuda"), torch.zeros_like(alen)
    g.verify(tr, z, None, u, alen, path, bonus)
    for kw in (dict(z=z.half()), dict(z=z[:, :, :32].contiguous()), dict(u=u[:, :2].contiguous()), dict(z=torch.zeros((B, rows + 1, 64), device="cuda")),
               dict(T=torch.zeros(1, device="cuda")), dict(path=path[:1])):
        with pytest.raises(GraftError):
            g.verify(tr, kw.get("z", z), kw.get("T"), kw.get("u", u), alen, kw.get("path", path), bonus)
    torch.cuda.synchronize()


# ---- together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, Q8])
def test_rounds_of_a_small_model(dtype):
    """Several rounds: trees from graft_build_trees, a model of two attention layers over the cache, the sampled walk, the move of the accepted
    entries.  After every round the cache holds the committed tokens' entries, and attention over it is that of a plain prompt."""
    from paper_2608_20375_b200 import BF16, E4M3, Graft, KVCache
    rng, gen = np.random.default_rng(3), torch.Generator(device="cuda").manual_seed(3)
    B, L, V, K, Hq, Hk, D, page, layers, rounds = 3, 6, 300, 5, 4, 2, 64, 16, 2, 4
    g = Graft(V, L, K, 16, 8, B, 4, 24, 4, 0.0)
    N, E = g.nmax, Hq * D
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    emb, head = r(V, E), 0.3 * r(E, V)
    wq, wk, wv = r(layers, E, Hq * D) / E ** 0.5, r(layers, E, Hk * D) / E ** 0.5, r(layers, E, Hk * D) / E ** 0.5
    c = KVCache.alloc(layers, 40, Hk, page, D, E4M3 if dtype is Q8 else BF16)
    table = _i32(rng.permutation(40)[:B * 10].reshape(B, 10))

    def model(tokens, prefix_len, count, mask):
        """tokens [B, n] -> logits [B, n, V]; new entries go into the cache."""
        x = emb[tokens.long().clamp(0)]
        n = tokens.shape[1]
        for i in range(layers):
            q, k, v = ((x @ w[i]).to(BF).view(B, n, -1, D) for w in (wq, wk, wv))
            o = torch.zeros((B, n, Hq, D), dtype=BF, device="cuda")
            g.cache_write(c, i, table, prefix_len, count, k, v)
            g.tree_attention(c, i, table, q, prefix_len, count, mask, o)
            x = x + o.float().view(B, n, E)
        return x @ head

    prompt = [11, 29, 40]
    text = [list(rng.integers(0, V, n)) for n in prompt]
    n = max(prompt)
    padded = np.zeros((B, n), np.int32)
    for b in range(B):
        padded[b, :prompt[b]] = text[b]
    # (all tokens but the last: that is the first round's root)
    model(_i32(padded), _i32([1] * B), _i32([p - 1 for p in prompt]), None)
    prefix = _i32(prompt)
    out = g.alloc_out(B)
    alen, path, bonus = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,)))
    for _ in range(rounds):
        root = _i32([t[-1] for t in text])
        draft = 3.0 * r(B, L, V)
        g.build_trees(draft.to(BF), None, root, None, prefix, _i32([20, 4, 24]), out)
        logits = model(out.token, prefix, out.n_nodes, out.mask)
        # a target that likes some of what was drafted
        ids = out.token.long().clamp(0)
        par = out.parent.long().clamp(0)
        logits.view(B, -1).scatter_add_(1, par * V + ids, torch.where(out.parent >= 0, 8.0 * torch.rand(ids.shape, generator=gen, device="cuda"), 0.0))
        u = torch.rand((B, N), generator=gen, device="cuda")
        g.verify(out, logits, None, u, alen, path, bonus)
        torch.cuda.synchronize()
        o = out.cpu()
        for b in range(B):
            zb = logits[b].cpu().double().numpy()
            a, pa, bo = ref.walk(int(o["n_nodes"][b]), o["parent"][b], o["token"][b], lambda i: zb[i], 1.0, u[b].cpu().double().numpy(), L)
            assert (int(alen[b]), int(bonus[b])) == (a, bo) and np.array_equal(path[b].cpu().numpy(), pa)
            text[b] += [int(o["token"][b][i]) for i in pa[:a]] + [bo]
        g.cache_keep(c, table, prefix, alen, path, prefix)
        assert prefix.tolist() == [len(t) for t in text]
        # a fresh cache, the committed tokens as a prompt: the same entries
        fresh = KVCache.alloc(layers, 40, Hk, page, D, E4M3 if dtype is Q8 else BF16)
        used, c = c, fresh
        n = max(len(t) for t in text)
        padded = np.zeros((B, n), np.int32)
        for b in range(B):
            padded[b, :len(text[b])] = text[b]
        model(_i32(padded), _i32([1] * B), prefix - 1, None)
        c = used
        for b in range(B):
            s = np.arange(len(text[b]) - 1)
            tr = table[b].cpu().numpy()
            for i in range(layers):
                for x, y, xe, ye in ((used.k, fresh.k, used.k_exp, fresh.k_exp), (used.v, fresh.v, used.v_exp, fresh.v_exp)):
                    p_, q_ = (ref.entries(t[i].cpu(), None if e is None else e[i].cpu(), tr, s) for t, e in ((x, xe), (y, ye)))
                    # layer 0: the same numbers; layer 1 behind an attention whose sums may run in another order: a rounding of bf16 of its
                    # result moves the next layer's numbers by 2^-8 of the attention's part, and in e4m3 a number may fall to the other side
                    # of a rounding of 2^-4
                    rel = 0.0 if i == 0 else 2.0 ** -7 if dtype is BF else 2.0 ** -3
                    assert np.linalg.norm(p_ - q_) <= rel * np.linalg.norm(q_)
    assert min(len(t) - p for t, p in zip(text, prompt)) >= rounds
