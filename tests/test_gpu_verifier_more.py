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
@pytest.mark.parametrize("rows,shared", [(1, 0), (30, 0), (30, 32), (100, 0)])
def test_no_sequence_has_rows(dtype, rows, shared):
    _attend(3, 3, rows, 4, 2, 64, 16, [33, 40, 90], [0, 0, 0], dtype, "tree", shared=shared)
    _attend(3, 3, rows, 4, 2, 64, 16, [33, 40, 90], [0, 1, 0], dtype, "tree", shared=shared)


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_short_units_among_long_ones(dtype):
    """What a unit costs beside its tiles is in the line too: stretches may begin behind a unit's tiles, or have none of any."""
    rng = np.random.default_rng(4)
    for rows, lens in ((1, [1] * 70 + [1800]), (40, [1] * 40 + [3000]), (70, rng.integers(1, 140, 37).tolist())):
        _attend(rows, len(lens), rows, 4, 2, 64, 16, lens, [rows] * len(lens), dtype, None)
    _attend(9, 30, 9, 32, 2, 64, 16, [129 + i for i in range(30)], [9] * 30, dtype, "tree", shared=128)


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_calls_in_two_graphs_and_of_two_shapes_follow_one_another(dtype):
    """Captured calls of several shapes share their context's workspace: replayed one behind another on one stream, results stay."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    B, Hq, Hk, D, page = 4, 8, 2, 128, 16
    g = _graft(64, B)
    table, n_pages = ref.page_table(np.random.default_rng(2), B, 60)
    c = _cache(gen, (1, n_pages, Hk, page, D), dtype, garbage=False)
    key, value = (torch.randn((B, 900, Hk, D), generator=gen, device="cuda").to(BF) for _ in range(2))
    tb = _i32(table)
    g.cache_write(c, 0, tb, _i32([1] * B), _i32([900] * B), key, value)
    calls = []
    for rows in (1, 20, 64):
        q = torch.randn((B, rows, Hq, D), generator=gen, device="cuda").to(BF)
        o = torch.zeros_like(q)
        args = (c, 0, tb, q, _i32([900 - rows - 7 * b for b in range(B)]), _i32([rows] * B), None, o)
        g.tree_attention(*args)
        calls.append((args, o, o.clone()))
    torch.cuda.synchronize()
    graphs = []
    for args, o, _ in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            g.tree_attention(*args)
    for _ in range(3):
        for graph, (_, o, _) in zip(graphs, calls):
            o.zero_()
            graph.replay()
        for _, o, want in calls:
            assert torch.equal(o, want)


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


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_micro_batches_with_caches(dtype):
    """Two micro-batches around a target of one attention layer, each with its cache: on streams of their own the rounds' results are the
    sequential schedule's, and those of the calls made one by one; the cache holds the committed tokens."""
    from paper_2608_20375_b200 import BF16, E4M3, Graft, KVCache, MicroBatch, Sampled, join, run_rounds
    B, L, V, K, Hq, Hk, D, page, rounds = 3, 6, 300, 5, 4, 2, 64, 16, 4
    gen = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    E = Hq * D
    emb, head = r(V, E), 0.5 * r(E, V)
    w = [(r(E, h * D) / E ** 0.5) for h in (Hq, Hk, Hk)]
    table = torch.arange(B * 8, dtype=torch.int32, device="cuda").view(B, 8)
    drafts = [[3.0 * r(B, L, V) for _ in range(rounds)] for _ in range(2)]
    uniform = [[torch.rand((B, 64), generator=gen, device="cuda") for _ in range(rounds)] for _ in range(2)]

    def run(how):
        log, micro, roots = [], [], []
        for i in range(2):
            g = Graft(V, L, K, 16, 8, B, 4, 24, 4, 0.0)
            c = KVCache.alloc(1, B * 8, Hk, page, D, E4M3 if dtype is Q8 else BF16)
            micro.append(MicroBatch(g, B, L, cache=c, table=table, prefix_len=_i32([1, 1, 1])))
            roots.append(_i32([3, 5 + i, 7]))

        def draft(i, k):
            mb = micro[i]
            root = roots[i] if k == 0 else mb.bonus_token.clone()
            return dict(logits=drafts[i][k].to(BF), root_token=root, fixed_budget=_i32([20, 4, 24]))

        def verify(i, k, out):
            mb = micro[i]
            x = emb[out.token.long().clamp(0)]
            q, key, value = ((x @ m).to(BF).view(B, mb.graft.nmax, -1, D) for m in w)
            o = torch.zeros((B, mb.graft.nmax, Hq, D), dtype=BF, device="cuda")
            if how == "by hand":
                mb.graft.cache_write(mb.cache, 0, table, mb.prefix_len, out.n_nodes, key, value)
                mb.graft.tree_attention(mb.cache, 0, table, q, mb.prefix_len, out.n_nodes, out.mask, o)
            else:
                mb.attend(0, q, key, value, o)
            z = (x + o.float().view(B, mb.graft.nmax, E)) @ head
            z.view(B, -1).scatter_add_(1, out.parent.long().clamp(0) * V + out.token.long().clamp(0), torch.where(out.parent >= 0, 9.0, 0.0))
            return Sampled(z, uniform[i][k][:, :mb.graft.nmax].contiguous())

        def after(i, k, mb):
            log.append([t.clone() for t in (mb.accept_len, mb.accept_path, mb.bonus_token, mb.prefix_len, mb.status)])

        if how == "by hand":
            for k in range(rounds):
                for i, mb in enumerate(micro):
                    x = draft(i, k)
                    mb.graft.build_trees(x["logits"], None, x["root_token"], None, mb.prefix_len, x["fixed_budget"], mb.out)
                    a = verify(i, k, mb.out)
                    mb.graft.verify(mb.out, a.logits, a.temperature, a.uniform, mb.accept_len, mb.accept_path, mb.bonus_token)
                    mb.graft.cache_keep(mb.cache, table, mb.prefix_len, mb.accept_len, mb.accept_path, mb.prefix_len, mb.status)
                    after(i, k, mb)
        else:
            run_rounds(micro, rounds, draft, verify, overlap=how == "overlapped", after_round=after)
            join(micro)
        torch.cuda.synchronize()
        return [[t.cpu() for t in x] for x in log], micro

    want, micro = run("by hand")
    for how in ("sequential", "overlapped"):
        got, other = run(how)
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
        for a, b in zip(micro, other):
            n = int(a.prefix_len.min()) - 1
            kb = [torch.empty((B, n, Hk, D), dtype=BF, device="cuda") for _ in range(4)]
            for mb, x in ((a, kb[:2]), (b, kb[2:])):
                mb.graft.cache_read(mb.cache, 0, table, _i32([1] * B), _i32([n] * B), *x)
            torch.cuda.synchronize()
            assert torch.equal(kb[0], kb[2]) and torch.equal(kb[1], kb[3])
    for i, mb in enumerate(micro):
        lens = sum(x[0] for x in want[i::2]) + rounds + 1
        assert torch.equal(lens.int(), mb.prefix_len.cpu()) and not mb.status.any()
    assert sum(int(x[0].sum()) for x in want) > 0


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("V,offset", [(4001, 0), (4001, 1), (150001, 1), (150001, 3), (13, 1)])
def test_walk_of_wide_trees_and_rows_on_any_address(dtype, V, offset):
    """Hundreds of children of one node (tokens twice among them), logits that begin on any element."""
    from test_gpu_verifier import _verify
    from paper_2608_20375_b200 import Graft
    B, nmax, L, n = 6, 401, 4, 401
    rng, gen = np.random.default_rng(V), torch.Generator(device="cuda").manual_seed(V)
    g = Graft(V, L, 4, 16, 8, B, 1, nmax - 1, 1, 0.0)
    rows = 5
    parent, token = np.full((B, nmax), -1, np.int32), np.full((B, nmax), -1, np.int32)
    counts = np.full(B, rows)
    flat = torch.zeros(offset + B * nmax * V if V < 50000 else offset + B * rows * V, dtype=dtype, device="cuda")
    wide = V < 50000
    rows = nmax if wide else rows
    counts[:] = rows
    for b in range(B):
        parent[b, 1:rows] = 0
        parent[b, rows - 2:rows] = 1  # two grandchildren
        token[b, 1:rows] = rng.integers(0, V, rows - 1)
    z = flat[offset:].view(B, rows, V)
    z.copy_(torch.randn((B, rows, V), generator=gen, device="cuda"))
    for b in range(B):
        z[b, 0, torch.from_numpy(token[b, 1:rows].astype(np.int64)).cuda()] += 5.0 if b % 2 else 1.0
    u = torch.rand((B, nmax), generator=gen, device="cuda")
    u[1, 1:] = 0.999
    alen, path, bonus, st = _verify(g, B, rows, nmax, counts, parent, token, z, None, u, L)
    again = _verify(g, B, rows, nmax, counts, parent, token, z, None, u, L)
    assert not st.any() and all(np.array_equal(x, y) for x, y in zip((alen, path, bonus), again))
    uc = u.cpu().double().numpy()
    for b in range(B):
        a, pa, bo = ref.walk(rows, parent[b], token[b], lambda i: z[b, i].cpu().double().numpy(), 1.0, uc[b], L)
        assert (alen[b], bonus[b]) == (a, bo) and np.array_equal(path[b], pa), (b, alen[b], a, bonus[b], bo)


def test_walk_and_move_captured():
    """A round's walk and move in a graph, replayed with other numbers: the results of the calls."""
    from paper_2608_20375_b200 import Graft, TreeOut
    B, nmax, L, V, Hk, D, page, layers = 4, 33, 8, 5003, 2, 64, 16, 5
    rng, gen = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(1)
    from test_gpu_verifier import _trees
    g = Graft(V, L, 4, 16, 8, B, 1, nmax - 1, 1, 0.0)
    counts = np.array([33, 20, 1, 30])
    parent, _, _, token = _trees(rng, B, nmax, counts, V, L)
    tr = TreeOut(_i32(counts), None, _i32(token), _i32(parent), None, None, None, None, None)
    table, n_pages = ref.page_table(rng, B, 10)
    c = _cache(gen, (layers, n_pages, Hk, page, D), BF, garbage=False)
    tb, z, u = _i32(table), torch.zeros((B, nmax, V), device="cuda"), torch.zeros((B, nmax), device="cuda")
    pl, nxt = _i32([1, 30, 77, 100]), _i32([0] * B)
    outs = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,))]

    def fill(seed):
        gen.manual_seed(seed)
        z.copy_(torch.randn(z.shape, generator=gen, device="cuda"))
        for b in range(B):
            for i in range(1, counts[b]):
                z[b, parent[b, i], token[b, i]] += 9.0
        u.copy_(torch.rand(u.shape, generator=gen, device="cuda"))
        c.k.copy_(torch.randn(c.k.shape, generator=gen, device="cuda"))
        c.v.copy_(torch.randn(c.v.shape, generator=gen, device="cuda"))

    def call():
        g.verify(tr, z, None, u, *outs)
        g.cache_keep(c, tb, pl, outs[0], outs[1], nxt)

    fill(1)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    seen = 0
    for seed in (2, 3):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*outs, nxt, c.k, c.v)]
        fill(seed)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (*outs, nxt, c.k, c.v)))
        assert torch.equal(nxt, pl + outs[0] + 1)
        seen += int(outs[0].sum())
    assert seen > 0
