"""The operators of the verification half of a decoding round, as cases that can be timed and compared.

Four kinds, every one through the package's public entry points:

  attention  attention of the trees' nodes (or single tokens) over a paged cache: Graft.tree_attention
  verify     the walk along a tree that keeps the target's distribution, from given random numbers: Graft.verify
  cache      new keys and values into a paged cache, quantised as they are written, and read back: Graft.cache_write, cache_read
  keep       the accepted nodes' cache entries moved up behind the prefix, in all layers: Graft.cache_keep

`own` False: the same in elementary torch operations.  Sequence b's slot s lives in page table[b, s // page_size]; row i of a call
sits in slot prefix_len[b] - 1 + i (row 0 is the last committed token).
"""
import functools
import math

import numpy as np
import torch

own = False

BOOST = 64     # tokens a target's row favours
MAX_DEPTH = 16  # block length of the drafter


# ---- cases ---------------------------------------------------------------------------------------------------------
def _attention(name, batch, nodes, q_heads, kv_heads, head_dim, len_lo, len_hi, shared=0, page=64, dtype="bf16", min_nodes=1,
               chain=False):
    return dict(name=name, kind="attention", batch=batch, nodes=nodes, min_nodes=min_nodes, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, len_lo=len_lo, len_hi=len_hi, shared=shared, page=page, dtype=dtype, chain=chain)


def _verify(name, batch, nodes, V, dtype="bf16", temperature=1.0, greedy_every=0, min_nodes=2):
    return dict(name=name, kind="verify", batch=batch, nodes=nodes, min_nodes=min_nodes, V=V, dtype=dtype, temperature=temperature,
                greedy_every=greedy_every)


def _cache(name, batch, rows, kv_heads, head_dim, len_lo, len_hi, page=64, dtype="e4m3", min_rows=1):
    return dict(name=name, kind="cache", batch=batch, rows=rows, min_rows=min_rows, kv_heads=kv_heads, head_dim=head_dim,
                len_lo=len_lo, len_hi=len_hi, page=page, dtype=dtype)


def _keep(name, batch, layers, nodes, kv_heads, head_dim, slots, page=64):
    return dict(name=name, kind="keep", batch=batch, layers=layers, nodes=nodes, kv_heads=kv_heads, head_dim=head_dim, slots=slots,
                page=page)


def listed():
    return [
        # one user, the tree of a fixed budget of 64 nodes over a short conversation: latency
        _attention("attn_b1_n65_len1500", 1, 65, 32, 8, 128, 1500, 1500, min_nodes=65),
        # single tokens of a full server over long contexts of unlike lengths, a quantised cache: bytes
        _attention("attn_b64_n1_len16000_e4m3", 64, 1, 32, 8, 128, 2000, 16000, dtype="e4m3"),
        # an ordinary serving batch, trees of unlike sizes, a quantised cache
        _attention("attn_b32_n65_len4096_e4m3", 32, 65, 32, 8, 128, 500, 4096, dtype="e4m3", min_nodes=17),
        # sequences behind one long system prompt, small trees, four key heads
        _attention("attn_b64_n17_shared8192", 64, 17, 32, 4, 128, 8193, 9200, shared=8192, min_nodes=17),
        # the largest budgets over long prefixes: operations
        _attention("attn_b16_n513_len8192", 16, 513, 32, 8, 128, 6000, 8192, min_nodes=257),
        # one user of a small vocabulary, a fixed budget, fp32 logits
        _verify("verify_b1_n65_v32000_f32", 1, 65, 32000, "f32", min_nodes=65),
        # the ordinary serving batch
        _verify("verify_b64_n65_v151936", 64, 65, 151936, min_nodes=17),
        # large budgets, a cooler target, some sequences greedy, a vocabulary that divides by nothing
        _verify("verify_b16_n257_v50021", 16, 257, 50021, temperature=0.7, greedy_every=4, min_nodes=129),
        # the nodes of a round's trees into the cache of one layer, quantised, and back
        _cache("cache_b64_n65_e4m3", 64, 65, 8, 128, 500, 4096, min_rows=17),
        # prompts of unlike lengths into an empty cache of one layer
        _cache("cache_b8_prompt8192_e4m3", 8, 8192, 8, 128, 1, 1, min_rows=1000),
        # one user: accepted entries of 36 layers
        _keep("keep_b1_l36", 1, 36, 65, 8, 128, 192),
        # the serving batch
        _keep("keep_b64_l24", 64, 24, 65, 8, 128, 192),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 5 + ["verify"] * 3 + ["cache"] * 2 + ["keep"] * 2)
    page = rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["bf16", "e4m3"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    head_dim = rng.choice([64, 128, 128])
    if kind == "attention":
        nodes = rng.choice([1, rng.randint(2, 65), _log_uniform(rng, 2, 513)])
        q_heads = kv_heads * rng.choice([1, 4, 4, 5, 7, 8])
        hi = _log_uniform(rng, 64, 16000)
        # no more key rows and no more products than the largest listed ones
        most = min(64, 64 * 16000 * 8 // (hi * kv_heads), 16 * 513 * 32 * 8192 // (nodes * q_heads * (hi + nodes)))
        batch = _log_uniform(rng, 1, max(1, most))
        shared = rng.choice([0, 0, 0, (hi // 2) // page * page])
        lo = max(shared + 1, rng.choice([1, hi // 2, hi]))
        c = _attention("", batch, nodes, q_heads, kv_heads, head_dim, lo, hi, shared, page, dtype, rng.randint(1, nodes),
                       rng.random() < 0.2)
    elif kind == "verify":
        V = rng.choice([32000, 128256, 151936, _log_uniform(rng, 1000, 151936)])
        nodes = _log_uniform(rng, 2, 257)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 64 * 65 * 151936 * 2 // (nodes * V * (4 if dtype == "f32" else 2))
        batch = _log_uniform(rng, 1, max(1, min(128, most)))
        c = _verify("", batch, nodes, V, dtype, rng.choice([1.0, 0.7, 1.3]), rng.choice([0, 0, 3]), rng.randint(1, nodes))
    elif kind == "cache":
        rows = rng.choice([1, rng.randint(2, 513), _log_uniform(rng, 2, 8192)])
        batch = _log_uniform(rng, 1, max(1, min(128, 8 * 8192 * 8 // (rows * kv_heads))))
        c = _cache("", batch, rows, kv_heads, head_dim, 1, _log_uniform(rng, 2, 4096), page, dtype, rng.randint(1, rows))
    else:
        layers = rng.randint(1, 36)
        batch = _log_uniform(rng, 1, max(1, min(64, 64 * 24 * 8 // (layers * kv_heads))))
        c = _keep("", batch, layers, rng.randint(2, 65), kv_heads, head_dim, rng.randint(130, 192), page)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------
def _spread(rng, lo, hi, n):
    """n whole numbers spread evenly over lo..hi, in random order."""
    return rng.permutation(np.rint(np.linspace(lo, hi, n)) if n > 1 else np.array([(lo + hi) // 2])).astype(np.int32)


def _trees(rng, n_nodes, nmax):
    """Trees in level order, no deeper than MAX_DEPTH: parents [B, nmax], depths, ancestor-or-self masks [B, nmax, W] as bits."""
    B, W = len(n_nodes), (nmax + 31) // 32
    parent = np.full((B, nmax), -1, np.int32)
    depth = np.full((B, nmax), -1, np.int32)
    mask = np.zeros((B, nmax, W), np.uint32)
    depth[:, 0] = 0
    mask[:, 0, 0] = 1
    for b, n in enumerate(n_nodes):
        if n < 2:
            continue
        levels = int(min(rng.integers(4, MAX_DEPTH + 1), n - 1))
        cuts = np.sort(rng.choice(np.arange(2, n), levels - 1, replace=False)) if levels > 1 else np.zeros(0, np.int64)
        ends = np.concatenate([[0, 1], cuts, [n]]).astype(np.int64)  # level d: nodes ends[d] .. ends[d + 1] - 1
        for d in range(1, levels + 1):
            i = np.arange(ends[d], ends[d + 1])
            # the first of a level, likelier than the others, have most of the children
            p = ends[d - 1] + np.sort(np.floor((ends[d] - ends[d - 1]) * rng.random(len(i)) ** 3)).astype(np.int64)
            parent[b, i], depth[b, i] = p, d
            mask[b, i] = mask[b, p]
            mask[b, i, i // 32] |= (np.uint32(1) << (i % 32).astype(np.uint32))
    return parent, depth, mask.view(np.int32)


def _table(rng, batch, width, shared_pages=0):
    """Page numbers [batch, width], all pages apart (but for the shared ones), in random order; and how many pages there are."""
    n = shared_pages + batch * (width - shared_pages)
    pages = rng.permutation(n).astype(np.int32)
    t = np.empty((batch, width), np.int32)
    t[:, :shared_pages] = pages[:shared_pages]
    t[:, shared_pages:] = pages[shared_pages:].reshape(batch, width - shared_pages)
    return t, n


def _heads(gen, shape):
    """Keys as models have them: N(0, 1) with a few channels that are several times larger."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    x[..., 3::37] *= 3
    return x


@functools.lru_cache(maxsize=8)
def _context(V, L, nmax, batch):
    from paper_2608_20375_b200 import Graft
    return Graft(V, L, 4, 16, 8, batch, 1, nmax - 1, 1, 0.0)


def prepare(case, seed):
    c = case
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    B = c["batch"]
    s = dict(kind=c["kind"], B=B)
    if c["kind"] == "verify":
        V, N = c["V"], c["nodes"]
        n_nodes = _spread(rng, c["min_nodes"], N, B)
        parent, depth, mask = _trees(rng, n_nodes, N)
        # the target's rows: 2 N(0, 1), and tokens that it favours, the likelier ones rather than the others drafted as children
        z = 2.0 * torch.randn((B, N, V), generator=gen, device="cuda", dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        n_fav = min(BOOST, V)
        first, step = rng.integers(0, V, (B, N)), rng.integers(1, max(2, V // BOOST), (B, N))
        fav = (first[:, :, None] + step[:, :, None] * np.arange(n_fav)) % V
        top = math.log(V) + 2.0  # about where one token weighs as much as all the others' noise
        height = rng.uniform(top - 1, top + 5, (B, N, 1)) * np.arange(1, n_fav + 1) ** -0.7
        z.scatter_add_(2, dev(fav), dev(height.astype(np.float32)).to(z.dtype))
        token = np.full((B, N), -1, np.int32)
        token[:, 0] = rng.integers(0, V, B)
        rank = np.zeros((B, N), np.int64)
        for i in range(1, N):  # children of a node in level order stand side by side
            rank[:, i] = np.where(parent[:, i] == parent[:, i - 1], rank[:, i - 1] + 1, 0)
        rows = np.arange(B)[:, None]
        child = fav[rows, np.maximum(parent, 0), rank % n_fav]
        alive = np.arange(N)[None, :] < n_nodes[:, None]
        token[:, 1:] = np.where(alive, child, -1)[:, 1:]
        temperature = np.full(B, c["temperature"], np.float32)
        if c["greedy_every"]:
            temperature[:: c["greedy_every"]] = 0.0
        s.update(logits=z, n_nodes=dev(n_nodes), token=dev(token), parent=dev(parent), depth=dev(depth), mask=dev(mask),
                 temperature=dev(temperature), uniform=torch.rand((B, N), generator=gen, device="cuda"), V=V, N=N,
                 accept_len=torch.empty(B, dtype=torch.int32, device="cuda"),
                 accept_path=torch.empty((B, MAX_DEPTH), dtype=torch.int32, device="cuda"),
                 bonus=torch.empty(B, dtype=torch.int32, device="cuda"))
        if own:
            s["graft"] = _context(V, MAX_DEPTH, N, B)
        return s
    Hk, D, page = c["kv_heads"], c["head_dim"], c["page"]
    s.update(Hk=Hk, D=D, page=page)
    if c["kind"] == "attention":
        N, Hq = c["nodes"], c["q_heads"]
        n_nodes = _spread(rng, c["min_nodes"], N, B)
        lens = _spread(rng, c["len_lo"], c["len_hi"], B)  # prefix lengths, the root included
        width = -(-(c["len_hi"] - 1 + N) // page)
        table, n_pages = _table(rng, B, width, c["shared"] // page)
        shape = (1, n_pages, Hk, page, D)
        k, v = _heads(gen, shape), torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
        k_exp = v_exp = None
        if c["dtype"] == "e4m3":
            (k, k_exp), (v, v_exp) = _quantise(k), _quantise(v)
        mask = None if c["chain"] else dev(_trees(rng, n_nodes, N)[2])
        s.update(k=k, v=v, k_exp=k_exp, v_exp=v_exp, table=dev(table), n_nodes=dev(n_nodes), prefix_len=dev(lens), mask=mask,
                 q=torch.randn((B, N, Hq, D), generator=gen, device="cuda", dtype=torch.bfloat16), shared=c["shared"],
                 out=torch.zeros((B, N, Hq, D), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((B, N, Hq), dtype=torch.float32, device="cuda"), N=N, Hq=Hq)
        if own:
            s["graft"] = _context(64, MAX_DEPTH, N + 1 if N == 1 else N, B)
            if N == 1 and mask is not None:  # the context's trees have room for a child
                s["mask"] = torch.nn.functional.pad(mask, (0, 0, 0, 1))
    elif c["kind"] == "cache":
        N = c["rows"]
        count = _spread(rng, c["min_rows"], N, B)
        lens = _spread(rng, c["len_lo"], c["len_hi"], B)
        width = -(-(c["len_hi"] - 1 + N) // page)
        table, n_pages = _table(rng, B, width)
        shape = (1, n_pages, Hk, page, D)
        q8 = c["dtype"] == "e4m3"
        blank = lambda: torch.zeros(shape, dtype=torch.float8_e4m3fn if q8 else torch.bfloat16, device="cuda")  # noqa: E731
        exps = lambda: torch.full(shape[:-1], 127, dtype=torch.uint8, device="cuda") if q8 else None  # noqa: E731
        rows = (B, N, Hk, D)
        s.update(k=blank(), v=blank(), k_exp=exps(), v_exp=exps(), table=dev(table), count=dev(count), prefix_len=dev(lens), N=N,
                 key=_heads(gen, rows), value=torch.randn(rows, generator=gen, device="cuda", dtype=torch.bfloat16),
                 key_back=torch.zeros(rows, dtype=torch.bfloat16, device="cuda"),
                 value_back=torch.zeros(rows, dtype=torch.bfloat16, device="cuda"))
        if own:
            s["graft"] = _context(64, MAX_DEPTH, 2, B)
    else:
        lens = _spread(rng, max(1, (c["slots"] - c["nodes"]) // 2), c["slots"] - c["nodes"], B)
        width = -(-c["slots"] // page)
        table, n_pages = _table(rng, B, width)
        shape = (c["layers"], n_pages, Hk, page, D)
        accept_len = np.minimum(_spread(rng, 0, MAX_DEPTH, B), c["nodes"] - 1)
        path = np.full((B, MAX_DEPTH), -1, np.int32)
        for b in range(B):  # node indices of an accepted path: they grow along it
            path[b, :accept_len[b]] = np.sort(rng.choice(np.arange(1, c["nodes"]), accept_len[b], replace=False))
        s.update(k=torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16), table=dev(table), prefix_len=dev(lens),
                 v=torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16), k_exp=None, v_exp=None,
                 accept_len=dev(accept_len), accept_path=dev(path),
                 next_prefix=torch.zeros(B, dtype=torch.int32, device="cuda"))
        if own:
            s["graft"] = _context(64, MAX_DEPTH, c["nodes"], B)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return {"attention": _run_attention, "verify": _run_verify, "cache": _run_cache, "keep": _run_keep}[s["kind"]](s)


def _own_cache(s):
    from paper_2608_20375_b200 import KVCache
    return KVCache(s["k"], s["v"], s["k_exp"], s["v_exp"])


def _quantise(x):
    """e4m3 numbers and, a row, the exponent of their scale: the smallest power of two with max|x| <= 448 times it."""
    x = x.float()
    amax = x.abs().amax(-1)
    f, e = torch.frexp(amax)
    e = torch.where(f <= 0.875, e - 9, e - 8).clamp(-120, 120)
    bad = ~torch.isfinite(amax)
    y = torch.ldexp(x, -e[..., None]).masked_fill(bad[..., None], 0.0).to(torch.float8_e4m3fn)
    return y, (e + 127).masked_fill(bad, 255).to(torch.uint8)


def _values(y, exp):
    """What a cache's entries stand for, in fp32."""
    if exp is None:
        return y.float()
    e = exp.int()
    return torch.ldexp(y.float(), (e - 127)[..., None]).masked_fill((e == 255)[..., None], float("nan"))


def _gather(s, x, exp, slots):
    """Entries at slots [B, S] of layer 0 -> [B, Hk, S, D], fp32."""
    page = s["table"].gather(1, slots // s["page"]).long()
    at = slots % s["page"]
    return _values(x[0][page, :, at], None if exp is None else exp[0][page, :, at]).transpose(1, 2)


def _run_attention(s):
    if own:
        s["graft"].tree_attention(_own_cache(s), 0, s["table"], s["q"], s["prefix_len"], s["n_nodes"], s["mask"], s["out"],
                                  lse=s["lse"], shared=s["shared"])
        return dict(out=s["out"], lse=s["lse"])
    B, N, Hq, Hk, D = s["B"], s["N"], s["Hq"], s["Hk"], s["D"]
    G, S = Hq // Hk, s["table"].shape[1] * s["page"]
    slots = torch.arange(S, device="cuda").expand(B, S)
    k, v = _gather(s, s["k"], s["k_exp"], slots), _gather(s, s["v"], s["v_exp"], slots)
    q = s["q"].float().view(B, N, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, N * G, D)
    sc = (q @ k.transpose(2, 3)).view(B, Hk, N, G, S) * D ** -0.5
    # slot base + j is visible to node i if j < 0 or bit j of the node's mask is set
    j = torch.arange(S, device="cuda")[None, :] - (s["prefix_len"] - 1)[:, None]
    if s["mask"] is None:
        seen = j[:, None, :] <= torch.arange(N, device="cuda")[None, :, None]
    else:
        bits = (s["mask"][:, :, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        bits = bits.view(B, N, -1)
        seen = (j < 0)[:, None, :] | (bits.gather(2, j.clamp(0, bits.shape[2] - 1)[:, None, :].expand(B, N, S)) > 0)
    seen = seen & (j < s["n_nodes"][:, None])[:, None, :]
    sc.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    w = (sc - top).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(B, Hk, N * G, S) @ v).view(B, Hk, N, G, D) / total
    alive = torch.arange(N, device="cuda")[None, :] < s["n_nodes"][:, None]
    o = o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).to(torch.bfloat16)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, N, Hq)
    s["out"].copy_(torch.where(alive[:, :, None, None], o, s["out"]))
    s["lse"].copy_(torch.where(alive[:, :, None], lse, s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


def _run_verify(s):
    if own:
        from paper_2608_20375_b200 import TreeOut
        trees = TreeOut(s["n_nodes"], None, s["token"], s["parent"], s["depth"], None, None, s["mask"], None)
        s["graft"].verify(trees, s["logits"], s["temperature"], s["uniform"], s["accept_len"], s["accept_path"], s["bonus"])
        return dict(accept_len=s["accept_len"], accept_path=s["accept_path"], bonus=s["bonus"])
    B, N, V = s["B"], s["N"], s["V"]
    z, T = s["logits"], s["temperature"]
    greedy = T == 0
    inv = torch.where(greedy, 1.0, T)
    i = torch.arange(N, device="cuda")
    alive = i[None, :] < s["n_nodes"][:, None]
    child = alive & (i > 0)[None, :]
    par = torch.where(child, s["parent"], 0).long()
    top, best = z.float().max(-1)
    best = (z == top[:, :, None].to(z.dtype)).to(torch.uint8).argmax(-1)  # the lowest of equal ones
    Z = ((z.float() - top[:, :, None]) / inv[:, None, None]).exp().sum(-1, dtype=torch.float64)
    tok = s["token"].clamp(0).long()
    e = (z.view(B, N * V).gather(1, par * V + tok).double() - top.gather(1, par).double()) / inv[:, None].double()
    e = torch.where(greedy[:, None], (best.gather(1, par) == tok).double(), e.exp())
    Z = torch.where(greedy[:, None], 1.0, Z)
    e = torch.where(child, e, 0.0)
    # weight of the siblings ahead of a node: those stand side by side
    ahead = e.cumsum(1) - e
    first = torch.full((B, N), N, dtype=torch.int64, device="cuda").scatter_reduce_(1, par, torch.where(child, i, N), "amin")
    ahead = ahead - ahead.gather(1, first.gather(1, par).clamp(max=N - 1))
    ok = child & (s["uniform"].double() * (Z.gather(1, par) - ahead) < e)
    taken = torch.full((B, N), N, dtype=torch.int64, device="cuda").scatter_reduce_(1, par, torch.where(ok, i, N), "amin")
    chosen = (child & (taken.gather(1, par) == i)) | (i == 0)[None, :]
    # on the path: chosen, and all ancestors too
    bits = ((s["mask"][:, :, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).view(B, N, -1)[:, :, :N] > 0
    on = alive & ~(bits & ~chosen[:, None, :]).any(-1)
    accept_len = on.sum(1) - 1
    path = torch.full((B, MAX_DEPTH + 1), -1, dtype=torch.int64, device="cuda")
    path.scatter_(1, torch.where(on & child, s["depth"] - 1, MAX_DEPTH).long(), torch.where(on & child, i, -1))
    last = torch.where(on, i, 0).amax(1)
    zl = z[torch.arange(B, device="cuda"), last].double()
    w = ((zl - zl.amax(1, keepdim=True)) / inv[:, None].double()).exp()
    w = torch.nn.functional.pad(w, (0, 1))
    w.scatter_(1, torch.where(child & (par == last[:, None]), tok, V), 0.0)
    cdf = w[:, :V].cumsum(1)
    bonus = (cdf <= s["uniform"][:, :1].double() * cdf[:, -1:]).sum(1)
    bonus = torch.where(greedy, best.gather(1, last[:, None])[:, 0], bonus.clamp(max=V - 1))
    for t, x in (("accept_len", accept_len), ("accept_path", path[:, :MAX_DEPTH]), ("bonus", bonus)):
        s[t].copy_(x)
    return dict(accept_len=s["accept_len"], accept_path=s["accept_path"], bonus=s["bonus"])


def _run_cache(s):
    if own:
        g, cache = s["graft"], _own_cache(s)
        g.cache_write(cache, 0, s["table"], s["prefix_len"], s["count"], s["key"], s["value"])
        g.cache_read(cache, 0, s["table"], s["prefix_len"], s["count"], s["key_back"], s["value_back"])
        return dict(key=s["key_back"], value=s["value_back"])
    B, N = s["B"], s["N"]
    i = torch.arange(N, device="cuda")
    slots = (s["prefix_len"] - 1)[:, None] + i
    alive = i[None, :] < s["count"][:, None]
    page = s["table"].gather(1, slots.clamp(max=s["table"].shape[1] * s["page"] - 1) // s["page"]).long()
    p, at = page[alive], (slots % s["page"])[alive]
    for x, into, exps, back in ((s["key"], s["k"], s["k_exp"], s["key_back"]), (s["value"], s["v"], s["v_exp"], s["value_back"])):
        rows = x[alive]
        if exps is None:
            into[0][p, :, at] = rows
            back[alive] = into[0][p, :, at]
        else:
            y, e = _quantise(rows)
            into[0].view(torch.uint8)[p, :, at] = y.view(torch.uint8)
            exps[0][p, :, at] = e
            got = into[0].view(torch.uint8)[p, :, at].view(torch.float8_e4m3fn)
            back[alive] = _values(got, exps[0][p, :, at]).to(torch.bfloat16)
    return dict(key=s["key_back"], value=s["value_back"])


def _run_keep(s):
    if own:
        s["graft"].cache_keep(_own_cache(s), s["table"], s["prefix_len"], s["accept_len"], s["accept_path"], s["next_prefix"])
        return dict(k=s["k"], v=s["v"], next_prefix=s["next_prefix"])
    step = torch.arange(MAX_DEPTH, device="cuda")
    taken = step[None, :] < s["accept_len"][:, None]
    base = (s["prefix_len"] - 1)[:, None]
    src, dst = (base + s["accept_path"])[taken], (base + 1 + step)[taken]
    b = torch.arange(s["B"], device="cuda")[:, None].expand(-1, MAX_DEPTH)[taken]
    ps, pd = s["table"][b, src // s["page"]].long(), s["table"][b, dst // s["page"]].long()
    for x in (s["k"], s["v"]):
        x[:, pd, :, dst % s["page"]] = x[:, ps, :, src % s["page"]]
    s["next_prefix"].copy_(s["prefix_len"] + s["accept_len"] + 1)
    return dict(k=s["k"], v=s["v"], next_prefix=s["next_prefix"])


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    B = c["batch"]
    if c["kind"] == "verify":
        esz = 2 if c["dtype"] == "bf16" else 4
        nodes = (c["min_nodes"] + c["nodes"]) / 2
        # rows of the nodes on the path, the root's among them: about three, and five or six of a cooler target
        visited = min(3.0 if c["temperature"] >= 1 else 5.5, nodes)
        return dict(bytes=B * visited * c["V"] * esz + B * nodes * 12, flops=B * visited * c["V"] * 3)
    esz = 2 if c.get("dtype", "bf16") == "bf16" else 1 + 1 / c["head_dim"]
    row = c["kv_heads"] * c["head_dim"]
    if c["kind"] == "attention":
        n = (c["min_nodes"] + c["nodes"]) / 2
        own_slots = (c["len_lo"] + c["len_hi"]) / 2 - 1 - c["shared"]
        slots = c["shared"] + B * (own_slots + n)
        q_row = c["q_heads"] * c["head_dim"]
        seen = c["shared"] + own_slots + min(n, MAX_DEPTH) / 2
        return dict(bytes=2 * slots * row * esz + B * n * q_row * 4 + B * n * c["q_heads"] * 4,
                    flops=4 * B * n * seen * q_row)
    if c["kind"] == "cache":
        n = (c["min_rows"] + c["rows"]) / 2
        return dict(bytes=2 * B * n * row * (2 + 2 * esz + 2), flops=0)
    moved = B * min(MAX_DEPTH / 2, c["nodes"] - 1)
    return dict(bytes=c["layers"] * 2 * moved * row * 2 * 2, flops=0)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "verify": _exact_verify, "cache": _exact_cache, "keep": _exact_keep}[case["kind"]](s)


def _entry(x, exp, page, at):
    """One sequence's entries at places [S] of pages [S] -> [S, Hk, D], fp64."""
    y = x[0][page, :, at].double()
    if exp is not None:
        e = exp[0][page, :, at].double()
        y = y * torch.where(e == 255, float("nan"), 2.0 ** (e - 127))[..., None]
    return y


def _exact_attention(s):
    out, lse = s["out"].double(), s["lse"].double()
    G = s["Hq"] // s["Hk"]
    mask = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    for b in range(s["B"]):
        n, base = int(s["n_nodes"][b]), int(s["prefix_len"][b]) - 1
        slot = torch.arange(base + n, device="cuda")
        page, at = s["table"][b].long()[slot // s["page"]], slot % s["page"]
        k, v = _entry(s["k"], s["k_exp"], page, at), _entry(s["v"], s["v_exp"], page, at)
        if mask is None:
            tree = np.tril(np.ones((n, n), bool))
        else:
            tree = np.array([[(mask[b, i, j // 32] >> (j % 32)) & 1 for j in range(n)] for i in range(n)], bool)
        hide = torch.zeros((n, base + n), dtype=torch.bool, device="cuda")
        hide[:, base:] = torch.from_numpy(~tree).cuda()
        for h in range(s["Hq"]):
            sc = s["q"][b, :n, h].double() @ k[:, h // G].T / math.sqrt(s["D"])
            sc = sc.masked_fill(hide, -math.inf)
            lse[b, :n, h] = torch.logsumexp(sc, 1)
            out[b, :n, h] = torch.softmax(sc, 1) @ v[:, h // G]
    return dict(out=out, lse=lse)


def _exact_verify(s):
    B, V = s["B"], s["V"]
    n_nodes, parent, token, T, u = (s[k].cpu().numpy() for k in ("n_nodes", "parent", "token", "temperature", "uniform"))
    length, path, bonus = np.zeros(B, np.int32), np.full((B, MAX_DEPTH), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        cur, a = 0, 0
        while True:
            z = s["logits"][b, cur].double().cpu().numpy()
            if T[b] == 0:
                w = np.zeros(V)
                w[np.argmax(z)] = 1.0
            else:
                w = np.exp((z - z.max()) / float(T[b]))
            nxt = -1
            for c in range(1, n_nodes[b]):
                if parent[b, c] == cur:
                    if float(u[b, c]) * w.sum() < w[token[b, c]]:
                        nxt = c
                        break
                    w[token[b, c]] = 0.0
            if nxt < 0:
                break
            path[b, a] = nxt
            a, cur = a + 1, nxt
        length[b] = a
        cdf = np.cumsum(w)
        bonus[b] = min(int(np.searchsorted(cdf, float(u[b, 0]) * cdf[-1], side="right")), V - 1)
    return dict(accept_len=length, accept_path=path, bonus=bonus)


def _exact_cache(s):
    back = []
    for x, into in ((s["key"], s["key_back"]), (s["value"], s["value_back"])):
        y = x.double()
        if s["k_exp"] is not None:
            amax = y.abs().amax(-1, keepdim=True)
            # amax / 448 = m 2^x with m in [0.5, 1): the power of two at or above it
            m, x2 = torch.frexp(amax / 448)
            scale = torch.ldexp(torch.ones_like(m), torch.where(m == 0.5, x2 - 1, x2).clamp(-120, 120))
            t = (y / scale).abs()
            # e4m3: three bits behind the leading one, multiples of 2^-9 at least, ties to even
            unit = torch.ldexp(torch.ones_like(t), torch.frexp(t.clamp(min=2.0 ** -6))[1] - 4)
            y = torch.sign(y) * torch.round(t / unit) * unit * scale
        alive = torch.arange(s["N"], device="cuda")[None, :] < s["count"][:, None]
        back.append(torch.where(alive[:, :, None, None], y, into.double()))
    return dict(key=back[0], value=back[1])


def _exact_keep(s):
    k, v = s["k"].double(), s["v"].double()
    length, path, prefix, table = (s[t].cpu().numpy() for t in ("accept_len", "accept_path", "prefix_len", "table"))
    for b in range(s["B"]):
        for i in range(length[b]):
            src, dst = prefix[b] - 1 + path[b, i], prefix[b] + i
            ps, pd = table[b, src // s["page"]], table[b, dst // s["page"]]
            for x in (k, v):
                x[:, pd, :, dst % s["page"]] = x[:, ps, :, src % s["page"]]
    return dict(k=k, v=v, next_prefix=prefix + length + 1)
