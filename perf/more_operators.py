"""What a target layer with rotary positions and a sliding window needs of its cache, as cases that can be timed and compared.

Three kinds, every one through the package's public entry points:

  append  queries and keys rotated by their positions (one axis, or time, height and width), keys and values written into a paged
          cache, quantised as they are written: Graft.cache_append
  window  attention over the cache of rows that see the last `window` positions and the first `sinks`: single tokens, the nodes of
          trees, chunks of prompts: Graft.window_attention
  layer   the one behind the other, as a layer of the target calls them

`own` False: the same in elementary torch operations.  Sequence b's slot s lives in page table[b, s // page_size]; row i of a call
sits in slot prefix_len[b] - 1 + i (row 0 is the last committed token).
"""
import functools
import math

import numpy as np
import torch

own = False

MAX_DEPTH = 16  # block length of the drafter


# ---- cases ---------------------------------------------------------------------------------------------------------
def _append(name, batch, rows, q_heads, kv_heads, head_dim, rot_dim, len_lo, len_hi, min_rows=1, page=64, dtype="bf16", axes=1,
            interleaved=False, tree=False, base=500000.0):
    return dict(name=name, kind="append", batch=batch, rows=rows, min_rows=min_rows, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, rot_dim=rot_dim, len_lo=len_lo, len_hi=len_hi, page=page, dtype=dtype, axes=axes,
                interleaved=interleaved, tree=tree, base=base)


def _window(name, batch, rows, q_heads, kv_heads, head_dim, len_lo, len_hi, window, sinks=4, min_rows=1, page=64, dtype="bf16",
            tree=False):
    return dict(name=name, kind="window", batch=batch, rows=rows, min_rows=min_rows, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, len_lo=len_lo, len_hi=len_hi, window=window, sinks=sinks, page=page, dtype=dtype, tree=tree)


def _layer(name, batch, rows, q_heads, kv_heads, head_dim, len_lo, len_hi, window, sinks=4, min_rows=1, page=64, dtype="bf16",
           tree=False, axes=1):
    c = _append(name, batch, rows, q_heads, kv_heads, head_dim, head_dim, len_lo, len_hi, min_rows, page, dtype, axes, False, tree)
    return dict(c, kind="layer", window=window, sinks=sinks)


def listed():
    return [
        # one user, the tree of a fixed budget of 64 nodes: latency
        _append("append_b1_n65", 1, 65, 32, 8, 128, 128, 1500, 1500, min_rows=65, tree=True),
        # the nodes of a serving batch's trees into a quantised cache, and back
        _append("append_b64_n65_e4m3", 64, 65, 32, 8, 128, 128, 500, 4096, min_rows=17, dtype="e4m3", tree=True),
        # prompts of unlike lengths into an empty cache: bytes
        _append("append_b8_prompt8192", 8, 8192, 32, 8, 128, 128, 1, 1, min_rows=1000),
        # prompts with pictures and clips, positions of three axes, half of every head rotated, neighbours paired
        _append("append_b4_clips4096_axes3", 4, 4096, 28, 4, 128, 64, 1, 1, min_rows=2500, axes=3, interleaved=True, base=1000000.0),
        # one user far into a conversation, a token at a time: latency
        _window("window_b1_n1_w4096", 1, 1, 32, 8, 128, 30001, 30001, 4096),
        # single tokens of a full server, a quantised cache: bytes
        _window("window_b64_n1_w4096_e4m3", 64, 1, 32, 8, 128, 2000, 32000, 4096, dtype="e4m3"),
        # an ordinary serving batch, trees of unlike sizes, a short window
        _window("window_b32_n65_w1024", 32, 65, 32, 8, 128, 500, 9000, 1024, min_rows=17, tree=True),
        # the largest budgets behind a long window, a quantised cache, small heads
        _window("window_b16_n513_w4096_d64_e4m3", 16, 513, 32, 8, 64, 3000, 20000, 4096, min_rows=257, dtype="e4m3", tree=True),
        # prompts of unlike lengths, a short window: operations
        _window("window_b4_prompt8192_w1024", 4, 8192, 32, 8, 128, 1, 1, 1024, min_rows=3000),
        # one long prompt behind an earlier part of it, a window that divides by nothing, no sinks
        _window("window_b1_prompt12000_w4001", 1, 12000, 28, 4, 128, 4097, 4097, 4001, sinks=0, min_rows=12000),
        # a layer of the target for single tokens
        _layer("layer_b48_n1_w2048", 48, 1, 32, 8, 128, 100, 16000, 2048),
        # and for trees, quantised
        _layer("layer_b24_n65_w2048_e4m3", 24, 65, 32, 4, 128, 300, 16000, 2048, min_rows=17, dtype="e4m3", tree=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append"] * 4 + ["window"] * 6 + ["layer"] * 3)
    page = rng.choice([16, 32, 64, 64, 128, 256])
    dtype = rng.choice(["bf16", "e4m3"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    head_dim = rng.choice([64, 128, 128])
    q_heads = kv_heads * rng.choice([1, 4, 4, 5, 7, 8])
    form = rng.choice(["token", "tree", "tree", "chunk"])
    rows = dict(token=1, tree=rng.choice([rng.randint(2, 65), _log_uniform(rng, 2, 513)]), chunk=_log_uniform(rng, 2, 8192))[form]
    # no more numbers than the largest listed one
    most = 8 * 4600 * 48 * 128 // (rows * (q_heads + 2 * kv_heads) * head_dim)
    if kind == "append":
        batch = _log_uniform(rng, 1, max(1, min(128, most)))
        axes = rng.choice([1, 1, 3])
        c = _append("", batch, rows, q_heads, kv_heads, head_dim, rng.choice([head_dim, head_dim, head_dim // 2, 32]), 1,
                    rng.choice([1, _log_uniform(rng, 2, 100000)]) if rows < 8192 else 1, rng.randint(1, rows), page, dtype, axes,
                    rng.random() < 0.3, form == "tree" and axes == 1, rng.choice([10000.0, 500000.0]))
    else:
        window = rng.choice([128, 512, 1024, 4096, _log_uniform(rng, 16, 4096)])
        hi = 1 if form == "chunk" and rng.random() < 0.5 else _log_uniform(rng, 64, 32000)
        # no more key rows and no more products than the largest listed ones
        most = min(64, most, 64 * 4096 * 8 // (min(window, hi + rows) * kv_heads), 4 * 5600 * 32 * 1024 // (rows * q_heads * min(window, hi + rows)))
        batch = _log_uniform(rng, 1, max(1, most))
        args = (batch, rows, q_heads, kv_heads, head_dim, rng.choice([1, max(1, hi // 2), hi]), hi, window, rng.choice([0, 4, 4, rng.randint(1, 128)]),
                rng.randint(1, rows), page, dtype, form == "tree")
        c = _layer("", *args, axes=rng.choice([1, 1, 3])) if kind == "layer" else _window("", *args)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------
def _spread(rng, lo, hi, n):
    """n whole numbers spread evenly over lo..hi, in random order."""
    return rng.permutation(np.rint(np.linspace(lo, hi, n)) if n > 1 else np.array([hi])).astype(np.int32)


def _trees(rng, n_nodes, nmax):
    """Trees in level order, no deeper than MAX_DEPTH: depths [B, nmax] (-1 behind a tree), ancestor-or-self masks [B, nmax, W] as bits."""
    B, W = len(n_nodes), (nmax + 31) // 32
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
            depth[b, i] = d
            mask[b, i] = mask[b, p]
            mask[b, i, i // 32] |= (np.uint32(1) << (i % 32).astype(np.uint32))
    return depth, mask.view(np.int32)


def _axes3(rng, B, N):
    """Positions of text with pictures and clips in it, [B, N, 3]: text counts on along all axes, frames of h x w patches have a time,
    a row and a column; what follows counts on behind the largest of them."""
    pos = np.zeros((B, N, 3), np.int32)
    for b in range(B):
        i, p = 0, 0
        while i < N:
            n = int(min(rng.integers(20, 300), N - i))
            pos[b, i:i + n] = (p + np.arange(n))[:, None]
            i, p = i + n, p + n
            t, h, w = int(rng.choice([1, 1, 4, 8])), int(rng.integers(8, 24)), int(rng.integers(8, 24))
            grid = np.stack(np.meshgrid(np.arange(t), np.arange(h), np.arange(w), indexing="ij"), -1).reshape(-1, 3)[:N - i]
            pos[b, i:i + len(grid)] = p + grid
            i, p = i + len(grid), p + max(t, h, w)
    return pos


def _table(rng, batch, width, used):
    """Page numbers [batch, width]: pages apart for the places that are used, -1 (given back) elsewhere; and how many pages there are."""
    n = int(used.sum())
    t = np.full((batch, width), -1, np.int32)
    t[used] = rng.permutation(n).astype(np.int32)
    return t, n


def _heads(gen, shape):
    """Keys as models have them: N(0, 1) with a few channels that are several times larger."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    x[..., 3::37] *= 3
    return x


@functools.lru_cache(maxsize=8)
def _context(nmax, batch):
    from paper_2608_20375_b200 import Graft
    return Graft(64, MAX_DEPTH, 4, 16, 8, batch, 1, nmax - 1, 1, 0.0)


def prepare(case, seed):
    c = case
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    B, N, Hq, Hk, D, page = c["batch"], c["rows"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    count = _spread(rng, c["min_rows"], N, B)
    lens = _spread(rng, c["len_lo"], c["len_hi"], B)  # prefix lengths, the last committed token included
    depth, mask = _trees(rng, count, N) if c["tree"] else (None, None)
    position = None if depth is None else lens[:, None] - 1 + np.maximum(depth, 0)
    width = -(-(c["len_hi"] - 1 + N) // page)
    # pages that a row may see or is written to; a server takes back those that fell behind the window
    first = np.arange(width)[None, :] * page
    seen_from = lens[:, None] - c.get("window", 1 if c["kind"] == "append" else 0)
    used = ((first + page > seen_from) & (first < (lens + count)[:, None] - 1)) | (first < c.get("sinks", 0))
    table, n_pages = _table(rng, B, width, used)
    # a fused projection, as it comes out of one matrix product
    fused = torch.empty((B, N, (Hq + 2 * Hk) * D), dtype=torch.bfloat16, device="cuda")
    q, key, value = (x.view(B, N, -1, D) for x in fused.split([Hq * D, Hk * D, Hk * D], 2))
    q.copy_(torch.randn(q.shape, generator=gen, device="cuda", dtype=torch.bfloat16))
    q[..., 5::16] += 1  # what rows have in common, and the first tokens' keys answer to
    key.copy_(_heads(gen, key.shape))
    value.copy_(torch.randn(value.shape, generator=gen, device="cuda", dtype=torch.bfloat16))
    s = dict(kind=c["kind"], B=B, N=N, Hq=Hq, Hk=Hk, D=D, page=page, q=q, key=key, value=value, count=dev(count), prefix_len=dev(lens),
             table=dev(table), mask=None if mask is None else dev(mask), window=c.get("window"), sinks=c.get("sinks"),
             position=None if position is None else dev(position.astype(np.int32)), q8=c["dtype"] == "e4m3")
    shape = (1, n_pages, Hk, page, D)
    if c["kind"] == "append":
        k, v = torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    else:
        k, v = _heads(gen, shape), torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
        heads = table[:, :1][table[:, :1] >= 0]
        k[:, dev(heads).long(), :, :min(c["sinks"], page), 5::16] += 4
    s.update(k=k, v=v, k_exp=None, v_exp=None)
    if s["q8"]:
        (s["k"], s["k_exp"]), (s["v"], s["v_exp"]) = _quantise(k), _quantise(v)
    if c["kind"] != "window":
        pairs = c["rot_dim"] // 2
        freq = c["base"] ** -(np.arange(pairs) / pairs)
        s["freq"] = dev(freq[None, :].astype(np.float32))
        s["shift"] = None
        if c["axes"] == 3:  # a quarter of the pairs turn with time, the others with the row and the column
            axis = np.searchsorted([pairs // 4, pairs // 4 + 3 * pairs // 8], np.arange(pairs), side="right")
            s["freq"] = dev(np.where(axis[None, :] == np.arange(3)[:, None], freq[None, :], 0.0).astype(np.float32))
            # (pictures take fewer positions than slots: the first row's is given apart)
            s["position"] = dev(_axes3(rng, B, N)) if position is None else s["position"]
            s["shift"] = dev((lens - 1 if position is None else -(lens // 3)).astype(np.int32))
        s["interleaved"] = c["interleaved"]
        s["q_rot"] = torch.zeros((B, N, Hq, D), dtype=torch.bfloat16, device="cuda")
        if c["kind"] == "append" and s["q8"]:
            s["key_back"], s["value_back"] = (torch.zeros((B, N, Hk, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if c["kind"] != "append":
        s["out"] = torch.zeros((B, N, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((B, N, Hq), dtype=torch.float32, device="cuda")
    if own:
        from paper_2608_20375_b200 import KVCache, Rope
        s["graft"] = _context(max(N, 2), B) if mask is not None else _context(2, B)
        s["cache"] = KVCache(s["k"], s["v"], s["k_exp"], s["v_exp"])
        if c["kind"] != "window":
            s["rope"] = Rope(s["freq"], interleaved=s["interleaved"], shift=s["shift"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return {"append": _run_append, "window": _run_window, "layer": _run_layer}[s["kind"]](s)


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


def _slot_position(s):
    """Positions of the rows [B, N] where none are given: their slots."""
    return (s["prefix_len"] - 1)[:, None] + torch.arange(s["N"], device="cuda")


def _rotate(s, x):
    """x [B, N, heads, D] with its first numbers turned by their positions' angles, fp32."""
    pos = _slot_position(s) if s["position"] is None else s["position"]
    if pos.dim() == 2:
        pos = pos[..., None]
    if s["shift"] is not None:
        pos = pos + s["shift"][:, None, None]
    angle = (pos.double()[..., None] * s["freq"].double()).sum(2)[:, :, None, :]  # [B, N, 1, pairs]
    cos, sin = angle.cos().float(), angle.sin().float()
    pairs = s["freq"].shape[1]
    x = x.float()
    turned, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    if s["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = turned[..., :pairs], turned[..., pairs:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, rest), -1)


def _run_append(s):
    if own:
        g = s["graft"]
        g.cache_append(s["cache"], 0, s["table"], s["prefix_len"], s["count"], s["rope"], s["q"], s["key"], s["value"], s["q_rot"],
                       position=s["position"])
        if s["kind"] == "append" and s["q8"]:
            g.cache_read(s["cache"], 0, s["table"], s["prefix_len"], s["count"], s["key_back"], s["value_back"])
            return dict(q=s["q_rot"], key=s["key_back"], value=s["value_back"])
        return dict(q=s["q_rot"], k=s["k"], v=s["v"])
    alive = torch.arange(s["N"], device="cuda")[None, :] < s["count"][:, None]
    slots = _slot_position(s)
    page = s["table"].gather(1, slots.clamp(max=s["table"].shape[1] * s["page"] - 1) // s["page"]).long()
    p, at = page[alive], (slots % s["page"])[alive]
    s["q_rot"].copy_(torch.where(alive[:, :, None, None], _rotate(s, s["q"]).to(torch.bfloat16), s["q_rot"]))
    for name, x, into, exps in (("key_back", _rotate(s, s["key"]), s["k"], s["k_exp"]), ("value_back", s["value"], s["v"], s["v_exp"])):
        rows = x[alive]
        if exps is None:
            into[0][p, :, at] = rows.to(torch.bfloat16)
            continue
        y, e = _quantise(rows)
        into[0].view(torch.uint8)[p, :, at] = y.view(torch.uint8)
        exps[0][p, :, at] = e
        if s["kind"] == "append":
            got = into[0].view(torch.uint8)[p, :, at].view(torch.float8_e4m3fn)
            s[name][alive] = _values(got, exps[0][p, :, at]).to(torch.bfloat16)
    if s["kind"] == "append" and s["q8"]:
        return dict(q=s["q_rot"], key=s["key_back"], value=s["value_back"])
    return dict(q=s["q_rot"], k=s["k"], v=s["v"])


def _run_window(s, q=None):
    q = s["q"] if q is None else q
    if own:
        s["graft"].window_attention(s["cache"], 0, s["table"], q, s["prefix_len"], s["count"], s["mask"],
                                    None if s["mask"] is None else s["position"], s["window"], s["sinks"], s["out"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    B, N, Hq, Hk, D, sinks = s["B"], s["N"], s["Hq"], s["Hk"], s["D"], s["sinks"]
    G, S = Hq // Hk, s["table"].shape[1] * s["page"]
    window = min(s["window"], S + N)
    base = (s["prefix_len"] - 1)[:, None]
    # rows in blocks, each against the slots that its first row's window begins with up to its last row's own, and the sinks before them
    Q = N if s["mask"] is not None else min(N, max(window, 128))
    blocks = -(-N // Q)
    first = base + torch.arange(blocks, device="cuda") * Q - (window - 1)
    last = window - 1 + Q
    slot = torch.cat((first[:, :, None] + torch.arange(last, device="cuda"),
                      torch.arange(sinks, device="cuda").expand(B, blocks, sinks)), 2)
    there = (slot >= 0) & (slot < base[:, :, None] + s["count"][:, None, None])
    there[:, :, last:] &= slot[:, :, last:] < first[:, :, None]
    page = s["table"].gather(1, (slot.clamp(0, S - 1) // s["page"]).view(B, -1)).clamp(min=0).long().view(slot.shape)
    at = slot.clamp(0, S - 1) % s["page"]
    k, v = (_values(x[0][page, :, at], None if e is None else e[0][page, :, at]).transpose(2, 3)
            for x, e in ((s["k"], s["k_exp"]), (s["v"], s["v_exp"])))  # [B, blocks, Hk, slots, D]
    pad = blocks * Q - N
    q = torch.nn.functional.pad(q.float(), (0, 0, 0, 0, 0, pad)).view(B, blocks, Q, Hk, G, D).permute(0, 1, 3, 2, 4, 5)
    sc = (q.reshape(B, blocks, Hk, Q * G, D) @ k.transpose(3, 4)).view(B, blocks, Hk, Q, G, -1)
    sc *= D ** -0.5
    own_slot = base + torch.arange(blocks * Q, device="cuda")
    if s["mask"] is None:
        far = own_slot.view(B, blocks, Q, 1) - slot[:, :, None, :]
        seen = there[:, :, None, :] & (far >= 0) & ((far < s["window"]) | (slot < sinks)[:, :, None, :])
    else:
        pos = s["position"]
        j = slot - base[:, :, None]
        bits = ((s["mask"][:, :, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).view(B, N, -1)
        bit = bits.gather(2, j.clamp(0, bits.shape[2] - 1).expand(B, N, -1)) > 0
        slot_pos = torch.where(j < 0, slot, pos.gather(1, j.clamp(0, N - 1).view(B, -1)).view(slot.shape))
        near = (pos[:, :, None] - slot_pos < s["window"]) | (slot_pos < sinks)
        seen = (there & ((j < 0) | bit) & near)[:, None]
    sc.masked_fill_(~seen[:, :, None, :, None, :], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top = top.masked_fill(top == float("-inf"), 0.0)
    sc.sub_(top).exp_()
    total = sc.sum(-1, keepdim=True)
    o = (sc.view(B, blocks, Hk, Q * G, -1) @ v).view(B, blocks, Hk, Q, G, D) / total
    rows = lambda x: x.permute(0, 1, 3, 2, 4, 5).reshape(B, blocks * Q, Hq, -1)[:, :N]  # noqa: E731
    alive = (torch.arange(N, device="cuda")[None, :] < s["count"][:, None])[:, :, None]
    s["out"].copy_(torch.where(alive[..., None], rows(o).to(torch.bfloat16), s["out"]))
    s["lse"].copy_(torch.where(alive, rows(top + total.log())[..., 0], s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


def _run_layer(s):
    new = _run_append(s)
    done = _run_window(s, new["q"])
    return dict(done, q=new["q"])


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    B, Hq, Hk, D = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    n = (c["min_rows"] + c["rows"]) / 2 if B > 1 else c["rows"]
    esz = 2 if c["dtype"] == "bf16" else 1 + 1 / D
    need = dict(bytes=0.0, flops=0.0)
    if c["kind"] != "window":
        need["bytes"] += B * n * D * (Hq * 4 + 2 * Hk * (2 + esz))
        need["flops"] += B * n * 3 * (Hq + Hk) * c["rot_dim"]
        if c["kind"] == "append" and c["dtype"] == "e4m3":
            need["bytes"] += B * n * D * 2 * Hk * (2 + esz)
    if c["kind"] != "append":
        before = (c["len_lo"] + c["len_hi"]) / 2 - 1
        # slots that a row sees: as many as the window holds, or as there are
        depth = min(n, MAX_DEPTH) / 2 if c["tree"] else n / 2
        seen = min(c["window"] + c["sinks"], before + depth + 1)
        if not c["tree"] and before < c["window"]:  # (the first rows of a prompt see fewer)
            short = min(n, c["window"] - before)
            seen = (short * (before + short / 2) + (n - short) * min(c["window"] + c["sinks"], before + n)) / n
        slots = min(c["window"] + c["sinks"], before) + n
        need["bytes"] += B * (2 * slots * Hk * D * esz + n * Hq * (4 * D + 4))
        need["flops"] += 4 * B * n * seen * Hq * D
    return need


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "window":
        return _exact_window(s, s["q"])
    done = _exact_append(s)
    if s["kind"] == "append":
        return done
    # (the queries that attention is given are those that were rounded on the way; entries of the cache likewise)
    return dict(_exact_window(s, done["q"].to(torch.bfloat16)), q=done["q"])


def _exact_turned(s, x, b):
    """One sequence's heads [N, heads, D] as complex numbers times e^(i angle), fp64."""
    x = x[b].double()
    i = torch.arange(s["N"], device="cuda", dtype=torch.float64)
    angle = torch.zeros((s["N"], s["freq"].shape[1]), dtype=torch.float64, device="cuda")
    for a in range(s["freq"].shape[0]):
        if s["position"] is None:
            p = i + (int(s["prefix_len"][b]) - 1)
        else:
            p = (s["position"][b] if s["position"].dim() == 2 else s["position"][b, :, a]).double()
        if s["shift"] is not None:
            p = p + int(s["shift"][b])
        angle += p[:, None] * s["freq"][a].double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
    P = angle.shape[1]
    y = x.clone()
    if s["interleaved"]:
        z = torch.view_as_complex(x[..., :2 * P].reshape(*x.shape[:-1], P, 2).contiguous()) * turn
        y[..., 0:2 * P:2], y[..., 1:2 * P:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :P], x[..., P:2 * P]) * turn
        y[..., :P], y[..., P:2 * P] = z.real, z.imag
    return y


def _held(y):
    """What rows of fp64 numbers are as e4m3 numbers with a power of two a row."""
    amax = y.abs().amax(-1, keepdim=True)
    # amax / 448 = m 2^x with m in [0.5, 1): the power of two at or above it
    m, x2 = torch.frexp(amax / 448)
    scale = torch.ldexp(torch.ones_like(m), torch.where(m == 0.5, x2 - 1, x2).clamp(-120, 120))
    t = (y / scale).abs()
    # e4m3: three bits behind the leading one, multiples of 2^-9 at least, ties to even
    unit = torch.ldexp(torch.ones_like(t), torch.frexp(t.clamp(min=2.0 ** -6))[1] - 4)
    return torch.sign(y) * torch.round(t / unit) * unit * scale


def _exact_append(s):
    q = s["q_rot"].double()
    q8 = s["q8"]
    k, v = (x.double() if not q8 else None for x in (s["k"], s["v"]))
    back = [torch.zeros(s["key"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    for b in range(s["B"]):
        n, base = int(s["count"][b]), int(s["prefix_len"][b]) - 1
        q[b, :n] = _exact_turned(s, s["q"], b)[:n]
        new = _exact_turned(s, s["key"], b)[:n], s["value"][b, :n].double()
        slot = torch.arange(base, base + n, device="cuda")
        page, at = s["table"][b].long()[slot // s["page"]], slot % s["page"]
        for x, into, held, y in zip(back, (k, v), ((s["k"], s["k_exp"]), (s["v"], s["v_exp"])), new):
            x[b, :n] = _held(y) if q8 else y
            if not q8:
                into[0, page, :, at] = y
            if s["kind"] == "layer":  # what attention then reads
                if q8:
                    z, e = _quantise(y)
                    held[0][0].view(torch.uint8)[page, :, at] = z.view(torch.uint8)
                    held[1][0][page, :, at] = e
                else:
                    held[0][0][page, :, at] = y.to(torch.bfloat16)
    return dict(q=q, key=back[0], value=back[1]) if q8 else dict(q=q, k=k, v=v)


def _exact_window(s, q):
    out, lse = s["out"].double(), s["lse"].double()
    G = s["Hq"] // s["Hk"]
    mask = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    for b in range(s["B"]):
        n, base = int(s["count"][b]), int(s["prefix_len"][b]) - 1
        begin = max(0, base - s["window"] + 1)  # nothing between the sinks and this slot is seen by any row
        slot = torch.cat((torch.arange(min(s["sinks"], begin), device="cuda"), torch.arange(begin, base + n, device="cuda")))
        page, at = s["table"][b].long()[slot // s["page"]], slot % s["page"]
        k, v = (x[0][page, :, at].double() for x in (s["k"], s["v"]))
        if s["q8"]:
            k, v = (x * torch.ldexp(torch.ones_like(e[0][page, :, at], dtype=torch.float64), e[0][page, :, at].int() - 127)[..., None]
                    for x, e in ((k, s["k_exp"]), (v, s["v_exp"])))
        if mask is None:
            row_pos, slot_pos = base + torch.arange(n, device="cuda"), slot
            hide = slot[None, :] > row_pos[:, None]
        else:
            row_pos = s["position"][b, :n]
            slot_pos = torch.where(slot < base, slot, row_pos[(slot - base).clamp(0)])
            tree = np.array([[(mask[b, i, j // 32] >> (j % 32)) & 1 for j in range(n)] for i in range(n)], bool)
            hide = torch.zeros((n, len(slot)), dtype=torch.bool, device="cuda")
            hide[:, len(slot) - n:] = torch.from_numpy(~tree).cuda()
        hide |= (row_pos[:, None] - slot_pos[None, :] >= s["window"]) & (slot_pos >= s["sinks"])[None, :]
        for h in range(s["Hq"]):
            sc = q[b, :n, h].double() @ k[:, h // G].T / math.sqrt(s["D"])
            sc = sc.masked_fill_(hide, -math.inf)
            lse[b, :n, h] = torch.logsumexp(sc, 1)
            out[b, :n, h] = torch.softmax(sc, 1) @ v[:, h // G]
    return dict(out=out, lse=lse)
