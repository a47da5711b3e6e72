"""The tree kernel's halves of key tiles (e4m3 slots behind a window): what the softmax's warps and the warp that issues products tell each other,
run through on the CPU in random orders.  Each half of a tile has barriers of its own for scores, weights and products with V."""
import random
import re

import pytest

from test_verifier_protocols import _kernel

WARPS = 4  # of a stream


class _Barrier:
    """Completed phases; a wait for a parity ends when the phase under way has the other one."""

    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def passed(self, parity):
        return self.done & 1 != parity


def _wait_o(n_s, c):
    """Which part's barrier, and the parity: as the kernel's wait_o."""
    return (1, (n_s & 1) ^ 1) if c == 0 else (0, n_s & 1)


def _stream(pieces, rng, wait_o=_wait_o, p_parity=lambda n: n & 1, s_parity=lambda n: n & 1):
    """One stream along pieces of so many key tiles.  The first thing that goes wrong, or None."""
    q_full = _Barrier(WARPS + 1)
    s_full, p_full, o_done = ([_Barrier(n) for _ in range(2)] for n in (1, WARPS, 1))
    holds = [[None] * WARPS for _ in range(2)]  # of each part's columns, a warp's rows: ("scores" or "weights", tile)
    queue, wrong = [], []                       # what was issued and is not done yet: it is done in this order
    under_way = lambda: any(x[0] == "pv" for x in queue)  # noqa: E731

    def softmax(w):
        n_s = 0
        for n, tiles in enumerate(pieces):
            q_full.arrive()
            has = False
            for _ in range(tiles):
                for c in range(2):
                    yield lambda c=c: s_full[c].passed(s_parity(n_s))
                    if holds[c][w] != ("scores", n_s):
                        wrong.append(f"tile {n_s}, part {c}: the scores are {holds[c][w]}")
                    if has and rng.random() < 0.5:  # a maximum has grown: O is rescaled
                        part, parity = wait_o(n_s, c)
                        yield lambda: o_done[part].passed(parity)
                        for _ in range(3):
                            if under_way():
                                wrong.append(f"tile {n_s}, part {c}: rescaled under a product")
                            yield lambda: True
                    yield lambda: True
                    holds[c][w] = ("weights", n_s)
                    yield lambda: True
                    p_full[c].arrive()
                    has = True
                n_s += 1
            if has:
                part, parity = wait_o(n_s, 0)
                yield lambda: o_done[part].passed(parity)
                if under_way():
                    wrong.append(f"the end of piece {n}: O is read under a product")
            else:
                yield lambda: q_full.passed(n & 1)

    def products():
        n_p = 0
        for n, tiles in enumerate(pieces):
            q_full.arrive()
            yield lambda: q_full.passed(n & 1)
            for c in range(2 if tiles else 0):
                queue.extend([("qk", c, n_p), ("commit", s_full[c])])
            for t in range(tiles):
                for c in range(2):
                    yield lambda c=c: p_full[c].passed(p_parity(n_p))
                    queue.extend([("pv", c, n_p), ("commit", o_done[c])])
                    yield lambda: True
                    if t + 1 < tiles:
                        queue.extend([("qk", c, n_p + 1), ("commit", s_full[c])])
                n_p += 1

    def tensor_cores():
        kind, *rest = queue.pop(0)
        if kind == "commit":
            rest[0].arrive()
        elif kind == "qk":
            holds[rest[0]] = [("scores", rest[1])] * WARPS
        elif holds[rest[0]] != [("weights", rest[1])] * WARPS:
            wrong.append(f"tile {rest[1]}, part {rest[0]}: multiplied {holds[rest[0]]}")

    warps = {w: softmax(w) for w in range(WARPS)}
    warps["products"] = products()
    waits = {w: next(g) for w, g in warps.items()}
    while waits and not wrong:
        ready = [w for w in waits if waits[w]()] + (["tensor"] * 2 if queue else [])
        if not ready:
            return "nobody can go on"
        w = rng.choice(ready)
        if w == "tensor":
            tensor_cores()
            continue
        try:
            waits[w] = next(warps[w])
        except StopIteration:
            del waits[w]
    return wrong[0] if wrong else None


def _pieces(rng):
    return [rng.choice([0, 1, 1, 2, 3, 5]) for _ in range(rng.randrange(1, 6))]


def test_halves_are_handed_over_in_every_order():
    rng = random.Random(1)
    for _ in range(3000):
        pieces = _pieces(rng)
        assert _stream(pieces, rng) is None, pieces


@pytest.mark.parametrize("how", [
    dict(wait_o=lambda n, c: (1, n & 1) if c == 0 else (0, n & 1)),              # the first half's parity
    dict(wait_o=lambda n, c: (1, (n & 1) ^ 1) if c == 0 else (0, (n & 1) ^ 1)),  # the second half's
    dict(wait_o=lambda n, c: (c, (n & 1) ^ 1)),                                  # the same half's product, one tile back
    dict(wait_o=lambda n, c: (0, (n & 1) ^ 1) if c == 0 else (0, n & 1)),        # the other half's ahead of the first
    dict(p_parity=lambda n: (n & 1) ^ 1),
    dict(s_parity=lambda n: (n & 1) ^ 1),
])
def test_mistakes_are_found(how):
    rng = random.Random(2)
    assert any(_stream(_pieces(rng), rng, **how) for _ in range(500))


def test_the_kernel_has_these_steps():
    """The order of what is issued and told, and the barriers and parities that are waited for, as in the model."""
    k = re.sub(r"\s+", " ", _kernel("tree_attn.cu", "tree_attn_kernel"))
    assert "wait_for(o_done(i, c == 0 ? kSubs - 1 : 0), c == 0 ? (n_s & 1) ^ 1 : n_s & 1, gave_up)" in k
    assert "wait_for(s_full(i, c), n_s & 1, gave_up)" in k and "wait_for(p_full(i, c), n_p & 1, gave_up)" in k
    for name, count in (("s_full", 1), ("p_full", WARPS), ("o_done", 1)):
        assert f"mbar_init({name}(i, c), {count});" in k
    soft, issue = k[:k.index("n_turn = 0")], k[k.index("n_turn = 0"):]

    def ordered(text, *steps):
        at = 0
        for s in steps:
            assert s in text[at:], s
            at = text.index(s, at) + len(s)

    ordered(soft, "for (int c = 0; c < kSubs; ++c)", "wait_s(c)", "if (any)", "wait_o(c)", "rescale<D>", "tmem_st_32x32(tSc", "any = true;",
            "mbar_arrive(p_full(i, c))", "n_s += 1;", "if (any) ok = wait_o(0);")
    ordered(issue, "wait_for(q_full, n_piece & 1, gave_up)", "qk(c, a, bk);", "umma_commit(s_full(i, c));", "for (int t = t0; t < T; t += dt)",
            "for (int c = 0; c < kSubs; ++c)", "wait_for(p_full(i, c)", "pv(c, t == t0, bv);", "umma_commit(o_done(i, c));", "if (more) qk(c, a, bk);",
            "if (more) umma_commit(s_full(i, c));", "n_p += 1;")
