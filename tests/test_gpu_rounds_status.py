"""Rounds of a micro-batch in which something goes wrong with some of the sequences: it is reported, and those are not moved on."""
import math

import numpy as np
import pytest
import torch

from test_gpu_verifier import BF, _i32

pytestmark = pytest.mark.gpu

B, L, V, Hq, Hk, D, page, layers, pages = 4, 6, 300, 4, 2, 64, 16, 2, 5
BAD_LOGITS, BAD_CACHE = 1, 16


class _Target:
    """A micro-batch with a cache of numbers, and a target that likes what was drafted."""

    def __init__(self, greedy=False, cache=True):
        from paper_2608_20375_b200 import Graft, KVCache, MicroBatch
        self.gen = torch.Generator(device="cuda").manual_seed(9)
        self.greedy = greedy
        g = Graft(V, L, 5, 16, 8, B, 4, 24, 4, 0.0)
        table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages).flip(1).contiguous()
        c = KVCache.alloc(layers, B * pages, Hk, page, D)
        c.k.copy_(self.rand(*c.k.shape)), c.v.copy_(self.rand(*c.v.shape))
        kw = dict(cache=c, table=table, prefix_len=_i32([20, 33, 1, 47])) if cache else {}
        self.mb = MicroBatch(g, B, L, **kw)
        self.cache = cache

    def rand(self, *s):
        return torch.randn(s, generator=self.gen, device="cuda")

    def draft(self, i, r):
        x = dict(logits=(3.0 * self.rand(B, L, V)).to(BF), root_token=_i32([3, 5, 7, 9]), fixed_budget=_i32([20] * B))
        return x if self.cache else dict(x, prefix_len=_i32([20, 33, 1, 47]))

    def attend(self, layer):
        n = self.mb.graft.nmax
        q, key, value = (self.rand(B, n, h, D).to(BF) for h in (Hq, Hk, Hk))
        self.mb.attend(layer, q, key, value, torch.zeros_like(q))

    def answer(self, out, spoil=None):
        from paper_2608_20375_b200 import Sampled
        n = self.mb.graft.nmax
        z = self.rand(B, n, V)
        z.view(B, -1).scatter_add_(1, out.parent.long().clamp(0) * V + out.token.long().clamp(0), torch.where(out.parent >= 0, 12.0, 0.0))
        if spoil:
            spoil(z)
        return z.argmax(2).int() if self.greedy else Sampled(z, torch.rand((B, n), generator=self.gen, device="cuda"))

    def round(self, verify):
        from paper_2608_20375_b200 import join, run_rounds
        before = None if not self.cache else (self.mb.prefix_len.clone(), self.kept())
        run_rounds([self.mb], 1, self.draft, verify)
        join([self.mb])
        torch.cuda.synchronize()
        return before

    def kept(self):
        """Every sequence's entries of its prefix."""
        out = []
        for b in range(B):
            s = np.arange(int(self.mb.prefix_len[b]) - 1)
            p, at = self.mb.table[b][torch.from_numpy(s // page)].long(), torch.from_numpy(s % page).cuda()
            out.append(torch.stack([self.mb.cache.k[:, p, :, at], self.mb.cache.v[:, p, :, at]]))
        return out

    def check(self, before, want):
        prefix, kept = before
        assert self.mb.status.tolist() == want
        bad = torch.tensor([w != 0 for w in want], device="cuda")
        assert torch.equal(self.mb.prefix_len, torch.where(bad, prefix, prefix + self.mb.accept_len + 1))
        for b in range(B):  # the prefix is as it was, whether the sequence moved on or not
            assert torch.equal(self.kept()[b][:, :kept[b].shape[1]], kept[b])

    def well(self):
        """A round in which nothing goes wrong: statuses of the one before are gone."""
        def verify(i, r, out):
            for layer in range(layers):
                self.attend(layer)
            return self.answer(out)

        before = self.round(verify)
        self.check(before, [0] * B)
        assert int(self.mb.accept_len.sum()) > 0


def test_a_walk_that_ends_on_bad_logits_moves_nothing():
    t = _Target()

    def verify(i, r, out):
        for layer in range(layers):
            t.attend(layer)

        def spoil(z):
            z[1, 0, 17] = math.nan            # at the root
            z[3, 1:, 4] = math.inf            # where the walk comes after a step, if it comes to any
        return t.answer(out, spoil)

    before = t.round(verify)
    assert int(t.mb.accept_len[3]) > 0 and t.mb.bonus_token[3] == -1 and t.mb.bonus_token[1] == -1
    t.check(before, [0, BAD_LOGITS, 0, BAD_LOGITS])
    t.well()


@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("which", range(layers))
@pytest.mark.parametrize("again", [False, True])
def test_a_table_that_is_bad_in_one_layers_call_is_reported(which, greedy, again):
    """The layers behind it, and a second call of the same layer, find everything well: the round remembers."""
    t = _Target(greedy)

    def verify(i, r, out):
        for layer in range(layers):
            if layer == which:
                good = t.mb.table.clone()
                t.mb.table[1, 2] = B * pages
                t.attend(layer)
                t.mb.table.copy_(good)
                if again:
                    t.attend(layer)
            else:
                t.attend(layer)
        return t.answer(out)

    before = t.round(verify)
    t.check(before, [0, BAD_CACHE, 0, 0])
    t.well()


def test_nodes_that_do_not_fit_in_the_table():
    """21 nodes behind 65 slots of 80: the attention leaves the sequence out, and what would be accepted fits."""
    t = _Target()
    t.mb.prefix_len.copy_(_i32([20, 66, 1, 47]))

    def verify(i, r, out):
        for layer in range(layers):
            t.attend(layer)
        return t.answer(out)

    before = t.round(verify)
    assert 66 + int(t.mb.accept_len[1]) + 1 <= pages * page and int(t.mb.out.n_nodes[1]) == 21
    t.check(before, [0, BAD_CACHE, 0, 0])


def test_a_move_that_does_not_fit_is_reported_without_attention():
    """A verifier with an attention of its own: the move itself finds that what was accepted does not fit."""
    t = _Target(greedy=True)
    t.mb.prefix_len.copy_(_i32([20, 80, 1, 47]))  # (the last slot is the root's)
    before = t.round(lambda i, r, out: t.answer(out))
    assert int(t.mb.accept_len[1]) >= 1
    t.check(before, [0, BAD_CACHE, 0, 0])


def test_walks_without_a_cache_have_a_status():
    t = _Target(cache=False)

    def spoil(z):
        z[2, 0, 0] = math.nan

    t.round(lambda i, r, out: t.answer(out, spoil))
    assert t.mb.status.tolist() == [0, 0, BAD_LOGITS, 0]
    t.round(lambda i, r, out: t.answer(out))
    assert t.mb.status.tolist() == [0] * B


def test_rounds_captured_in_a_graph_report_too():
    """The layers' calls in a graph that is replayed inside of the round."""
    t = _Target()
    q, key, value = (t.rand(B, t.mb.graft.nmax, h, D).to(BF) for h in (Hq, Hk, Hk))
    t.mb.graft.build_trees(*(t.draft(0, 0)[k] for k in ("logits",)), None, _i32([3, 5, 7, 9]), None, t.mb.prefix_len, _i32([20] * B), t.mb.out)
    out = torch.zeros_like(q)
    t.mb.attend(0, q, key, value, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in range(layers):
            t.mb.attend(layer, q, key, value, out)
    good = t.mb.table.clone()

    def verify(i, r, trees):
        if r == 0:
            t.mb.table[2, 0] = -1
        graph.replay()
        t.mb.table.copy_(good)
        return t.answer(trees)

    before = t.round(verify)
    t.check(before, [0, 0, BAD_CACHE, 0])

    def fine(i, r, trees):
        graph.replay()
        return t.answer(trees)

    before = t.round(fine)
    t.check(before, [0] * B)


def test_attention_by_hand_leaves_its_status():
    """Outside of a round a layer's call reports what it found, as the library's calls do."""
    t = _Target()
    x = t.draft(0, 0)
    t.mb.graft.build_trees(x["logits"], None, x["root_token"], None, t.mb.prefix_len, x["fixed_budget"], t.mb.out)
    good = t.mb.table.clone()
    for layer in (0, 1, 1):
        t.mb.table[3, 1] = -1
        t.attend(layer)
        assert t.mb.status.tolist() == [0, 0, 0, BAD_CACHE]
        t.mb.table.copy_(good)
        t.attend(layer)
        assert not t.mb.status.any()
    t.well()
    t.mb.table[3, 1] = -1
    t.attend(0)
    assert t.mb.status.tolist() == [0, 0, 0, BAD_CACHE]


def test_a_cache_that_comes_after_the_micro_batch():
    """A micro-batch that was made without a cache is given one, and another of more layers: rounds report as if it had had it."""
    from paper_2608_20375_b200 import KVCache
    t = _Target()
    for more in (layers, layers + 3):
        mb = _Target(cache=False).mb
        c = KVCache.alloc(more, B * pages, Hk, page, D)
        mb.cache, mb.table, mb.prefix_len = c, t.mb.table, _i32([20, 33, 1, 47])
        t.mb, t.cache = mb, True
        t.well()

        def verify(i, r, out):
            good = t.mb.table.clone()
            t.mb.table[1, 2] = B * pages
            t.attend(more - 1)
            t.mb.table.copy_(good)
            t.attend(0)
            return t.answer(out)

        t.check(t.round(verify), [0, BAD_CACHE, 0, 0])
    t.mb.cache = KVCache.alloc(1, B * pages, Hk, page, D)
    t.check(t.round(lambda i, r, out: (t.attend(0), t.answer(out))[1]), [0] * B)
