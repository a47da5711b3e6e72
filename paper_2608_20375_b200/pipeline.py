"""Decoding rounds of several micro-batches on streams of their own.

One decoding round is draft -> build the tree -> verify -> walk, each step waiting for the one before it; the
conclusion of the paper names the idle time this leaves as future work.  Nothing in one sequence's round can
overlap, but the rounds of different sequences are independent, so the batch is split into micro-batches, each with
its own library context (scratch memory) and CUDA stream: while the target model verifies one micro-batch, the tree
builder of another runs, and the tree kernel, which keeps fewer CTAs than the GPU has SMs, shares the GPU with the
verifier's kernels.  This module only orders the calls; every step still runs in the library's kernels (the
verifier is the caller's).

A verifier may answer with the target's likeliest tokens (the greedy walk) or with its logits and random numbers (`Sampled`: the walk that
keeps the target's distribution).  A micro-batch that holds the target's key/value cache gives the verifier its attention (`attend`), and
after the walk the accepted nodes' entries are moved up behind the prefix.  What goes wrong with a sequence in any call of its round is in
the micro-batch's `status`, and such a sequence is not moved on: its prefix and entries stay as they were before the round's nodes.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Callable, Sequence

import torch

from .binding import Graft, GraftError, KVCache, TreeOut


@dataclass
class MicroBatch:
    """A context, its stream and the buffers one micro-batch's rounds write."""
    graft: Graft
    batch: int
    L: int
    stream: torch.cuda.Stream = None
    out: TreeOut = None
    accept_len: torch.Tensor = None
    accept_path: torch.Tensor = None
    bonus_token: torch.Tensor = None
    rounds_done: int = field(default=0)
    # the target's cache and its page table [batch, pages] (None: the verifier keeps its own); after every walk prefix_len [batch] is
    # moved on by the committed tokens.  status [batch]: the bits of all calls of the round, 0 when all is well (greedy walks without a
    # cache report nothing); a sequence with any is not moved on, and what the round says it accepted is not to be used
    cache: KVCache = None
    table: torch.Tensor = None
    prefix_len: torch.Tensor = None
    status: torch.Tensor = None

    def __post_init__(self):
        dev = torch.device("cuda", torch.cuda.current_device())
        if self.stream is None:
            self.stream = torch.cuda.Stream(device=dev)
        if self.out is None:
            self.out = self.graft.alloc_out(self.batch)
        i32 = torch.int32
        if self.accept_len is None:
            self.accept_len = torch.empty(self.batch, dtype=i32, device=dev)
        if self.accept_path is None:
            self.accept_path = torch.empty((self.batch, self.L), dtype=i32, device=dev)
        if self.bonus_token is None:
            self.bonus_token = torch.empty(self.batch, dtype=i32, device=dev)
        if self.cache is not None:
            if self.table is None or self.prefix_len is None:
                raise GraftError("a micro-batch with a cache has a table and prefix lengths")
        if self.status is None:
            self.status = torch.zeros(self.batch, dtype=i32, device=dev)
        self._attended = None  # layers of the round under way (None: there is none, calls are made by hand)
        self._calls = None
        if self.cache is not None:
            self._rows()

    def _rows(self):
        """A row of statuses a call: two a layer (write, attention), earlier calls of layers that were attended to again, walk, move."""
        n = 2 * self.cache.k.shape[0] + 3
        if self._calls is None or self._calls.shape[0] != n:  # (a micro-batch may be given its cache later)
            self._calls = torch.zeros((n, self.batch), dtype=torch.int32, device=self.status.device)
            self._bits = (1 << torch.arange(6, dtype=torch.int32, device=self.status.device)).view(-1, 1, 1)  # (ST_BAD_LOGITS .. ST_BAD_TREE)
        return self._calls

    def begin_round(self):
        """Forget the statuses of the round before.  run_rounds calls it, then draft and verify, then walk."""
        if self.cache is not None:
            self._rows().zero_()
            self._attended = set()

    def attend(self, layer, q, key, value, out, lse=None, scale=None, shared=0):
        """One layer of the target over this round's trees: the nodes' new entries go into the cache, q [batch, rows, q_heads, head_dim]
        sees the prefix and the nodes above its own.  Outside of a round (by hand, without begin_round) status
        is this call's."""
        if self.cache is None:
            raise GraftError("the micro-batch has no cache")
        if not 0 <= layer < self.cache.k.shape[0]:
            raise GraftError(f"layer must be below {self.cache.k.shape[0]}, got {layer}")
        calls = self._rows()
        written, attended = calls[2 * layer], calls[2 * layer + 1]
        if self._attended is not None:
            if layer in self._attended:
                calls[-3].bitwise_or_(written | attended)
            self._attended.add(layer)
        self.graft.cache_write(self.cache, layer, self.table, self.prefix_len, self.out.n_nodes, key, value, written)
        self.graft.tree_attention(self.cache, layer, self.table, q, self.prefix_len, self.out.n_nodes, self.out.mask, out, lse, scale, shared,
                                  attended)
        if self._attended is None:
            torch.bitwise_or(written, attended, out=self.status)

    def walk(self, answer):
        """The walk along this round's trees by what the verifier answered, and with a cache the move of what was accepted."""
        calls = self._rows() if self.cache is not None else None
        at = self.status if calls is None else calls[-2]
        if isinstance(answer, Sampled):
            self.graft.verify(self.out, answer.logits, answer.temperature, answer.uniform, self.accept_len, self.accept_path, self.bonus_token, at)
        else:
            self.graft.accept(self.out, answer, self.accept_len, self.accept_path, self.bonus_token)
        if calls is None:
            return
        self._attended = None
        torch.sum((calls[:-1] & self._bits).amax(1), 0, dtype=torch.int32, out=self.status)
        # (an accepted length below 0 leaves a sequence where it is; lengths are below 64)
        moved = torch.sub(self.accept_len, self.status, alpha=64)
        self.graft.cache_keep(self.cache, self.table, self.prefix_len, moved, self.accept_path, self.prefix_len, calls[-1])
        torch.where(self.status == 0, calls[-1], self.status, out=self.status)


@dataclass
class Sampled:
    """What a verifier that samples answers: the target's logits behind every node [batch, rows, V], numbers in [0, 1)
    [batch, n_max], temperatures [batch] (None: 1)."""
    logits: torch.Tensor
    uniform: torch.Tensor
    temperature: torch.Tensor = None


# draft(mb_index, round) -> dict(logits, hidden, root_token, hist, prefix_len, fixed_budget) of device tensors
DraftFn = Callable[[int, int], dict]
# verify(mb_index, round, tree_out) -> target_next [batch, n_max] int32 device tensor, or Sampled; enqueued on the current stream
VerifyFn = Callable[[int, int, TreeOut], "torch.Tensor | Sampled"]


def run_rounds(micro: Sequence[MicroBatch], n_rounds: int, draft: DraftFn, verify: VerifyFn, overlap: bool = True,
               after_round: Callable[[int, int, MicroBatch], None] | None = None) -> None:
    """Enqueue `n_rounds` rounds of every micro-batch.

    overlap=True: micro-batch i runs on micro[i].stream, so its build overlaps the others' verification.
    overlap=False: the same calls in the same order on the current stream (the sequential schedule).
    `draft` and `verify` are called with the micro-batch's stream current and must enqueue their work there.
    `after_round` (optional) is called after a micro-batch's walk was enqueued, e.g. to copy results aside.
    The streams first wait for the work already enqueued on the current stream; the caller joins them with
    `join(micro)` (or synchronises) before it reads the results.
    """
    cur = torch.cuda.current_stream()
    if overlap:
        for mb in micro:
            mb.stream.wait_stream(cur)
    for r in range(n_rounds):
        for i, mb in enumerate(micro):
            with torch.cuda.stream(mb.stream if overlap else cur):
                mb.begin_round()
                x = draft(i, r)
                mb.graft.build_trees(x["logits"], x.get("hidden"), x["root_token"], x.get("hist"),
                                     x.get("prefix_len", mb.prefix_len), x.get("fixed_budget"), mb.out)
                mb.walk(verify(i, r, mb.out))
                mb.rounds_done += 1
                if after_round is not None:
                    after_round(i, r, mb)


def join(micro: Sequence[MicroBatch]) -> None:
    """Make the current stream wait for every micro-batch's stream."""
    cur = torch.cuda.current_stream()
    for mb in micro:
        cur.wait_stream(mb.stream)
