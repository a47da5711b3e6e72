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
after the walk the accepted nodes' entries are moved up behind the prefix.
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
    # moved on by the committed tokens, status [batch] is the last call's
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

    def attend(self, layer, q, key, value, out, lse=None, scale=None, shared=0):
        """One layer of the target over this round's trees: the nodes' new entries go into the cache, q [batch, rows, q_heads, head_dim]
        sees the prefix and the nodes above its own."""
        if self.cache is None:
            raise GraftError("the micro-batch has no cache")
        self.graft.cache_write(self.cache, layer, self.table, self.prefix_len, self.out.n_nodes, key, value, self.status)
        self.graft.tree_attention(self.cache, layer, self.table, q, self.prefix_len, self.out.n_nodes, self.out.mask, out, lse, scale, shared,
                                  self.status)


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
                x = draft(i, r)
                mb.graft.build_trees(x["logits"], x.get("hidden"), x["root_token"], x.get("hist"),
                                     x.get("prefix_len", mb.prefix_len), x.get("fixed_budget"), mb.out)
                answer = verify(i, r, mb.out)
                if isinstance(answer, Sampled):
                    mb.graft.verify(mb.out, answer.logits, answer.temperature, answer.uniform, mb.accept_len, mb.accept_path,
                                    mb.bonus_token)
                else:
                    mb.graft.accept(mb.out, answer, mb.accept_len, mb.accept_path, mb.bonus_token)
                if mb.cache is not None:
                    mb.graft.cache_keep(mb.cache, mb.table, mb.prefix_len, mb.accept_len, mb.accept_path, mb.prefix_len, mb.status)
                mb.rounds_done += 1
                if after_round is not None:
                    after_round(i, r, mb)


def join(micro: Sequence[MicroBatch]) -> None:
    """Make the current stream wait for every micro-batch's stream."""
    cur = torch.cuda.current_stream()
    for mb in micro:
        cur.wait_stream(mb.stream)
