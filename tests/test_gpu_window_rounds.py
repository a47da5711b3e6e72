"""Rounds of a micro-batch whose target has rotary positions and a window: what every layer's attention gives is the plain form's over
all that was committed, round after round, and what goes wrong is reported."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref
import window_ref as win
from test_gpu_verifier import BF, Q8, _i32

pytestmark = pytest.mark.gpu
B, L, V, K, Hq, Hk, D, page, pages = 3, 6, 300, 5, 4, 2, 64, 16, 8


def _target(dtype, gen):
    from paper_2608_20375_b200 import BF16, E4M3, Graft, KVCache, MicroBatch
    g = Graft(V, L, K, 16, 8, B, 4, 24, 4, 0.0)
    table = torch.randperm(B * pages, generator=gen, device="cuda").int().view(B, pages)
    return MicroBatch(g, B, L, cache=KVCache.alloc(1, B * pages, Hk, page, D, E4M3 if dtype is Q8 else BF16), table=table, prefix_len=_i32([1, 1, 1]))


@pytest.mark.parametrize("dtype", [BF, Q8])
@pytest.mark.parametrize("window,sinks,axes", [(20, 3, 1), (7, 0, 3), (None, 0, 1)])
def test_rounds_of_a_rotary_target(dtype, window, sinks, axes):
    from paper_2608_20375_b200 import Rope, Sampled, join, run_rounds
    gen = torch.Generator(device="cuda").manual_seed(window or 1)
    mb = _target(dtype, gen)
    n = mb.graft.nmax
    shift = _i32([0, 40, 7])
    rope = Rope.of(D, 100.0, sections=None if axes == 1 else [8, 12, 12], shift=shift)
    freq = rope.freq.cpu().numpy()
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(BF)  # noqa: E731
    kept = [[] for _ in range(B)]  # turned keys (with what they may be off by) and values of the committed tokens, plain
    worst = []
    state = {}

    def draft(i, r):
        return dict(logits=3 * torch.randn((B, L, V), generator=gen, device="cuda").to(BF),
                    root_token=_i32([3, 5, 7]) if r == 0 else mb.bonus_token.clone(), fixed_budget=_i32([20, 4, 24]))

    def verify(i, r, out):
        q, key, value = rand(B, n, Hq, D), rand(B, n, Hk, D), rand(B, n, Hk, D)
        turned, o, lse = torch.zeros_like(q), torch.zeros((B, n, Hq, D), dtype=BF, device="cuda"), torch.zeros((B, n, Hq), device="cuda")
        was = q.clone()
        mb.attend(0, q, key, value, o, lse=lse, rope=rope, q_out=turned, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert torch.equal(q, was)
        for b in range(B):
            m, base = int(out.n_nodes[b]), int(mb.prefix_len[b]) - 1
            pos = out.position[b, :m].cpu().numpy()
            at = np.broadcast_to((pos + int(shift[b]))[:, None], (m, axes))
            qt, qe = win.turned(q[b, :m].cpu().double().numpy(), at, freq, False, 1.0)
            kt, ke = win.turned(key[b, :m].cpu().double().numpy(), at, freq, False, 1.0)
            state[b] = (kt, value[b, :m].cpu().double().numpy())
            got = turned[b, :m].cpu().double().numpy()
            assert (np.abs(got - qt) <= qe + 2.0 ** -8 * (np.abs(qt) + qe)).all()
            # keys and values as they were held: what attention is compared with
            slots = np.arange(base + m)
            held = [ref.entries(t[0].cpu(), None if e is None else e[0].cpu(), mb.table[b].cpu().numpy(), slots)
                    for t, e in ((mb.cache.k, mb.cache.k_exp), (mb.cache.v, mb.cache.v_exp))]
            want = [np.concatenate([np.stack([x[j] for x in kept[b]]).reshape(-1, Hk, D) if kept[b] else np.zeros((0, Hk, D)), new])
                    for j, new in ((0, kt), (1, state[b][1]))]
            step = 2.0 ** -4 if dtype is Q8 else 2.0 ** -8  # half a step of the type; e4m3: or of the row's least exponent, 2^-10 of its scale
            for h, w in zip(held, want):
                least = np.abs(w).max(-1, keepdims=True) * 2.0 ** -17 if dtype is Q8 else 0.0
                assert h.shape == w.shape and (np.abs(h - w) <= step * (np.abs(w) + 1e-5) + 1e-5 + least).all()
            bits = ref.bits(out.mask[b].cpu().numpy(), n)
            seen = np.stack([win.sees(j, slots, base, m, pos, bits[j], window or 10 ** 6, sinks) for j in range(m)])
            a, l, tol, ltol = ref.attention(got, held[0], held[1], seen, D ** -0.5)
            worst.append((np.abs(o[b, :m].cpu().double().numpy() - a) / tol).max())
            assert worst[-1] <= 1 and (np.abs(lse[b, :m].cpu().double().numpy() - l) <= ltol).all()
        z = torch.randn((B, n, V), generator=gen, device="cuda")
        z.view(B, -1).scatter_add_(1, out.parent.long().clamp(0) * V + out.token.long().clamp(0), torch.where(out.parent >= 0, 12.0, 0.0))
        return Sampled(z, torch.rand((B, n), generator=gen, device="cuda"))

    def after(i, r, _):
        torch.cuda.synchronize()
        assert not mb.status.any()
        for b in range(B):
            for node in [0] + mb.accept_path[b, :int(mb.accept_len[b])].tolist():
                kept[b].append((state[b][0][node], state[b][1][node]))

    run_rounds([mb], 5, draft, verify, after_round=after)
    join([mb])
    assert max(len(x) for x in kept) > 8 and [len(x) + 1 for x in kept] == mb.prefix_len.tolist()


@pytest.mark.parametrize("which", ["append", "attention"])
def test_a_sequence_whose_pages_are_gone_is_not_moved_on(which):
    """A page of the window is missing for the attention only (the sinks' page, which an append does not touch), or for both."""
    from paper_2608_20375_b200 import Rope, join, run_rounds
    gen = torch.Generator(device="cuda").manual_seed(3)
    mb = _target(BF, gen)
    mb.prefix_len.copy_(_i32([50, 50, 50]))
    mb.table[1, 0 if which == "attention" else 3] = -1
    n = mb.graft.nmax
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(BF)  # noqa: E731

    def verify(i, r, out):
        o = torch.zeros((B, n, Hq, D), dtype=BF, device="cuda")
        mb.attend(0, rand(B, n, Hq, D), rand(B, n, Hk, D), rand(B, n, Hk, D), o, rope=Rope.of(D), window=10, sinks=2)
        return torch.zeros((B, n), dtype=torch.int32, device="cuda")

    run_rounds([mb], 1, lambda i, r: dict(logits=rand(B, L, V), root_token=_i32([1, 2, 3]), fixed_budget=_i32([8] * B)), verify)
    join([mb])
    torch.cuda.synchronize()
    assert mb.status.tolist() == [0, 16, 0]
    assert mb.prefix_len.tolist() == [51 + int(mb.accept_len[0]), 50, 51 + int(mb.accept_len[2])]


def test_refusals():
    from paper_2608_20375_b200 import GraftError, KVCache, Rope
    gen = torch.Generator(device="cuda").manual_seed(0)
    mb = _target(BF, gen)
    g, c, t, one = mb.graft, mb.cache, mb.table, _i32([1, 1, 1])
    n = g.nmax
    q, key = (torch.zeros((B, n, h, D), dtype=BF, device="cuda") for h in (Hq, Hk))
    out, pos, mask = torch.zeros_like(q), torch.zeros((B, n), dtype=torch.int32, device="cuda"), mb.out.mask.zero_()
    rope = Rope.of(D)

    def append(rope=rope, q=q, key=key, value=key, q_out=None, cache=c, **kw):
        g.cache_append(cache, 0, t, one, one, rope, q, key, value, q_out, **kw)

    def attend(mask=mask, position=pos, window=5, sinks=0, q=q, out=out, scale=None, cache=c, layer=0, **kw):
        g.window_attention(cache, layer, t, q, one, one, mask, position, window, sinks, out, scale=scale, **kw)

    append(), attend(), attend(None, None)
    other = KVCache.alloc(1, B * pages, Hk, page, 128)
    wide = Rope(torch.zeros((9, 32), device="cuda"))
    for call in (lambda: append(rope=Rope.of(2 * D)), lambda: append(rope=Rope(torch.zeros((1, 12), device="cuda"))), lambda: append(rope=wide),
                 lambda: append(rope=Rope.of(D, gain=math.inf)), lambda: append(rope=Rope.of(D, gain=math.nan)),
                 lambda: append(rope=Rope(rope.freq.double())), lambda: append(rope=Rope.of(D, shift=pos)), lambda: append(position=pos[:, :n - 1].contiguous()),
                 lambda: append(position=pos.float()), lambda: append(q=q.float()), lambda: append(q=q[:, :-1]), lambda: append(q_out=out[:, :-1]),
                 lambda: append(q=None, q_out=out), lambda: append(value=key[:, :-1]), lambda: append(cache=other), lambda: append(status=pos),
                 lambda: append(q_out=torch.zeros((B, n, Hq, 2 * D), dtype=BF, device="cuda")[..., :D]),
                 lambda: attend(window=0), lambda: attend(window=-3), lambda: attend(sinks=-1), lambda: attend(mask=None), lambda: attend(position=None),
                 lambda: attend(position=pos[:, :n - 1].contiguous()), lambda: attend(mask=mask[:1]), lambda: attend(scale=math.inf), lambda: attend(scale=math.nan),
                 lambda: attend(q=q[:, :, :3]), lambda: attend(out=out.float()), lambda: attend(layer=1), lambda: attend(cache=other),
                 lambda: attend(lse=torch.zeros((B, n), device="cuda")),
                 lambda: mb.attend(0, q, key, key, out, window=4, shared=16), lambda: mb.attend(0, q, key, key, out, sinks=4),
                 lambda: mb.attend(0, q, key, key, out, q_out=q), lambda: mb.attend(0, q, key, key, out, window=0)):
        with pytest.raises(GraftError):
            call()
    # the same array with another stride
    buf = torch.zeros((B * n * Hq * D * 2,), dtype=BF, device="cuda")
    a, b = buf[:B * n * Hq * D].view(B, n, Hq, D), buf.view(B, n, 2 * Hq * D)[..., :Hq * D].unflatten(2, (Hq, D))
    with pytest.raises(GraftError):
        append(q=a, q_out=b)
    torch.cuda.synchronize()
    append(), attend()  # and the context is as good as before
    torch.cuda.synchronize()
