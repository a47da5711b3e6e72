"""The plain forms that the verifier's GPU tests compare with, against what they are meant to be (CPU), and refusals that need no GPU."""
import math

import numpy as np
import pytest
import torch

import verifier_ref as ref


def test_walk_keeps_the_targets_distribution():
    """Over all uniform numbers (a fine grid of them), the first committed token has the target's own distribution, whatever the tree."""
    z = np.array([0.3, -1.0, 1.2, 0.0, -math.inf, 0.7])
    T = 0.8
    p = np.exp(z / T) / np.exp(z / T).sum()
    token, parent = np.array([9, 2, 0, 4]), np.array([-1, 0, 0, 0])  # children: tokens 2, 0 and 4 (which the target rules out)
    g = 40
    grid = (np.arange(g) + 0.5) / g
    got = np.zeros(6)
    for u1 in grid:
        for u2 in grid:
            for u0 in grid:
                a, path, bonus = ref.walk(4, parent, token, lambda i: z, T, np.array([u0, u1, u2, 0.5]), 1)
                got[token[path[0]] if a else bonus] += 1
    # (a test against a grid of g points is off by at most one point each; three numbers decide)
    assert np.abs(got / g ** 3 - p).max() <= 3 / g
    assert got[4] == 0


def test_greedy_walk_is_the_acceptance_walk():
    import oracle
    rng = np.random.default_rng(3)
    for _ in range(20):
        n, V, L = int(rng.integers(1, 40)), 12, 6
        parent, depth, _ = ref.tree(rng, n, n, L)
        token = rng.integers(0, V, n).astype(np.int32)
        for i in range(1, n):  # siblings' tokens differ
            sib = [j for j in range(1, i) if parent[j] == parent[i]]
            token[i] = (token[sib[-1]] + 1) % V if sib else token[i]
        z = np.rint(rng.standard_normal((n, V)) * 2)  # ties
        a, path, bonus = ref.walk(n, parent, token, lambda i: z[i], 0.0, np.zeros(n), L)
        nxt = z.argmax(1).astype(np.int32)
        if len({(int(parent[i]), int(token[i])) for i in range(1, n)}) != n - 1:
            continue
        want = oracle.accept(n, token, parent, nxt, L)
        assert (a, list(path), bonus) == (want[0], list(want[1]), want[2])


def test_quantised_rows_are_torchs_e4m3_at_the_stated_scale():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn((200, 64), generator=g) * torch.logspace(-30, 30, 200)[:, None]).to(torch.bfloat16).float()
    x[3] = 0
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    x[6] = 448.0
    x[7] = 450.0
    val, e = ref.quantise_rows(x.numpy())
    assert e[4] == 255 and e[5] == 255 and np.isnan(val[4]).all() and e[3] == 7 and e[6] == 127 and e[7] == 128
    for i in [j for j in range(200) if j not in (4, 5)]:
        s = 2.0 ** (int(e[i]) - 127)
        amax = float(x[i].abs().max())
        assert amax <= 448 * s and (amax > 224 * s or e[i] == 7)
        y = (x[i].double() / s).float().to(torch.float8_e4m3fn).double() * s
        assert np.array_equal(val[i], y.numpy())


def test_trees_of_the_tests_are_level_ordered_with_ancestor_masks():
    rng = np.random.default_rng(0)
    for n in (1, 2, 33, 200):
        parent, depth, mask = ref.tree(rng, n, 210)
        b = ref.bits(mask, 210)
        for i in range(1, n):
            assert 0 <= parent[i] < i and parent[i] >= parent[i - 1] and depth[i] == depth[parent[i]] + 1 <= 16
            assert np.array_equal(b[i], b[parent[i]] | (np.arange(210) == i))
        assert not b[n:].any()


def test_binding_refuses_what_it_can_see():
    """Shapes, types and places of tensors are looked at before the library is called: CPU tensors are enough to see it."""
    from paper_2608_20375_b200 import BF16, E4M3, GraftError, KVCache, binding
    c = KVCache(torch.zeros((1, 2, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 2, 16, 64), dtype=torch.bfloat16))
    t = torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(GraftError, match="CUDA"):
        c._c(t, 1, 0)
    with pytest.raises(GraftError, match="pages"):
        c._c(t[0], 1, 0)
    with pytest.raises(GraftError, match="exponents"):
        KVCache(c.k, c.v, torch.zeros((1, 2, 2, 16), dtype=torch.uint8))._c(t, 1, 0)
    with pytest.raises(GraftError, match="bfloat16 or float8"):
        KVCache(c.k.float(), c.v.float())._c(t, 1, 0)
    with pytest.raises(GraftError, match="shape"):
        binding._shaped("x", torch.zeros(3), torch.float32, (4,), 0)
    with pytest.raises(GraftError, match=r"\[batch, rows, 2, 64\]"):
        binding._token_rows("key", torch.zeros((1, 3, 2, 32), dtype=torch.bfloat16), 2, 64, 0)
    with pytest.raises(GraftError, match="CUDA"):
        binding._token_rows("key", torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16), 2, 64, 0)
    assert (BF16, E4M3) == (1, 2)
