"""The verifier's calls on the most sequences that they take, and on one more."""
import numpy as np
import pytest
import torch

from test_gpu_verifier import BF, _i32

pytestmark = pytest.mark.gpu

MOST, V, L, D, page = 65535, 40, 2, 64, 16


def _setup(B):
    from paper_2608_20375_b200 import Graft, KVCache, TreeOut
    gen = torch.Generator(device="cuda").manual_seed(B)
    g = Graft(V, L, 4, 16, 8, MOST + 1, 1, 2, 1, 0.0)
    c = KVCache.alloc(1, B, 1, page, D)
    table = torch.randperm(B, generator=gen, device="cuda").int().view(B, 1)
    rows = torch.randn((2, B, 2, 1, D), generator=gen, device="cuda").to(BF)
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    tree = TreeOut(3 * one, None, torch.randint(0, V, (B, g.nmax), generator=gen, device="cuda", dtype=torch.int32),
                   _i32([[-1, 0, 1]]).repeat(B, 1), None, None, None, None, None)
    z, u = torch.randn((B, 3, V), generator=gen, device="cuda"), torch.rand((B, g.nmax), generator=gen, device="cuda")
    return g, c, table, rows, one, tree, z, u


def test_the_most_sequences():
    import verifier_ref as ref
    B = MOST
    g, c, table, (key, value), one, tree, z, u = _setup(B)
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    kb, vb = torch.zeros_like(key), torch.zeros_like(value)
    g.cache_write(c, 0, table, one, 2 * one, key, value, st)
    assert not st.any()
    g.cache_read(c, 0, table, one, 2 * one, kb, vb, st)
    assert not st.any() and torch.equal(kb, key) and torch.equal(vb, value)
    q = key[:, 1:].contiguous()
    out = torch.zeros_like(q)
    g.tree_attention(c, 0, table, q, 2 * one, one, None, out, status=st)
    assert not st.any()
    p = torch.softmax((q.double() * key.double()).sum(3, keepdim=True) * D ** -0.5, 1)  # (over the two slots)
    want = (p * value.double()).sum(1, keepdim=True)
    # weights and result are rounded to bf16; scores of 64 products and their exponential in fp32
    size = (p * value.double().abs()).sum(1, keepdim=True)
    assert ((out.double() - want).abs() <= 2.0 ** -8 * (size + want.abs()) * 1.02 + 2.0 ** -12 * size).all()
    alen, path, bonus = (torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,)))
    g.verify(tree, z, None, u, alen, path, bonus, st)
    assert not st.any()
    zc, uc, tok = z.cpu().double().numpy(), u.cpu().double().numpy(), tree.token.cpu().numpy()
    for b in (*range(0, B, 4099), B - 1):
        a, pa, bo = ref.walk(3, np.array([-1, 0, 1]), tok[b], lambda i: zc[b, i], 1.0, uc[b], L)
        assert (int(alen[b]), int(bonus[b])) == (a, bo) and path[b].tolist() == list(pa)
    nxt = torch.zeros_like(one)
    g.cache_keep(c, table, one, alen, path, nxt, st)
    assert not st.any() and torch.equal(nxt, alen + 2)


def test_one_sequence_more_is_refused():
    from paper_2608_20375_b200 import GraftError
    g, c, table, (key, value), one, tree, z, u = _setup(MOST + 1)
    alen, path, bonus = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((MOST + 1,), (MOST + 1, L), (MOST + 1,)))
    for call in (lambda: g.cache_write(c, 0, table, one, one, key, value), lambda: g.cache_read(c, 0, table, one, one, key, value),
                 lambda: g.cache_keep(c, table, one, alen, path), lambda: g.verify(tree, z, None, u, alen, path, bonus),
                 lambda: g.tree_attention(c, 0, table, key, one, one, None, value)):
        with pytest.raises(GraftError, match="supported"):
            call()
        torch.cuda.synchronize()
        assert int(one.sum()) == MOST + 1  # (nothing of a refusal is left for the next launch)


@pytest.mark.parametrize("dtype", [BF, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows", [1, 20])
def test_the_largest_scale(rows, dtype):
    """Scores of the usual size from tiny products; a scale beyond fp32's range once it stands in powers of two is refused."""
    import verifier_ref as ref
    from paper_2608_20375_b200 import GraftError
    from test_gpu_verifier import _cache, _graft
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g, n = _graft(max(2, rows), 1), 300 + rows
    table, n_pages = ref.page_table(np.random.default_rng(1), 1, 30)
    c = _cache(gen, (1, n_pages, 1, page, D), dtype)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    key, value, q = (2.0 ** -60 * r(1, n, 1, D)).to(BF), r(1, n, 1, D).to(BF), (2.0 ** -60 * r(1, rows, 2, D)).to(BF)
    out, lse, one = torch.zeros_like(q), torch.zeros((1, rows, 2), device="cuda"), _i32([1])
    g.cache_write(c, 0, _i32(table), one, _i32([n]), key, value)
    call = lambda scale: g.tree_attention(c, 0, _i32(table), q, _i32([301]), _i32([rows]), None, out, lse, scale=scale)  # noqa: E731
    call(2.0 ** 118)
    torch.cuda.synchronize()
    slots = np.arange(n)
    exps = (None, None) if dtype is BF else (c.k_exp[0].cpu(), c.v_exp[0].cpu())
    k, v = (ref.entries(t[0].cpu(), e, table[0], slots) for t, e in zip((c.k, c.v), exps))
    seen = slots[None, :] <= 300 + np.arange(rows)[:, None]
    wo, wl, tol, ltol = ref.attention(q[0].cpu().double().numpy(), k, v, seen, 2.0 ** 118)
    assert (np.abs(out[0].cpu().double().numpy() - wo) <= tol).all() and (np.abs(lse[0].cpu().double().numpy() - wl) <= ltol).all()
    for scale in (2.2e38, -2.2e38):
        call(scale)
    for scale in (2.4e38, -2.4e38, 3.4e38):
        with pytest.raises(GraftError, match="invalid"):
            call(scale)
    torch.cuda.synchronize()
