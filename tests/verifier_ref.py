"""Plain fp64 forms of the verifier's operators (numpy on the CPU, one sequence at a time), for their tests."""
import math

import numpy as np
import torch


def quantise_rows(x):
    """x [..., D] (values of bf16 numbers) -> (values of the e4m3 entries times their scale, exponent bytes)."""
    x = np.asarray(x, np.float64)
    amax = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        m, e = np.frexp(np.where(bad, 0.0, amax) / 448.0)  # amax / 448 = m 2^e, m in [0.5, 1)
    e = np.where(m == 0.5, e - 1, e)
    e = np.clip(np.where(amax == 0, -120, e), -120, 120)
    t = np.ldexp(np.where(bad[..., None], 0.0, x), -e[..., None])
    unit = np.ldexp(1.0, np.frexp(np.maximum(np.abs(t), 2.0 ** -6))[1] - 4)  # three bits behind the leading one
    y = np.rint(t / unit) * unit
    return np.where(bad[..., None], np.nan, np.ldexp(y, e[..., None])), np.where(bad, 255, e + 127).astype(np.uint8)


def bits(mask, n):
    """[rows, W] int32 words -> [rows, n] truth values, bit j of row i."""
    w = np.ascontiguousarray(mask).view(np.uint32)
    j = np.arange(n)
    return ((w[:, j // 32] >> (j % 32).astype(np.uint32)) & 1).astype(bool)


def attention(q, k, v, seen, scale):
    """One sequence: q [n, Hq, D], k, v [S, Hk, D], seen [n, S] -> out, lse, and bounds on what fp32 scores and bf16 weights and results
    may be off by.  A weight is rounded to bf16 (2^-8 of itself), the result too; a score is a sum of D products in fp32 (D + 2 roundings of
    what the products' magnitudes add up to), which moves a weight by that share of itself, and the weights' fp32 sum, S additions."""
    n, Hq, D = q.shape
    S, Hk, _ = k.shape
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -math.inf)
    tol, ltol = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // Hk)], v[:, h // (Hq // Hk)]
        s = np.where(seen, scale * (q[:, h] @ np.nan_to_num(kh).T), -math.inf)
        size = abs(scale) * (np.abs(q[:, h]) @ np.abs(np.nan_to_num(kh)).T)
        es = (D + 2) * 2.0 ** -24 * np.where(seen, size, 0.0).max(1, initial=0.0)
        top = s.max(1, initial=-math.inf)
        ok = np.isfinite(top)
        w = np.exp(s - np.where(ok, top, 0.0)[:, None])
        z = w.sum(1)
        p = w / np.where(ok, z, 1.0)[:, None]
        vf = np.nan_to_num(vh, nan=0.0, posinf=0.0, neginf=0.0)
        out[:, h] = p @ vf
        # entries that a row sees and that are not numbers reach that row
        for j in np.nonzero(~np.isfinite(vh).all(1))[0]:
            with np.errstate(invalid="ignore"):
                out[seen[:, j], h] += np.where(np.isfinite(vh[j]), 0.0, p[seen[:, j], j][:, None] * vh[j])
        lse[ok, h] = top[ok] + np.log(z[ok])
        a = p @ np.abs(vf)
        e_sum = S * 2.0 ** -24
        # (scores are worked out in the log2 domain: one more rounding of the score, and the 2^x instruction's 2^-22)
        e_w = 2 * es + np.where(ok, np.abs(top), 0.0) * 2.0 ** -22 + 2.0 ** -21
        tol[:, h] = 2.0 ** -8 * (a + np.abs(np.nan_to_num(out[:, h]))) * (1 + 2.0 ** -6) + (2 * e_w + 2 * e_sum)[:, None] * a + 1e-30
        ltol[:, h] = e_w + e_sum + np.where(ok, np.abs(lse[:, h]), 0.0) * 2.0 ** -23
    return out, lse, tol, ltol


def walk(n, parent, token, logits, T, u, L):
    """One sequence of graft_verify: accepted length, path [L], bonus.  logits: a function of the node that gives fp64 logits."""
    path, cur, a = np.full(L, -1, np.int32), 0, 0
    while True:
        z = np.asarray(logits(cur), np.float64)
        V = len(z)
        if np.isnan(z).any() or (z == math.inf).any() or not np.isfinite(z).any():
            return a, path, -1
        if T == 0:
            w = np.zeros(V)
            w[np.argmax(z)] = 1.0
        else:
            w = np.exp((z - z.max()) / float(T))
        nxt = -1
        for c in range(1, n if a < L else 0):
            if parent[c] != cur:
                continue
            t = token[c]
            if not 0 <= t < V:
                continue
            if float(u[c]) * w.sum() < w[t]:
                nxt = c
                break
            w[t] = 0.0
        if nxt < 0:
            break
        path[a] = nxt
        a, cur = a + 1, nxt
    cdf = np.cumsum(w)
    bonus = int(np.searchsorted(cdf, float(u[0]) * cdf[-1], side="right")) if cdf[-1] > 0 else int(np.argmax(z))
    return a, path, min(bonus, V - 1)


def tree(rng, n, nmax, L=16):
    """A random tree of n nodes in level order: parents, depths [nmax] (-1 behind n), masks [nmax, W] int32."""
    W = (nmax + 31) // 32
    parent, depth, mask = np.full(nmax, -1, np.int32), np.full(nmax, -1, np.int32), np.zeros((nmax, W), np.uint32)
    if n == 0:
        return parent, depth, mask.view(np.int32)
    depth[0] = 0
    mask[0, 0] = 1
    level, i = [0], 1
    while i < n:
        d = depth[level[0]] + 1
        size = n - i if d == L else min(n - i, int(rng.integers(1, 2 + 2 * len(level))))
        ps = np.sort(rng.choice(level, size))
        for p in ps:
            parent[i], depth[i] = p, d
            mask[i] = mask[p]
            mask[i, i // 32] |= np.uint32(1 << (i % 32))
            i += 1
        level = list(range(i - size, i))
    return parent, depth, mask.view(np.int32)


def page_table(rng, batch, width, spare=3, shared_pages=0):
    """Pages in random order, some of the cache in nobody's use."""
    n = shared_pages + batch * (width - shared_pages) + spare
    pages = rng.permutation(n).astype(np.int32)
    t = np.empty((batch, width), np.int32)
    t[:, :shared_pages] = pages[:shared_pages]
    t[:, shared_pages:] = pages[shared_pages:n - spare].reshape(batch, -1)
    return t, n


def entries(k, exp, table_row, slots):
    """Entries of slots (numpy) of one layer's k [n_pages, Hk, page, D] (torch, CPU) -> [S, Hk, D] fp64."""
    page_size = k.shape[2]
    page, at = torch.from_numpy(table_row[slots // page_size]).long(), torch.from_numpy(slots % page_size).long()
    y = k[page, :, at].double().numpy()
    if exp is None:
        return y
    e = exp[page, :, at].numpy().astype(np.int64)
    with np.errstate(invalid="ignore"):
        return np.where((e == 255)[..., None], np.nan, np.ldexp(y, (e - 127)[..., None]))
