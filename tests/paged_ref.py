"""64-bit statements of the operators over a paged cache, request by request and key by key, and error bounds that follow
from the arithmetic of 32- and 16-bit kernels.  Shares nothing with the library."""
import math

import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def make_cache(lens, hkv, h, dtype, page=16, seed=0, spare=3, layers=None, garbage=float("nan"), device="cpu"):
    """K, V with every request's pages scattered, slots that hold no key filled with `garbage`; (k, v, table, n_kv)."""
    g = torch.Generator().manual_seed(seed)
    pages = [(n + page - 1) // page for n in lens]
    n_pages, cols = sum(pages) + spare, max(max(pages, default=0), 1)
    order = torch.randperm(n_pages, generator=g)
    table = torch.full((len(lens), cols), -7, dtype=torch.int32)
    shape = (n_pages, hkv, page, h) if layers is None else (layers, n_pages, hkv, page, h)
    k, v = (torch.full(shape, garbage, dtype=dtype) for _ in range(2))
    at = 0
    for i, n in enumerate(lens):
        mine = order[at:at + pages[i]]
        at += pages[i]
        table[i, :pages[i]] = mine.to(torch.int32)
        for x in (k, v):
            for b, p in enumerate(mine.tolist()):
                c = min(page, n - b * page)
                x[..., p, :, :c, :] = torch.randn(*(shape[:-4] + (hkv, c, h)), generator=g).to(dtype)
    return tuple(t.to(device) for t in (k, v, table, torch.tensor(lens, dtype=torch.int32)))


def keys_of(pool, table_row, n, page):
    """[hkv, n, ...] in 64 bits."""
    pages = table_row[:(n + page - 1) // page].long()
    x = pool[pages].double()
    return x.transpose(0, 1).reshape(x.shape[1], -1, *x.shape[3:])[:, :n]


def tree_mask(parents, m, n):
    """[m, n] of what every node sees; parents None: a chain.  Unused nodes see nothing."""
    see = torch.zeros(m, n, dtype=torch.bool)
    for j in range(m):
        if parents is None:
            see[j, :n - m + j + 1] = True
            continue
        chain, a = [], j
        while a >= 0:
            chain.append(a)
            a = parents[a]
        if a == -1:
            see[j, :n - m] = True
            see[j, [n - m + c for c in chain]] = True
    return see


def attend(q, k, v, see, scale, dtype):
    """q [m, hq, h], k, v [hkv, n, h] (64 bits), see [m, n] or [m, hkv, n] -> out, lse, p [m, hq, n], and the bounds of the
    errors that a kernel with fp32 sums may have: out's per element, lse's and p's per row, p's relative."""
    m, hq, h = q.shape
    hkv, n = k.shape[:2]
    q = q.double().view(m, hkv, hq // hkv, h)
    if see.dim() == 2:
        see = see[:, None].expand(m, hkv, n)
    s = torch.einsum("mgrd,gnd->mgrn", q, k) * scale
    size = torch.einsum("mgrd,gnd->mgrn", q.abs(), k.abs()) * scale
    s = s.masked_fill(~see[:, :, None], -math.inf)
    size = size.masked_fill(~see[:, :, None], 0)
    lse = torch.logsumexp(s, -1) if n else torch.full((m, hkv, hq // hkv), -math.inf, dtype=torch.float64)
    p = torch.where(see[:, :, None], torch.exp(s - torch.where(lse == -math.inf, 0, lse)[..., None]), torch.zeros((), dtype=torch.float64))
    o = torch.einsum("mgrn,gnd->mgrd", p, v)
    spread = torch.einsum("mgrn,gnd->mgrd", p, v.abs())
    u = 2.0 ** -24
    # a score is a sum of h products, scaled, in fp32: it is off by at most ds (also after the change to base 2); an
    # exponential of it by a factor of 1 + ds plus a few units of its own, and a sum of n of them by n units more
    ds = (h + 8) * u * (size.amax(-1) if n else torch.zeros_like(lse))
    rel = 2 * ds + (n + 64) * u
    e = EPS[dtype]
    p_round = e if dtype == torch.bfloat16 else 0.0            # probabilities enter the second product in 16 bits
    d_out = (rel[..., None] + p_round) * spread + e * o.abs() + 1e-30
    d_lse = ds + (n + 64) * u + 8 * u * lse.abs().nan_to_num(posinf=0)
    return o.reshape(m, hq, h), lse.reshape(m, hq), p.reshape(m, hq, n), d_out.reshape(m, hq, h), d_lse.reshape(m, hq), \
        (rel + 8 * u * (1 + lse.abs().nan_to_num(posinf=0))).reshape(m, hq)


def evicted(weights, n, budget, sink, recent):
    """Which slot each of the slots 0 .. min(n, budget)-1 takes its key from (one layer and head; weights: a list)."""
    if n <= budget:
        return list(range(n))
    big = lambda w: math.inf if w != w else w
    cand = sorted(range(sink, n - recent), key=lambda x: (-big(weights[x]), 0 if weights[x] != weights[x] else 1, x))[:budget - sink - recent]
    kept = set(cand) | set(range(sink))
    come = list(range(budget - recent))
    holes = [x for x in come if x not in kept]
    movers = sorted(x for x in cand if x >= budget - recent)
    assert len(holes) == len(movers)
    for a, b in zip(holes, movers):
        come[a] = b
    return come + list(range(n - recent, n))


def block_scores(q, bounds, hkv):
    """q [hq, h], bounds [blocks, hkv, 2, h] (64 bits) -> [hkv, blocks]."""
    hq, h = q.shape
    q = q.double().view(hkv, hq // hkv, 1, h)
    b = bounds.double().permute(1, 0, 2, 3)[:, None]                     # [hkv, 1, blocks, 2, h]
    return torch.maximum(q * b[..., 0, :], q * b[..., 1, :]).sum(-1).amax(1)
