"""Operators over a paged key-value cache: tree attention, attention weights per key, eviction, block bounds, block attention.

Each case can be computed in its plain form (`own` false: elementary torch operations in 32 bits) or by the library's own
calls (`own` true).  A cache is K, V [page][kv head][slot][head_dim]; request i's key x lies in page page_table[i][x / 16],
slot x % 16, and the last q_len of its n_kv keys are the tokens whose queries are given.  Page-table entries behind a
request's last page are -1, slots behind its last key hold what an earlier owner of the page left there.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
GEOMETRY = {  # query heads, kv heads, head_dim, type: the shapes that the library ships
    "tiny": (4, 4, 64, "fp32"),
    "1b": (32, 8, 64, "bf16"),
    "8b": (32, 8, 128, "bf16"),
    "gqa": (8, 2, 128, "bf16"),
}
TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one device's small draft tree on the 1B model: the shortest call a server makes
        {"name": "tree one device", "op": "tree", "geometry": "1b", "batch": 1, "lo": 700, "hi": 700, "nodes_lo": 7, "nodes_hi": 7},
        # a step of the default serving batch on the 8B model, ragged trees
        {"name": "tree batch 16", "op": "tree", "geometry": "8b", "batch": 16, "lo": 512, "hi": 4096, "nodes_lo": 4, "nodes_hi": 24},
        # many devices with wide trees: as many query rows as keys' bytes can pay for
        {"name": "tree wide", "op": "tree", "geometry": "8b", "batch": 64, "lo": 512, "hi": 4096, "nodes_lo": 48, "nodes_hi": 64},
        # the 32-bit configuration
        {"name": "tree fp32", "op": "tree", "geometry": "tiny", "batch": 24, "lo": 64, "hi": 2000, "nodes_lo": 2, "nodes_hi": 9},
        # ordinary decoding of a batch with weights kept for eviction
        {"name": "weigh tokens", "op": "weigh", "geometry": "8b", "batch": 32, "lo": 128, "hi": 16384, "nodes_lo": 1, "nodes_hi": 1},
        # verification of a few devices' drafts with weights kept
        {"name": "weigh drafts", "op": "weigh", "geometry": "8b", "batch": 6, "lo": 3000, "hi": 6000, "nodes_lo": 5, "nodes_hi": 9},
        # one device of the 1B model goes back under its budget after a few steps
        {"name": "evict one device", "op": "evict", "geometry": "1b", "layers": 16, "batch": 1, "lo": 1061, "hi": 1061, "budget": 1024, "sink": 4, "recent": 64},
        # a batch of prompts is cut down to the budget in all layers at once
        {"name": "evict prompts", "op": "evict", "geometry": "8b", "layers": 32, "batch": 8, "lo": 1500, "hi": 6000, "budget": 2048, "sink": 4, "recent": 256},
        # the pages that a decoding step of a batch has filled
        {"name": "bounds append", "op": "bounds", "geometry": "8b", "batch": 48, "lo": 512, "hi": 8192, "fresh": 23},
        # whole prompts
        {"name": "bounds prompts", "op": "bounds", "geometry": "8b", "batch": 24, "lo": 2000, "hi": 16384, "fresh": 0},
        # one device with a long context, one token
        {"name": "blocks one device", "op": "blocks", "geometry": "8b", "batch": 1, "lo": 30011, "hi": 30011, "nodes_lo": 1, "nodes_hi": 1, "blocks": 64, "local": 4},
        # a batch of long contexts, drafts of several lengths
        {"name": "blocks batch", "op": "blocks", "geometry": "8b", "batch": 24, "lo": 3000, "hi": 32000, "nodes_lo": 2, "nodes_hi": 9, "blocks": 96, "local": 4},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "weigh", "evict", "bounds", "blocks"])
    geometry = rng.choice(["tiny", "1b", "8b", "8b", "gqa"])
    batch = _log_int(rng, 1, 48)
    lo = _log_int(rng, 40, 3000)
    hi = min(16384, _log_int(rng, lo, 8 * lo))
    case = {"op": op, "geometry": geometry, "batch": batch, "lo": lo, "hi": hi}
    if op in ("tree", "weigh"):
        most = rng.choice([1, 3, 9, 17, 33] if op == "tree" else [1, 4, 9])
        case.update(nodes_lo=rng.randint(1, most), nodes_hi=most)
    elif op == "evict":
        budget = _log_int(rng, max(40, lo // 4), hi)
        case.update(layers=rng.choice([1, 2, 5, 16]), budget=budget, sink=rng.randint(0, 8), recent=rng.randint(1, budget // 4),
                    batch=min(batch, 8))
    elif op == "bounds":
        case.update(fresh=rng.choice([0, 1, 9, 40]))
    else:
        local = rng.randint(1, 8)
        case.update(nodes_lo=1, nodes_hi=rng.choice([1, 5, 9]), blocks=local + _log_int(rng, 4, 120), local=local, lo=lo * 2, hi=min(32000, hi * 2))
    return case


def _sizes(case):
    """Cached keys and new tokens of every request: they follow from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n_kv, q_len = [], []
    for _ in range(case["batch"]):
        n = _log_int(rng, case["lo"], case["hi"])
        q = rng.randint(case["nodes_lo"], case["nodes_hi"]) if "nodes_lo" in case else 0
        n_kv.append(max(n, q))
        q_len.append(q)
    return n_kv, q_len


def _tree(rng, m):
    """A draft tree: node 0 continues the cached text, every other node hangs on one of the nodes shortly before it."""
    return [-1] + [rng.randint(max(0, j - 6), j - 1) for j in range(1, m)]


def _fresh_from(case, n):
    return 0 if case["fresh"] == 0 else max(0, n - case["fresh"])


def _moves(case, n):
    """Expected number of cache rows that an eviction has to move for one request, layer and kv head."""
    m, s, r = case["budget"], case["sink"], case["recent"]
    if n <= m:
        return 0.0
    return (m - r - s) * (n - m) / (n - r - s) + r


def work(case):
    hq, hkv, h, t = GEOMETRY[case["geometry"]]
    e = 4 if t == "fp32" else 2
    n_kv, q_len = _sizes(case)
    rows = sum(q_len) * hq
    meta = 4 * sum((n + PAGE - 1) // PAGE for n in n_kv)
    if case["op"] in ("tree", "weigh"):
        size = sum(n_kv) * 2 * hkv * h * e + 2 * rows * h * e + meta
        if case["op"] == "weigh":
            size += 8 * sum(n_kv) * hkv
        return {"bytes": size, "flops": sum(4 * h * q * hq * (n - q / 2) for n, q in zip(n_kv, q_len))}
    if case["op"] == "evict":
        per = sum(4 * n + 4 * min(n, case["budget"]) + _moves(case, n) * 4 * h * e for n in n_kv)
        return {"bytes": case["layers"] * hkv * per + meta, "flops": 0}
    if case["op"] == "bounds":
        keys = sum(n - _fresh_from(case, n) // PAGE * PAGE for n in n_kv)
        return {"bytes": keys * hkv * h * e * (1 + 2 / PAGE) + meta, "flops": 2 * keys * hkv * h}
    size, flops = 2 * rows * h * e + meta, 0
    for n, q in zip(n_kv, q_len):
        blocks = (n + PAGE - 1) // PAGE
        scored = max(0, blocks - case["local"]) if blocks > case["blocks"] else 0
        read = min(blocks, case["blocks"])
        size += scored * hkv * 2 * h * e + min(blocks, read * q) * PAGE * hkv * 2 * h * e
        flops += q * hq * (4 * h * scored + 4 * h * read * PAGE)
    return {"bytes": size, "flops": flops}


# --------------------------------------------------------------------------------------------------- the inputs
def prepare(case, seed):
    dev = "cuda"
    hq, hkv, h, t = GEOMETRY[case["geometry"]]
    dt = TYPE[t]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = random.Random(seed)
    n_kv, q_len = _sizes(case)
    batch = len(n_kv)
    pages = [(n + PAGE - 1) // PAGE for n in n_kv]
    cols, total = max(pages), sum(pages)
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((batch, cols), -1, dtype=torch.int32)
    host_order, at = order.cpu(), 0
    for i, p in enumerate(pages):
        table[i, :p] = host_order[at:at + p]
        at += p
    s = {"op": case["op"], "page_table": table.to(dev), "n_kv": torch.tensor(n_kv, dtype=torch.int32, device=dev),
         "most_keys": cols * PAGE, "most_nodes": max(q_len)}
    lead = (case["layers"],) if case["op"] == "evict" else ()
    shape = lead + (n_pages, hkv, PAGE, h)
    # queries of a head have a direction in common, and the keys of one page in sixteen lean that way: those draw the
    # attention, as a few places of a text do
    way = torch.randn(hkv, 1, h, generator=g, device=dev)
    lean = (torch.rand(n_pages, 1, 1, 1, generator=g, device=dev) < 1 / 16).float() * 0.4

    def cache(leaning):
        x = torch.empty(shape, dtype=dt, device=dev)
        for l in range(shape[0]) if lead else range(1):
            y = torch.randn(shape[-4:], generator=g, device=dev)
            (x[l] if lead else x).copy_(y + lean * way if leaning else y)
            del y
        return x

    s["k"] = cache(True)
    if case["op"] != "bounds":
        s["v"] = cache(False)
    if case["op"] in ("tree", "weigh", "blocks"):
        total_q = sum(q_len)
        q = torch.randn(total_q, hkv, hq // hkv, h, generator=g, device=dev) * 0.8 + 0.6 * way[None, :, :, :]
        s["q"] = q.reshape(total_q, hq, h).to(dt)
        cu = [0]
        for m in q_len:
            cu.append(cu[-1] + m)
        s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    if case["op"] in ("tree", "weigh"):
        s["parents"] = torch.tensor(sum((_tree(rng, m) for m in q_len), []), dtype=torch.int32, device=dev)
    if case["op"] == "weigh":
        s["key_weights"] = torch.rand(n_pages, hkv, PAGE, generator=g, device=dev)
    if case["op"] == "evict":
        # accumulated weights: a few keys have most of it
        w = torch.randn(shape[:-1], generator=g, device=dev) * 2
        s["key_weights"] = torch.exp(w)
        s["key_weights_out"] = torch.zeros_like(s["key_weights"])
        s.update(budget=case["budget"], sink=case["sink"], recent=case["recent"])
    if case["op"] == "bounds":
        s["first"] = torch.tensor([_fresh_from(case, n) for n in n_kv], dtype=torch.int32, device=dev)
        s["bounds"] = torch.zeros(n_pages, hkv, 2, h, dtype=dt, device=dev)
    if case["op"] == "blocks":
        s["bounds"] = torch.stack([s["k"].amin(2), s["k"].amax(2)], 2).contiguous()
        s.update(blocks=case["blocks"], local=case["local"])
    return s


# ----------------------------------------------------------------------------------------------- the plain forms
def _gathered(pool, s):
    """[batch, kv heads, keys, ...] of a pool [page, kv heads, slot, ...], in 32 bits; keys a request lacks are zero."""
    x = pool[s["page_table"].clamp_min(0).long()].float().transpose(1, 2)
    x = x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])
    there = torch.arange(x.shape[2], device=x.device) < s["n_kv"][:, None]
    there = there[:, None].reshape(there.shape[0], 1, there.shape[1], *(1 for _ in x.shape[3:]))
    return torch.where(there, x, 0)


def _rows(s):
    """Of every query: its request and its place among the request's queries."""
    t = torch.arange(s["q"].shape[0], device=s["q"].device)
    req = torch.searchsorted(s["cu_q"].long(), t, right=True) - 1
    return req, t - s["cu_q"].long()[req]


def _visible(s, req, j):
    """[batch, node, node]: which nodes a node sees, itself and its ancestors."""
    m = s["most_nodes"]
    step = torch.eye(m, dtype=torch.float64, device=req.device).repeat(s["n_kv"].shape[0], 1, 1)
    up = s["parents"].long()
    at = torch.where(up >= 0, up, j)
    step.index_put_((req, j, at), torch.ones_like(up, dtype=torch.float64))
    return torch.linalg.matrix_power(step, m) > 0


def _tree_plain(s):
    hq, h = s["q"].shape[1:]
    k, v = _gathered(s["k"], s), _gathered(s["v"], s)
    batch, hkv, keys = k.shape[:3]
    m = s["most_nodes"]
    req, j = _rows(s)
    q = torch.zeros(batch, m, hq, h, device=k.device)
    q[req, j] = s["q"].float()
    q = q.view(batch, m, hkv, hq // hkv, h).permute(0, 2, 1, 3, 4).reshape(batch, hkv, -1, h)
    n_new = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    node = torch.arange(keys, device=k.device) - (s["n_kv"].long() - n_new)[:, None]      # which node a key is
    seen = torch.gather(_visible(s, req, j), 2, node.clamp(0, m - 1)[:, None].expand(-1, m, -1))
    seen = torch.where(node[:, None] < 0, True, seen) & (node < n_new[:, None])[:, None]
    seen = seen[:, None, :, None].expand(-1, 1, -1, hq // hkv, -1).reshape(batch, 1, -1, keys)
    x = (q @ k.transpose(2, 3)) / math.sqrt(h)
    x = torch.where(seen, x, -math.inf)
    x = x - x.amax(-1, keepdim=True)
    x = torch.exp(x)
    p = x / x.sum(-1, keepdim=True)
    o = (p @ v).view(batch, hkv, m, hq // hkv, h).permute(0, 2, 1, 3, 4).reshape(batch, m, hq, h)[req, j].to(s["q"].dtype)
    if s["op"] == "tree":
        return o
    real = torch.arange(m, device=k.device)[None, :] < n_new[:, None]
    p = torch.where(real[:, None, :, None, None], p.view(batch, hkv, m, hq // hkv, keys), 0).sum((2, 3))
    key = torch.arange(keys, device=k.device)
    i, x = torch.nonzero(key < s["n_kv"][:, None], as_tuple=True)
    page = s["page_table"].long()[i, x // PAGE]
    s["key_weights"][page, :, x % PAGE] += p[i, :, x]
    return {"out": o, "key_weights": s["key_weights"]}


def _evict_plain(s):
    k, v, w, table, n = s["k"], s["v"], s["key_weights"], s["page_table"].long(), s["n_kv"].long()
    layers, _, hkv = w.shape[:3]
    budget, sink, recent = s["budget"], s["sink"], s["recent"]
    keys = table.shape[1] * PAGE
    slot = torch.arange(keys, device=w.device)
    cut = (n > budget)[:, None]
    there = slot < n[:, None]
    late = there & (slot >= (n - recent)[:, None])
    fixed = there & (slot < sink) | late
    wx = w[:, table.clamp_min(0)].transpose(2, 3).reshape(layers, len(n), hkv, keys)
    rank = torch.where(fixed[:, None], math.inf, wx)
    rank = torch.where(there[:, None], rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order))
    keep = torch.where(cut[:, None], place < budget, there[:, None])
    # where every slot's key comes from: itself, or the next kept candidate from behind, or a recent one
    end = torch.where(cut[:, 0], budget - recent, n)[:, None, None]
    early = slot < end
    hole = early & ~keep & there[:, None]
    move = keep & ~early & ~late[:, None]
    of_hole = torch.cumsum(hole, -1) - 1
    movers = torch.sort((~move).to(torch.int8), dim=-1, stable=True).indices
    source = torch.where(hole, torch.gather(movers, -1, of_hole.clamp_min(0)), slot)
    source = torch.where(~early & cut[:, None], slot + (n[:, None, None] - budget), source)
    last = torch.where(cut[:, 0], budget, n)
    l, i, g, x = torch.nonzero((slot < last[:, None])[None, :, None].expand(layers, -1, hkv, -1), as_tuple=True)
    y = source[l, i, g, x]
    to, frm = (l, table[i, x // PAGE], g, x % PAGE), (l, table[i, y // PAGE], g, y % PAGE)
    s["key_weights_out"].index_put_(to, w[frm])
    moved = x != y
    to, frm = tuple(t[moved] for t in to), tuple(t[moved] for t in frm)
    k.index_put_(to, k[frm])
    v.index_put_(to, v[frm])
    return {"k": k, "v": v, "key_weights": s["key_weights_out"]}


def _bounds_plain(s):
    slot = torch.arange(s["page_table"].shape[1] * PAGE, device=s["k"].device).view(-1, PAGE)
    asked = (slot[:, 0] < s["n_kv"][:, None]) & (slot[:, -1] >= s["first"][:, None])
    i, p = torch.nonzero(asked, as_tuple=True)
    page = s["page_table"].long()[i, p]
    there = (slot[p] < s["n_kv"][i, None])[:, None, :, None]
    x = s["k"][page].float()
    low, high = torch.where(there, x, math.inf).amin(2), torch.where(there, x, -math.inf).amax(2)
    s["bounds"][page] = torch.stack([low, high], 2).to(s["bounds"].dtype)
    return s["bounds"]


def _blocks_plain(s):
    q = s["q"].float()
    total, hq, h = q.shape
    hkv = s["k"].shape[1]
    req, j = _rows(s)
    n_new = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    at = (s["n_kv"].long() - n_new)[req] + j                            # key index of every query
    table = s["page_table"].clamp_min(0).long()
    # scores in 64 bits: two blocks next to the border must not change places
    m, cols = s["most_nodes"], table.shape[1]
    qq = torch.zeros(len(n_new), m, hkv, hq // hkv, h, dtype=torch.float64, device=q.device)
    qq[req, j] = s["q"].double().view(total, hkv, -1, h)
    qq = qq.permute(0, 2, 1, 3, 4).reshape(len(n_new), hkv, -1, h)
    low, high = (s["bounds"][table][:, :, :, b].double().permute(0, 2, 3, 1) for b in (0, 1))
    score = qq.clamp_min(0) @ high + qq.clamp_max(0) @ low
    score = score.view(len(n_new), hkv, m, hq // hkv, cols).amax(3).transpose(1, 2)[req, j]      # [total, hkv, cols]
    block = torch.arange(cols, device=q.device)
    mine = (at // PAGE)[:, None, None]
    score = torch.where((block > mine - s["local"]) & (block <= mine), math.inf, score)
    score = torch.where(block <= mine, score, -math.inf)
    count = min(s["blocks"], cols)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :count]          # [total, hkv, count]
    page = table[req[:, None, None], best]
    head = torch.arange(hkv, device=q.device)[None, :, None]
    key = best[..., None] * PAGE + torch.arange(PAGE, device=q.device)
    seen = ((key <= at[:, None, None, None]) & (best <= mine)[..., None]).reshape(total, hkv, 1, -1)
    k = s["k"][page, head].float().reshape(total, hkv, -1, h)
    x = (q.view(total, hkv, -1, h) @ k.transpose(2, 3)) / math.sqrt(h)
    del k
    x = torch.where(seen, x, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    p = x / x.sum(-1, keepdim=True)
    v = s["v"][page, head].float().reshape(total, hkv, -1, h)
    v = torch.where(seen.transpose(2, 3), v, 0)
    return (p @ v).reshape(total, hq, h).to(s["q"].dtype)


PLAIN = {"tree": _tree_plain, "weigh": _tree_plain, "evict": _evict_plain, "bounds": _bounds_plain, "blocks": _blocks_plain}


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    if not own:
        return PLAIN[s["op"]](s)
    from paper_2506_09397_b200 import binding as B
    if s["op"] == "tree":
        return B.attention_tree(s["q"], s["k"], s["v"], s["page_table"], s["n_kv"], s["cu_q"], s["parents"])
    if s["op"] == "weigh":
        out = B.attention_tree(s["q"], s["k"], s["v"], s["page_table"], s["n_kv"], s["cu_q"], s["parents"],
                               key_weights=s["key_weights"])
        return {"out": out, "key_weights": s["key_weights"]}
    if s["op"] == "evict":
        B.evict_keys(s["k"], s["v"], s["key_weights"], s["page_table"], s["n_kv"], s["budget"], n_sink=s["sink"],
                     n_recent=s["recent"], key_weights_out=s["key_weights_out"])
        return {"k": s["k"], "v": s["v"], "key_weights": s["key_weights_out"]}
    if s["op"] == "bounds":
        B.block_bounds(s["k"], s["page_table"], s["n_kv"], s["bounds"], first=s["first"])
        return s["bounds"]
    return B.attention_blocks(s["q"], s["k"], s["v"], s["bounds"], s["page_table"], s["n_kv"], s["cu_q"],
                              n_blocks=s["blocks"], n_local=s["local"])


# --------------------------------------------------------------------------------- the definitions, in 64 bits
def _keys_of(pool, s, i):
    """Request i's rows of a pool, [kv heads, n, ...] in 64 bits."""
    n = int(s["n_kv"][i])
    pages = s["page_table"][i, :(n + PAGE - 1) // PAGE].long()
    return torch.cat(list(pool[pages].double()), 1)[:, :n]


def _exact_tree(s):
    cu, up = s["cu_q"].tolist(), s["parents"].tolist()
    total, hq, h = s["q"].shape
    out = torch.zeros(total, hq, h, dtype=torch.float64, device=s["q"].device)
    weights = s["key_weights"].double().clone() if s["op"] == "weigh" else None
    for i, n in enumerate(s["n_kv"].tolist()):
        k, v = _keys_of(s["k"], s, i), _keys_of(s["v"], s, i)
        hkv, m = k.shape[0], cu[i + 1] - cu[i]
        allowed = torch.zeros(m, n, dtype=torch.bool)
        allowed[:, :n - m] = True
        for j in range(m):
            a = j
            while a >= 0:
                allowed[j, n - m + a] = True
                a = up[cu[i] + a]
        allowed = allowed.to(k.device)
        x = torch.einsum("mgrd,gnd->grmn", s["q"][cu[i]:cu[i + 1]].double().view(m, hkv, -1, h), k) * h ** -0.5
        p = torch.softmax(x.masked_fill(~allowed, -math.inf), -1)
        out[cu[i]:cu[i + 1]] = torch.einsum("grmn,gnd->mgrd", p, v).reshape(m, hq, h)
        if weights is not None:
            per = p.sum((1, 2))
            for b, page in enumerate(s["page_table"][i, :(n + PAGE - 1) // PAGE].tolist()):
                here = per[:, b * PAGE:(b + 1) * PAGE]
                weights[page, :, :here.shape[1]] += here
    return out if weights is None else {"out": out, "key_weights": weights}


def _exact_evict(s):
    k, v, new = s["k"].clone(), s["v"].clone(), s["key_weights_out"].double().clone()
    layers, _, hkv = s["key_weights"].shape[:3]
    budget, sink, recent = s["budget"], s["sink"], s["recent"]
    for i, n in enumerate(s["n_kv"].tolist()):
        pages = s["page_table"][i, :(n + PAGE - 1) // PAGE].long()
        w = s["key_weights"][:, pages].double().cpu()                          # [layers, pages, hkv, PAGE]
        where = torch.arange(n)
        last = min(n, budget)
        for l in range(layers):
            for g in range(hkv):
                mine = w[l, :, g].reshape(-1)[:n].numpy()
                come = where.clone()
                if n > budget:
                    chosen = (sink + np.argsort(-mine[sink:n - recent], kind="stable")[:budget - sink - recent]).tolist()
                    held = set(chosen) | set(range(sink))
                    holes = [x for x in range(budget - recent) if x not in held]
                    for x, y in zip(holes, sorted(c for c in chosen if c >= budget - recent)):
                        come[x] = y
                    come[budget - recent:budget] = where[n - recent:n]
                come = come[:last]
                here = (pages[where[:last] // PAGE], (where[:last] % PAGE).to(pages.device))
                there = (pages[(come // PAGE).to(pages.device)], (come % PAGE).to(pages.device))
                new[l, here[0], g, here[1]] = s["key_weights"][l, there[0], g, there[1]].double()
                k[l, here[0], g, here[1]] = s["k"][l, there[0], g, there[1]]
                v[l, here[0], g, here[1]] = s["v"][l, there[0], g, there[1]]
    return {"k": k, "v": v, "key_weights": new}


def _exact_bounds(s):
    out = s["bounds"].double().clone()
    for i, (n, first) in enumerate(zip(s["n_kv"].tolist(), s["first"].tolist())):
        k = _keys_of(s["k"], s, i)
        for b in range(first // PAGE, (n + PAGE - 1) // PAGE):
            here = k[:, b * PAGE:(b + 1) * PAGE]
            out[int(s["page_table"][i, b])] = torch.stack([here.min(1).values, here.max(1).values], 1)
    return out


def _exact_blocks(s):
    cu = s["cu_q"].tolist()
    total, hq, h = s["q"].shape
    out = torch.zeros(total, hq, h, dtype=torch.float64, device=s["q"].device)
    for i, n in enumerate(s["n_kv"].tolist()):
        k, v = _keys_of(s["k"], s, i), _keys_of(s["v"], s, i)
        hkv = k.shape[0]
        pages = s["page_table"][i, :(n + PAGE - 1) // PAGE].long()
        bound = s["bounds"][pages].double()                                        # [blocks, hkv, 2, h]
        of_key = torch.arange(n, device=k.device) // PAGE
        for t in range(cu[i], cu[i + 1]):
            x = n - (cu[i + 1] - cu[i]) + t - cu[i]
            q = s["q"][t].double().view(hkv, -1, h)
            mine, early = x // PAGE, max(0, x // PAGE - s["local"] + 1)
            one = torch.maximum(q[None] * bound[:early, :, 0, None], q[None] * bound[:early, :, 1, None]).sum(-1).amax(-1)
            order = torch.argsort(one, dim=0, descending=True, stable=True)[:max(0, s["blocks"] - s["local"])]
            take = torch.zeros(mine + 1, hkv, dtype=torch.bool, device=k.device)
            take[early:] = True
            take.scatter_(0, order, True)
            allowed = take[of_key[:x + 1]].T
            y = torch.einsum("grd,gnd->grn", q, k[:, :x + 1]) / h ** 0.5
            p = torch.softmax(y.masked_fill(~allowed[:, None], -math.inf), -1)
            out[t] = (p @ v[:, :x + 1]).reshape(hq, h)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        if s["op"] in ("tree", "weigh"):
            return _exact_tree(s)
        if s["op"] == "evict":
            n_kv, _ = _sizes(case)
            if case["layers"] * GEOMETRY[case["geometry"]][1] * sum(n_kv) > 1e7:
                return None
            return _exact_evict(s)
        if s["op"] == "bounds":
            if sum(_sizes(case)[0]) > 1e6:
                return None
            return _exact_bounds(s)
        return _exact_blocks(s)
