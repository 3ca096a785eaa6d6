"""Operators of a decoding step over a caller's own paged cache: page tables and slot maps from lengths, rotary positions,
keys appended to the cache (in 8 bits, with a scale for each block of 16 tokens and head), attention over such a cache.

Each case can be computed in its plain form (`own` false: elementary torch operations in 32 bits, angles in 64) or by the
library's own calls (`own` true).  A cache is K, V [page][kv head][slot][head_dim]; request i's key x lies in page
page_table[i][x / page_size], slot x % page_size, and the last q_len of its n_kv keys are the new tokens.  A cache in 8 bits
holds e4m3 codes and, for every 16 slots of a page, a scale: scales [page][kv head][page_size / 16].  Page-table entries
behind a request's last page are -1, slots behind its last key hold what an earlier owner of the page left there.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16           # tokens that share a scale
LEAST = -126         # smallest exponent of a scale
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
        # one step of a serving batch: the rejected drafts of the last one go, the next drafts get their places
        {"name": "slots step", "op": "slots", "batch": 64, "lo": 512, "hi": 4096, "new_lo": 3, "new_hi": 9, "drop": 6, "page": 16},
        # a large batch of prompts arrives
        {"name": "slots prompts", "op": "slots", "batch": 300, "lo": 1, "hi": 700, "new_lo": 30, "new_hi": 8192, "drop": 0, "page": 16},
        # positions of a small decoding step
        {"name": "rotary step", "op": "rotary", "geometry": "8b", "tokens": 96, "style": "pairs", "part": 1.0, "scaling": "plain", "inverse": False, "far": 8192},
        # a chunk of prompts far out in a long context, queries and keys as slices of one projection
        {"name": "rotary prompts", "op": "rotary", "geometry": "8b", "tokens": 12011, "style": "halves", "part": 1.0, "scaling": "bands", "inverse": False, "far": 131072},
        # the gradient of a model that turns part of the head, 32-bit
        {"name": "rotary gradient", "op": "rotary", "geometry": "tiny", "tokens": 3001, "style": "halves", "part": 0.5, "scaling": "ramp", "inverse": True, "far": 32768},
        # the new tokens of a decoding step go into an 8-bit cache, most of them into blocks that have older keys
        {"name": "append step", "op": "append", "geometry": "8b", "cache": "e4m3", "batch": 48, "lo": 512, "hi": 8192, "new_lo": 1, "new_hi": 9, "page": 16},
        # prompts go into an 8-bit cache
        {"name": "append prompts", "op": "append", "geometry": "8b", "cache": "e4m3", "batch": 12, "lo": 0, "hi": 0, "new_lo": 2000, "new_hi": 16384, "page": 16},
        # a chunk of prompts goes into the 16-bit cache of the 1B model
        {"name": "append 16 bits", "op": "append", "geometry": "1b", "cache": "same", "batch": 20, "lo": 100, "hi": 3000, "new_lo": 200, "new_hi": 2000, "page": 32},
        # one device's small draft tree on the 1B model: the shortest call a server makes
        {"name": "attend one device", "op": "attend", "geometry": "1b", "batch": 1, "lo": 700, "hi": 700, "new_lo": 7, "new_hi": 7, "page": 16, "lse": False},
        # ordinary decoding of a batch of ragged contexts
        {"name": "attend tokens", "op": "attend", "geometry": "8b", "batch": 32, "lo": 128, "hi": 16384, "new_lo": 1, "new_hi": 1, "page": 16, "lse": True},
        # a few contexts of the greatest length, drafts
        {"name": "attend long", "op": "attend", "geometry": "8b", "batch": 4, "lo": 90000, "hi": 131072, "new_lo": 3, "new_hi": 5, "page": 16, "lse": False},
        # many devices with wide trees
        {"name": "attend wide", "op": "attend", "geometry": "8b", "batch": 64, "lo": 512, "hi": 4096, "new_lo": 48, "new_hi": 64, "page": 16, "lse": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slots", "rotary", "append", "attend", "attend"])
    if op == "rotary":
        return {"op": op, "geometry": rng.choice(["tiny", "1b", "8b", "gqa"]), "tokens": _log_int(rng, 1, 12000),
                "style": rng.choice(["pairs", "halves"]), "part": rng.choice([1.0, 0.5, 0.25]),
                "scaling": rng.choice(["plain", "linear", "bands", "ramp"]), "inverse": rng.random() < 0.3, "far": _log_int(rng, 500, 131072)}
    if op == "slots":
        most = rng.choice([1, 9, 40, 2000])
        lo = _log_int(rng, 10, 2000)
        return {"op": op, "batch": _log_int(rng, 1, 300), "lo": lo, "hi": _log_int(rng, lo, 8 * lo), "new_lo": rng.randint(0, most),
                "new_hi": most, "drop": rng.choice([0, 1, 8]), "page": rng.choice([16, 16, 32, 64])}
    geometry = rng.choice(["1b", "8b", "8b", "gqa"] if op == "attend" else ["tiny", "1b", "8b", "gqa"])
    lo = _log_int(rng, 40, 3000)
    case = {"op": op, "geometry": geometry, "batch": _log_int(rng, 1, 48), "lo": lo, "hi": min(16384, _log_int(rng, lo, 8 * lo)),
            "page": rng.choice([16, 16, 32, 64])}
    if op == "append":
        most = rng.choice([1, 9, 50, 1500])
        case.update(cache=rng.choice(["e4m3", "e4m3", "same"]), new_lo=rng.randint(1, most), new_hi=most)
    else:
        most = rng.choice([1, 1, 5, 9, 33])
        case.update(new_lo=rng.randint(1, most), new_hi=most, lse=rng.random() < 0.5)
        if rng.random() < 0.2:
            case.update(batch=rng.randint(1, 3), lo=16384, hi=_log_int(rng, 17000, 120000))
    return case


def _sizes(case):
    """Older keys, dropped ones among them and new tokens of every request: they follow from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k not in ("name", "lse"))))
    old, drop, new = [], [], []
    for _ in range(case["batch"]):
        n = _log_int(rng, case["lo"], case["hi"]) if case["lo"] else 0
        m = _log_int(rng, max(1, case["new_lo"]), case["new_hi"]) if case["new_hi"] > 64 else rng.randint(case["new_lo"], case["new_hi"])
        old.append(n)
        new.append(m)
        drop.append(rng.randint(0, min(n, case["drop"])) if case.get("drop") else 0)
    return old, drop, new


def _pages(n, page):
    return (n + page - 1) // page


def _tree(rng, m):
    """A draft tree: node 0 continues the cached text, every other node hangs on one of the nodes shortly before it."""
    return [-1] + [rng.randint(max(0, j - 6), j - 1) for j in range(1, m)]


def _rot(case):
    return max(2, int(GEOMETRY[case["geometry"]][2] * case["part"]) // 2 * 2)


def _frequencies(case):
    """Radians per position of every pair, in 64 bits, and what cosine and sine are multiplied by."""
    d = _rot(case)
    theta, factor, before = (1e4 if case["geometry"] == "tiny" else 5e5), 8.0, 8192.0
    f = theta ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "bands":      # low frequencies slowed down, high ones kept, smooth between 1 and 4 turns of the old length
        s = np.clip((before * f / (2 * math.pi) - 1) / (4 - 1), 0, 1)
        return f * (s + (1 - s) / factor), 1.0
    if case["scaling"] == "ramp":       # the same along the pairs' index, between those of 32 turns and 1, and a larger amplitude
        at = lambda turns: d * math.log(before / (turns * 2 * math.pi)) / (2 * math.log(theta))
        low, high = max(math.floor(at(32)), 0), min(math.ceil(at(1)), d - 1)
        s = 1 - np.clip((np.arange(d // 2) - low) / max(high - low, 0.001), 0, 1)
        return f * (s + (1 - s) / factor), 0.1 * math.log(factor) + 1
    return f, 1.0


def work(case):
    if case["op"] == "rotary":
        hq, hkv, h, t = GEOMETRY[case["geometry"]]
        n = case["tokens"] * (hq + hkv)
        return {"bytes": 2 * n * h * (4 if t == "fp32" else 2) + 4 * case["tokens"] + 4 * _rot(case), "flops": 3 * n * _rot(case)}
    old, drop, new = _sizes(case)
    page = case["page"]
    if case["op"] == "slots":
        taken = sum(max(0, _pages(n - d + m, page) - _pages(n, page)) for n, d, m in zip(old, drop, new))
        back = sum(max(0, _pages(n, page) - _pages(n - d + m, page)) for n, d, m in zip(old, drop, new))
        return {"bytes": 20 * len(old) + 8 * taken + 8 * back + 12 * sum(new), "flops": 0}
    hq, hkv, h, t = GEOMETRY[case["geometry"]]
    e = 4 if t == "fp32" else 2
    if case["op"] == "append":
        c = 1 if case["cache"] == "e4m3" else e
        blocks = sum(_pages(n + m, BLOCK) - n // BLOCK for n, m in zip(old, new))
        return {"bytes": 2 * sum(new) * hkv * h * (e + c) + (2 * blocks * hkv * 4 if c == 1 else 0) + 4 * blocks, "flops": 0}
    rows, keys = sum(new) * hq, sum(old) + sum(new)
    size = 2 * keys * hkv * h + 2 * sum(_pages(n + m, BLOCK) for n, m in zip(old, new)) * hkv * 4 + 2 * rows * h * e
    return {"bytes": size + 4 * sum(_pages(n + m, page) for n, m in zip(old, new)) + (4 * rows if case["lse"] else 0),
            "flops": sum(4 * h * m * hq * (n + m / 2) for n, m in zip(old, new))}


# --------------------------------------------------------------------------------------------------- the inputs
def _table(rng, counts, cols, n_pages):
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = np.full((len(counts), cols), -1, np.int32), 0
    for i, p in enumerate(counts):
        table[i, :p] = order[at:at + p]
        at += p
    return table, np.array(order[at:], np.int32)


def _ints(x, dev="cuda"):
    return torch.tensor(x, dtype=torch.int32).to(dev)


def _prepare_slots(case, seed):
    rng = random.Random(seed)
    page = case["page"]
    old, drop, new = _sizes(case)
    counts = [_pages(n, page) for n in old]
    after = [_pages(n - d + m, page) for n, d, m in zip(old, drop, new)]
    n_pages = sum(max(a, b) for a, b in zip(counts, after)) + rng.randint(3, 40)
    table, free = _table(rng, counts, max(max(a, b) for a, b in zip(counts, after)) + 2, n_pages)
    room = np.full(n_pages, -1, np.int32)
    room[:len(free)] = free
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
    rows = sum(new)
    return {"op": "slots", "page": page, "rows": rows, "n_kv": _ints(old), "n_keep": _ints([n - d for n, d in zip(old, drop)]), "n_new": _ints(new),
            "page_table": torch.from_numpy(table).cuda(), "free_pages": torch.from_numpy(room).cuda(), "n_free": _ints([len(free)]),
            "out": (i32(len(old)), i32(len(old) + 1), i32(rows), torch.empty(rows, dtype=torch.int64, device="cuda"), i32(1))}


def _projection(g, tokens, geometry):
    """Queries, keys and values of new tokens as slices of one projection; keys have a few channels that are much larger."""
    hq, hkv, h, t = GEOMETRY[geometry]
    x = torch.randn(tokens, hq + 2 * hkv, h, generator=g, device="cuda")
    x[:, hq:hq + hkv] *= 1 + 7 * (torch.rand(hkv, h, generator=g, device="cuda") < 1 / 16).float()
    x = x.to(TYPE[t])
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _prepare_rotary(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    q, k, _ = _projection(g, case["tokens"], case["geometry"])
    f, amplitude = _frequencies(case)
    positions, left = [], case["tokens"]
    while left:      # requests, each a run of positions
        m = min(left, _log_int(rng, 1, max(2, case["tokens"] // 3)))
        at = rng.randint(0, case["far"])
        positions += range(at, at + m)
        left -= m
    return {"op": "rotary", "q": q, "k": k, "positions": _ints(positions), "frequencies": torch.from_numpy(f).cuda(), "amplitude": amplitude,
            "style": case["style"], "inverse": case["inverse"], "q_out": torch.empty_like(q, memory_format=torch.contiguous_format),
            "k_out": torch.empty_like(k, memory_format=torch.contiguous_format)}


def _coded(x, whole):
    """Codes and scales of [page, kv heads, slot, head_dim]; whole: scales are powers of two."""
    p, g, s, h = x.shape
    y = x.view(p, g, s // BLOCK, BLOCK * h)
    scale = y.abs().amax(-1).clamp_min(1e-20) / 448
    if whole:
        scale = torch.exp2(torch.ceil(torch.log2(scale)))
    return (y / scale[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(p, g, s, h), scale


def _prepare_paged(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    hq, hkv, h, t = GEOMETRY[case["geometry"]]
    page = case["page"]
    old, _, new = _sizes(case)
    counts = [_pages(n + m, page) for n, m in zip(old, new)]
    n_pages = sum(counts) + 3
    table, _ = _table(rng, counts, max(counts), n_pages)
    s = {"op": case["op"], "page": page, "page_table": torch.from_numpy(table).cuda(), "n_kv": _ints([n + m for n, m in zip(old, new)]),
         "cu_q": _ints([0] + np.cumsum(new).tolist()), "most_new": max(new)}
    shape = (n_pages, hkv, page, h)
    if case["op"] == "append":
        _, s["k"], s["v"] = _projection(g, sum(new), case["geometry"])
        # what is there already: older tokens are somewhat smaller, so that blocks' scales have to grow now and then
        for name in ("k", "v"):
            x = torch.randn(shape, generator=g, device="cuda") * 0.7
            if case["cache"] == "e4m3":
                s[name + "_cache"], s[name + "_scale"] = _coded(x, True)
            else:
                s[name + "_cache"] = x.to(TYPE[t])
        return s
    # queries of a head have a direction in common, and the keys of one page in sixteen lean that way: those draw the
    # attention, as a few places of a text do; blocks differ in size
    way = torch.randn(hkv, 1, h, generator=g, device="cuda")
    lean = (torch.rand(n_pages, 1, 1, 1, generator=g, device="cuda") < 1 / 16).float() * 0.4
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device="cuda")
        x *= torch.exp(0.2 * torch.randn(n_pages, hkv, 1, 1, generator=g, device="cuda"))
        if name == "k":
            x += lean * way
        s[name], s[name + "_scale"] = _coded(x, False)
        del x
    q = torch.randn(sum(new), hkv, hq // hkv, h, generator=g, device="cuda") * 0.8 + 0.6 * way
    s["q"] = q.reshape(sum(new), hq, h).to(TYPE[t])
    s["parents"] = None if max(new) == 1 else _ints(sum((_tree(rng, m) for m in new), []))
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(sum(new), hq, device="cuda") if case["lse"] else None
    return s


def prepare(case, seed):
    if case["op"] == "slots":
        return _prepare_slots(case, seed)
    return _prepare_rotary(case, seed) if case["op"] == "rotary" else _prepare_paged(case, seed)


# ----------------------------------------------------------------------------------------------- the plain forms
def _slots_plain(s):
    n_kv, n_keep, n_new, table, free = s["n_kv"].long(), s["n_keep"].long(), s["n_new"].long(), s["page_table"], s["free_pages"]
    page, n_free = s["page"], s["n_free"].long()
    have, want = (n_kv + page - 1) // page, (n_keep + n_new + page - 1) // page
    take, back = (want - have).clamp_min(0), (have - want).clamp_min(0)
    col = torch.arange(table.shape[1], device=table.device)
    # the pages that are no longer needed go on top of the free ones, request by request in ascending order
    i, c = torch.nonzero((col >= want[:, None]) & (col < have[:, None]), as_tuple=True)
    before = torch.cumsum(back, 0) - back
    free[n_free + before[i] + c - want[i]] = table[i, c]
    top = n_free + back.sum()
    # new ones come from the top, request by request
    before = torch.cumsum(take, 0) - take
    i, c = torch.nonzero((col >= have[:, None]) & (col < want[:, None]), as_tuple=True)
    table[i, c] = free[top - 1 - (before[i] + c - have[i])]
    cu = torch.cat([torch.zeros_like(n_new[:1]), torch.cumsum(n_new, 0)])
    t = torch.arange(s["rows"], device=table.device)
    req = torch.searchsorted(cu, t, right=True) - 1
    at = n_keep[req] + t - cu[req]
    slots = table[req, at // page].long() * page + at % page
    i32 = torch.int32
    return {"n_kv": (n_keep + n_new).to(i32), "cu_q": cu.to(i32), "positions": at.to(i32), "slots": slots, "n_free": (top - take.sum()).to(i32),
            "page_table": table, "free_pages": free}


def _turn(x, cos, sin, style, inverse):
    d = 2 * cos.shape[-1]
    y = x[..., :d].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if style == "pairs" else (y[..., :d // 2], y[..., d // 2:])
    if inverse:
        sin = -sin
    u, w = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([u, w], -1).flatten(-2) if style == "pairs" else torch.cat([u, w], -1)
    return torch.cat([y.to(x.dtype), x[..., d:]], -1)


def _rotary_plain(s):
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    return {"q": _turn(s["q"], cos, sin, s["style"], s["inverse"]), "k": _turn(s["k"], cos, sin, s["style"], s["inverse"])}


def _append_plain(s):
    page, table, n = s["page"], s["page_table"].long(), s["n_kv"].long()
    cu = s["cu_q"].long()
    first = n - (cu[1:] - cu[:-1])
    per = page // BLOCK
    block = torch.arange(table.shape[1] * per, device=n.device)
    i, b = torch.nonzero((block * BLOCK < n[:, None]) & (block * BLOCK + BLOCK > first[:, None]), as_tuple=True)
    at = b[:, None] * BLOCK + torch.arange(BLOCK, device=n.device)                    # [blocks, 16]: keys
    fresh, older = (at >= first[i, None]) & (at < n[i, None]), at < first[i, None]
    row = torch.where(fresh, cu[i, None] + at - first[i, None], 0)
    where = table[i, b // per]
    done = {}
    for name in ("k", "v"):
        cache = s[name + "_cache"]
        rows = s[name][row].transpose(1, 2)                                           # [blocks, kv heads, 16, h]
        new = fresh[:, None, :, None]
        if cache.dtype == s[name].dtype:
            blocks = cache.view(cache.shape[0], cache.shape[1], per, BLOCK, -1)
            blocks[where, :, b % per] = torch.where(new, rows, blocks[where, :, b % per])
            done[name + "_cache"] = cache
            continue
        codes, scales = cache.view(torch.uint8).view(cache.shape[0], cache.shape[1], per, BLOCK, -1), s[name + "_scale"]
        x = torch.where(new, rows.float(), 0)
        f, e = torch.frexp(torch.where(torch.isfinite(x), x.abs(), 0).amax((2, 3)))    # the largest is f 2^e; 448 = 0.875 2^9
        least = torch.where(f > 0.875, e - 8, e - 9).clamp_min(LEAST)
        least = torch.where(f == 0, torch.full_like(least, LEAST), least)
        before = torch.where(older[:, :1], scales[where, :, b % per], 0)
        scale = torch.maximum(torch.exp2(least.float()), before)
        mine = codes[where, :, b % per]
        kept = mine.view(torch.float8_e4m3fn).float() * before[:, :, None, None]
        y = torch.where(new, x, torch.where(older[:, None, :, None], kept, 0)) / scale[:, :, None, None]
        y = y.to(torch.float8_e4m3fn).view(torch.uint8)
        codes[where, :, b % per] = torch.where(new | older[:, None, :, None], y, mine)
        scales[where, :, b % per] = scale
        done.update({name + "_cache": cache, name + "_scale": scales})
    return done


def _gathered(s, name):
    """[batch, kv heads, keys, head_dim] in 32 bits; keys that a request lacks are zero."""
    table = s["page_table"].clamp_min(0).long()
    x = s[name].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()           # [batch, cols, kv heads, page, h]
    x = x.view(*x.shape[:3], -1, BLOCK, x.shape[-1]) * s[name + "_scale"][table][..., None, None]
    x = x.flatten(3, 4).transpose(1, 2).flatten(2, 3)
    there = torch.arange(x.shape[2], device=x.device) < s["n_kv"][:, None]
    return torch.where(there[:, None, :, None], x, 0)


def _seen(s, req, j, n_new, keys):
    """[batch, new tokens, keys]: the older keys, itself and its ancestors (of a chain: all tokens before it)."""
    m, dev = s["most_new"], s["q"].device
    batch = len(n_new)
    node = torch.arange(keys, device=dev) - (s["n_kv"].long() - n_new)[:, None]       # which new token a key is
    if s["parents"] is None:
        sees = torch.tril(torch.ones(m, m, dtype=torch.bool, device=dev)).expand(batch, m, m)
    else:
        step = torch.eye(m, dtype=torch.float64, device=dev).repeat(batch, 1, 1)
        up = s["parents"].long()
        step.index_put_((req, j, torch.where(up >= 0, up, j)), torch.ones_like(up, dtype=torch.float64))
        sees = torch.linalg.matrix_power(step, m) > 0
    seen = torch.gather(sees, 2, node.clamp(0, m - 1)[:, None].expand(-1, m, -1))
    return torch.where(node[:, None] < 0, True, seen) & (node < n_new[:, None])[:, None]


def _attend_plain(s):
    total, hq, h = s["q"].shape
    k, v = _gathered(s, "k"), _gathered(s, "v")
    batch, hkv, keys = k.shape[:3]
    m, cu = s["most_new"], s["cu_q"].long()
    t = torch.arange(total, device=k.device)
    req = torch.searchsorted(cu, t, right=True) - 1
    j = t - cu[req]
    q = torch.zeros(batch, m, hq, h, device=k.device)
    q[req, j] = s["q"].float()
    q = q.view(batch, m, hkv, hq // hkv, h).permute(0, 2, 1, 3, 4).reshape(batch, hkv, -1, h)
    seen = _seen(s, req, j, cu[1:] - cu[:-1], keys)
    seen = seen[:, None, :, None].expand(-1, 1, -1, hq // hkv, -1).reshape(batch, 1, -1, keys)
    x = (q @ k.transpose(2, 3)) / math.sqrt(h)
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - top)
    total_p = x.sum(-1, keepdim=True)
    back = lambda y: y.view(batch, hkv, m, hq // hkv, -1).permute(0, 2, 1, 3, 4).reshape(batch, m, hq, -1)[req, j]
    o = {"out": back((x / total_p) @ v).to(s["q"].dtype)}
    if s["lse"] is not None:
        o["lse"] = back(top + torch.log(total_p))[..., 0]
    return o


PLAIN = {"slots": _slots_plain, "rotary": _rotary_plain, "append": _append_plain, "attend": _attend_plain}


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    if not own:
        return PLAIN[s["op"]](s)
    from paper_2506_09397_b200 import binding as B
    if s["op"] == "slots":
        o = B.page_slots(s["n_kv"], s["n_new"], s["page_table"], s["free_pages"], s["n_free"], page_size=s["page"], n_rows=s["rows"],
                         n_keep=s["n_keep"], out=s["out"])
        return {"n_kv": o[0], "cu_q": o[1], "positions": o[2], "slots": o[3], "n_free": o[4], "page_table": s["page_table"],
                "free_pages": s["free_pages"]}
    if s["op"] == "rotary":
        q, k = B.rotary(s["q"], s["k"], s["positions"], s["frequencies"], style=s["style"], amplitude=s["amplitude"], inverse=s["inverse"],
                        q_out=s["q_out"], k_out=s["k_out"])
        return {"q": q, "k": k}
    if s["op"] == "append":
        B.append_keys(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"], s["n_kv"], s["cu_q"], k_scale=s.get("k_scale"),
                      v_scale=s.get("v_scale"))
        return {name: s[name] for name in ("k_cache", "k_scale", "v_cache", "v_scale") if name in s}
    out = B.attention_tree(s["q"], s["k"], s["v"], s["page_table"], s["n_kv"], s["cu_q"], s["parents"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                           out=s["out"], lse=s["lse"])
    return {"out": out} if s["lse"] is None else {"out": out, "lse": s["lse"]}


# --------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_slots(s):
    page = s["page"]
    table, room = s["page_table"].cpu().numpy().copy(), s["free_pages"].cpu().numpy().copy()
    free = room[:int(s["n_free"])].tolist()
    was, keep, new = (s[x].tolist() for x in ("n_kv", "n_keep", "n_new"))
    for i in range(len(was)):
        free += table[i, _pages(keep[i] + new[i], page):_pages(was[i], page)].tolist()
    room[:len(free)] = free
    positions, slots, cu = [], [], [0]
    for i in range(len(was)):
        for c in range(_pages(was[i], page), _pages(keep[i] + new[i], page)):
            table[i, c] = free.pop()
        at = np.arange(keep[i], keep[i] + new[i])
        positions.append(at)
        slots.append(table[i, at // page].astype(np.int64) * page + at % page)
        cu.append(cu[-1] + new[i])
    whole = lambda x, t: torch.from_numpy(np.asarray(x, t))
    return {"n_kv": whole([a + b for a, b in zip(keep, new)], np.int32), "cu_q": whole(cu, np.int32), "positions": whole(np.concatenate(positions), np.int32),
            "slots": whole(np.concatenate(slots), np.int64), "n_free": whole([len(free)], np.int32), "page_table": torch.from_numpy(table),
            "free_pages": torch.from_numpy(room)}


def _exact_rotary(case, s):
    f, amplitude = _frequencies(case)
    d, half = 2 * len(f), len(f)
    # a turn is a product with exp(i angle); positions and frequencies multiplied in extended precision
    angle = np.asarray(s["positions"].cpu().numpy(), np.longdouble)[:, None] * np.asarray(f, np.longdouble)
    angle = np.asarray(np.remainder(angle, 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))), np.float64)
    turn = torch.from_numpy(amplitude * np.exp((-1j if s["inverse"] else 1j) * angle)).cuda()[:, None]
    o = {}
    for name in ("q", "k"):
        x = s[name].double()
        at = torch.arange(half, device=x.device)
        a, b = (2 * at, 2 * at + 1) if s["style"] == "pairs" else (at, at + half)
        z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * turn
        y = x.clone()
        y[..., a], y[..., b] = z.real, z.imag
        assert d <= y.shape[-1]
        o[name] = y
    return o


def _nearest_code(x):
    """The e4m3 number next to x, ties to an even mantissa."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6)))
    e = torch.where(torch.exp2(e) > x.abs().clamp_min(2.0 ** -6), e - 1, e)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    page, per, o = s["page"], s["page"] // BLOCK, {}
    cu, n_kv, table = s["cu_q"].tolist(), s["n_kv"].tolist(), s["page_table"].cpu()
    for name in ("k", "v"):
        cache = s[name + "_cache"].double().clone()
        coded = name + "_scale" in s
        scales = s[name + "_scale"].double().clone() if coded else None
        rows = s[name].double()
        for i, n in enumerate(n_kv):
            first = n - (cu[i + 1] - cu[i])
            if not coded:
                x = torch.arange(first, n)
                where = table[i, x // page].long().to(cache.device)
                cache[where, :, (x % page).to(cache.device)] = rows[cu[i]:cu[i + 1]]
                continue
            for whole in (True, False):       # blocks that have older keys one by one, the others of a request all at once
                starts = torch.arange(first // BLOCK, (n + BLOCK - 1) // BLOCK)
                starts = starts[starts * BLOCK >= first] if whole else starts[starts * BLOCK < first]
                if not len(starts):
                    continue
                at = starts[:, None] * BLOCK + torch.arange(BLOCK)
                there = (at >= first) & (at < n)
                x = rows[(cu[i] + at - first).clamp(cu[i], cu[i + 1] - 1).to(rows.device)].transpose(1, 2)     # [blocks, heads, 16, h]
                x = torch.where(there[:, None, :, None].to(x.device), x, 0)
                where, sub = table[i, starts // per].long().to(x.device), (starts % per).to(x.device)
                most = x.abs().amax((2, 3))
                least = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp_min(LEAST))
                least = torch.where(least / 2 * 448 >= most, (least / 2).clamp_min(2.0 ** LEAST), least)
                before = torch.zeros_like(least) if whole else scales[where, :, sub]
                scale = torch.maximum(least, before)
                slot = sub[:, None] * BLOCK + torch.arange(BLOCK, device=x.device)
                mine = cache[where[:, None], :, slot].transpose(1, 2)
                y = torch.where(there[:, None, :, None].to(x.device), x, mine * before[:, :, None, None])
                y = _nearest_code(y / scale[:, :, None, None])
                y = torch.where((at < n)[:, None, :, None].to(x.device), y, mine)
                cache[where[:, None], :, slot] = y.transpose(1, 2)
                scales[where, :, sub] = scale
        o[name + "_cache"] = cache
        if coded:
            o[name + "_scale"] = scales
    return o


def _exact_attend(s):
    cu, up = s["cu_q"].tolist(), None if s["parents"] is None else s["parents"].tolist()
    total, hq, h = s["q"].shape
    out = torch.zeros(total, hq, h, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(total, hq, dtype=torch.float64, device=s["q"].device)
    for i, n in enumerate(s["n_kv"].tolist()):
        pages = s["page_table"][i, :_pages(n, s["page"])].long()
        kv = []
        for name in ("k", "v"):
            codes = torch.cat(list(s[name].view(torch.uint8)[pages]), 1)[:, :n].view(torch.float8_e4m3fn).double()
            scale = torch.cat(list(s[name + "_scale"][pages]), 1).double().repeat_interleave(BLOCK, 1)[:, :n]
            kv.append(codes * scale[..., None])
        m = cu[i + 1] - cu[i]
        allowed = torch.zeros(m, n, dtype=torch.bool)
        allowed[:, :n - m] = True
        for j in range(m):
            a = j
            while a >= 0:
                allowed[j, n - m + a] = True
                a = a - 1 if up is None else up[cu[i] + a]
        allowed = allowed.to(out.device)
        hkv = kv[0].shape[0]
        x = torch.einsum("mgrd,gnd->grmn", s["q"][cu[i]:cu[i + 1]].double().view(m, hkv, -1, h), kv[0]) * h ** -0.5
        x = x.masked_fill(~allowed, -math.inf)
        lse[cu[i]:cu[i + 1]] = torch.logsumexp(x, -1).permute(2, 0, 1).reshape(m, hq)
        out[cu[i]:cu[i + 1]] = torch.einsum("grmn,gnd->mgrd", torch.softmax(x, -1), kv[1]).reshape(m, hq, h)
    return {"out": out} if s["lse"] is None else {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        if s["op"] == "slots":
            return _exact_slots(s)
        if s["op"] == "rotary":
            return _exact_rotary(case, s)
        return _exact_append(s) if s["op"] == "append" else _exact_attend(s)
