"""64-bit statements of a decoding step's operators over a caller's paged cache: places of new tokens, rotary positions, keys
appended in 8 bits, attention over codes with scales.  Shares nothing with the library."""
import math

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
BLOCK = 16


def up(a, b):
    return (a + b - 1) // b


def slots(n_kv, n_keep, n_new, table, free, n_free, page, n_rows):
    """table [n_reqs, cols] and free (numpy) as they are before the call; None where it cannot be done, else
    (n_kv, cu_q, positions, slots, n_free, table, free)."""
    table, free = table.copy(), free.copy()
    stack = free[:n_free].tolist()
    back = []
    for i, (n, k, m) in enumerate(zip(n_kv, n_keep, n_new)):
        back += table[i, up(k + m, page):up(n, page)].tolist()
    stack += back
    free[n_free:n_free + len(back)] = back
    if sum(max(0, up(k + m, page) - up(n, page)) for n, k, m in zip(n_kv, n_keep, n_new)) > len(stack):
        return None
    positions, places, cu = np.zeros(n_rows, np.int32), np.full(n_rows, -1, np.int64), [0]
    for i, (n, k, m) in enumerate(zip(n_kv, n_keep, n_new)):
        for c in range(up(n, page), up(k + m, page)):
            table[i, c] = stack.pop()
        x = np.arange(k, k + m)
        positions[cu[-1]:cu[-1] + m] = x
        places[cu[-1]:cu[-1] + m] = table[i, x // page].astype(np.int64) * page + x % page
        cu.append(cu[-1] + m)
    return [k + m for k, m in zip(n_keep, n_new)], cu, positions, places, len(stack), table, free


def rotary(x, positions, frequencies, halves, amplitude, inverse):
    """x [rows, heads, h] -> (turned in 64 bits, bound of a 32-bit kernel's error before its result is rounded)."""
    f = np.asarray(frequencies, np.longdouble)
    angle = np.asarray(positions, np.longdouble)[:, None] * f
    two_pi = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    turn = amplitude * np.exp((-1j if inverse else 1j) * np.asarray(angle - two_pi * np.rint(angle / two_pi), np.float64))[:, None]
    half = len(f)
    y = x.double().numpy().copy()
    a, b = (slice(0, half), slice(half, 2 * half)) if halves else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = (y[..., a] + 1j * y[..., b]) * turn
    size = np.abs(y[..., a]) + np.abs(y[..., b])
    y[..., a], y[..., b] = z.real, z.imag
    # sine and cosine: two units in the last place, a correction and the amplitude, then a product and a sum: 2^-22 + 5 2^-24; the
    # angle is formed of products in 64 bits, off by 4 roundings of its size
    off = np.zeros_like(y)
    off[..., a] = off[..., b] = abs(amplitude) * size * (2.0 ** -22 + 5 * 2.0 ** -24 + 4 * 2.0 ** -53 * np.abs(np.asarray(angle, np.float64))[:, None])
    return torch.from_numpy(y), torch.from_numpy(off)


def nearest_code(x):
    """The e4m3 number next to x (64 bits, at most 448 away from 0), ties to the one of even mantissa."""
    size = x.abs().clamp_min(2.0 ** -6)
    e = torch.floor(torch.log2(size))
    e = torch.where(torch.exp2(e) > size, e - 1, e)
    return torch.round(x / torch.exp2(e - 3)) * torch.exp2(e - 3)


def append(rows, codes, scales, table, n, first, page):
    """One request's rows [m, hkv, h] as keys first .. n-1 into codes [n_pages, hkv, page, h] (their values, 64 bits) and scales, in place."""
    for b in range(first // BLOCK, up(n, BLOCK)):
        lo, hi = max(first, b * BLOCK), min(n, (b + 1) * BLOCK)
        p, sub = int(table[b * BLOCK // page]), b * BLOCK % page // BLOCK
        s0 = b * BLOCK % page
        for g in range(codes.shape[1]):
            x = rows[lo - first:hi - first, g].double()
            most = float(torch.where(x.isfinite(), x.abs(), 0).max())
            e = -126
            while most > 448 * 2.0 ** e:
                e += 1
            before = float(scales[p, g, sub]) if lo > b * BLOCK else 0.0
            s = max(2.0 ** e, before)
            quotient = lambda y: (y.float() / torch.tensor(s, dtype=torch.float32)).double()     # a quotient of 32 bits
            y = torch.where(x.isfinite(), nearest_code(quotient(torch.where(x.isfinite(), x, 0))), math.nan)
            codes[p, g, s0 + lo % BLOCK:s0 + lo % BLOCK + hi - lo] = y
            if lo > b * BLOCK and s != before:
                old = codes[p, g, s0:s0 + lo % BLOCK]
                codes[p, g, s0:s0 + lo % BLOCK] = nearest_code(quotient((old.float() * before)))
            scales[p, g, sub] = s


def coded(x, whole=True):
    """Codes (e4m3) and scales of [n_pages, hkv, page, h]; NaN stays."""
    p, g, s, h = x.shape
    y = x.float().view(p, g, s // BLOCK, BLOCK * h)
    scale = y.abs().nan_to_num(0).amax(-1).clamp_min(1e-20) / 448
    if whole:
        scale = torch.exp2(torch.ceil(torch.log2(scale)))
    return (y / scale[..., None]).clamp(-448, 448).to(E4M3).view(p, g, s, h), scale


def values(codes, scales):
    """What a cache in 8 bits stands for, in 64 bits."""
    p, g, s, h = codes.shape
    return (codes.double().view(p, g, s // BLOCK, BLOCK, h) * scales.double()[..., None, None]).view(p, g, s, h)
