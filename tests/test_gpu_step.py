"""A decoding step's operators over a caller's paged cache against 64-bit statements of them (tests/step_ref.py, and
tests/paged_ref.py for attention): places of new tokens, rotary positions, keys appended in 8 bits or as they are, attention over
a cache in 8 bits, and the four in a row."""
import math
import random

import numpy as np
import paged_ref as R
import pytest
import step_ref as S
import torch

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]).tolist() if len(lens) else [0])


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------- places
def _slots_case(rng, n_kv, n_keep, n_new, page, *, spare=3, extra_rows=0, cols=None, short=0):
    """Runs the call and compares everything with the statement."""
    have = [S.up(n, page) for n in n_kv]
    want = [S.up(k + m, page) for k, m in zip(n_keep, n_new)]
    cols = cols or max([1] + have + want)
    order = list(range(sum(have) + sum(max(0, b - a) for a, b in zip(have, want)) + spare))
    rng.shuffle(order)
    table = np.full((len(n_kv), cols), -5, np.int32)
    for i, p in enumerate(have):
        table[i, :p] = [order.pop() for _ in range(p)]
    n_free = len(order) - short
    free = np.full(len(order) + sum(max(0, a - b) for a, b in zip(have, want)), -9, np.int32)
    free[:len(order)] = order
    rows = sum(n_new) + extra_rows
    want_all = S.slots(n_kv, n_keep, n_new, table, free, n_free, page, rows)
    d_table = torch.full((len(n_kv), cols + 2), -6, dtype=torch.int32, device="cuda")     # a slice: rows are further apart
    d_table[:, :cols] = torch.from_numpy(table)
    d_free, status = torch.from_numpy(free.copy()).cuda(), _status()
    args = (_i32(n_kv), _i32(n_new), d_table[:, :cols], d_free, _i32([n_free]))
    for again in range(2):     # the inputs are as they were: the call can be repeated
        o = B.page_slots(*args, page_size=page, n_rows=rows, n_keep=_i32(n_keep), status=status)
        assert bool((d_table[:, cols:] == -6).all())
        if want_all is None:
            with pytest.raises(B.SledError) as e:
                B.check_status(status)
            assert e.value.code == B.SLED_ERR_NO_PAGES
            want = (n_kv, [0] * (len(n_kv) + 1), np.zeros(rows), np.full(rows, -1), n_free, table, free)
        else:
            B.check_status(status)
            want = want_all
        got = (o.n_kv, o.cu_q, o.positions, o.slots, o.n_free, d_table[:, :cols], d_free)
        for name, x, y in zip(("n_kv", "cu_q", "positions", "slots", "n_free", "table", "free"), got, want):
            assert np.array_equal(x.cpu().numpy().reshape(-1), np.asarray(y).reshape(-1)), (name, again)
    if list(n_keep) == list(n_kv):
        o = B.page_slots(*args, page_size=page, n_rows=rows)
        assert np.array_equal(o.n_kv.cpu().numpy(), np.asarray(want[0]).reshape(-1))
    return o


@pytest.mark.parametrize("page", [1, 3, 16, 64, 256])
@pytest.mark.parametrize("batch", [1, 2, 31, 257, 1000])
def test_places(batch, page):
    rng = random.Random(batch * 1000 + page)
    n_kv = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, 5 * page)]) for _ in range(batch)]
    keep = [rng.choice([n, n, max(0, n - 1), rng.randint(0, n)]) for n in n_kv]
    new = [rng.choice([0, 1, page, rng.randint(0, 3 * page)]) for _ in range(batch)]
    _slots_case(rng, n_kv, keep, new, page, extra_rows=rng.choice([0, 5]))
    _slots_case(rng, n_kv, n_kv, new, page, spare=0)


def test_places_of_prompts_and_of_nobody():
    rng = random.Random(1)
    _slots_case(rng, [0, 100, 7], [0, 90, 0], [70000, 0, 12345], 16)
    _slots_case(rng, [], [], [], 16)
    _slots_case(rng, [], [], [], 16, extra_rows=300)
    _slots_case(rng, [5], [0], [0], 16)


@pytest.mark.parametrize("batch", [8192, 8193, 20000, 65535])
def test_places_of_very_many_requests(batch):
    rng = random.Random(batch)
    n_kv = [rng.randint(0, 40) for _ in range(batch)]
    keep = [rng.randint(max(0, n - 20), n) for n in n_kv]
    _slots_case(rng, n_kv, keep, [rng.choice([0, 0, 1, 2, 30]) for _ in range(batch)], 16)


def test_returned_pages_serve_at_once():
    rng = random.Random(7)
    # nothing is free; three requests give back what two others need, exactly
    _slots_case(rng, [160, 0, 160, 16, 90], [0, 0, 33, 16, 80], [0, 100, 0, 60, 5], 16, spare=0, short=10)
    assert S.slots([160, 0], [0, 0], [0, 160], np.arange(20, dtype=np.int32).reshape(2, 10), np.zeros(10, np.int32), 0, 16, 160) is not None


def test_too_few_pages_move_nothing():
    rng = random.Random(8)
    _slots_case(rng, [16, 40, 3], [16, 20, 3], [17, 0, 14], 16, spare=0, short=2, extra_rows=2)


@pytest.mark.parametrize("change", [dict(n_kv=[-1, 5]), dict(n_new=[1, -1]), dict(n_keep=[4, 5]), dict(n_keep=[-1, 5]), dict(n_new=[62, 1]), dict(n_kv=[65, 5]),
                                    dict(n_new=[9, 9]), dict(n_free=-1), dict(n_free=9), dict(n_new=[2 ** 31 - 1, 2 ** 31 - 1])], ids=str)
def test_numbers_that_do_not_hold_together_move_nothing(change):
    a = dict(n_kv=[3, 5], n_keep=[3, 5], n_new=[2, 3], n_free=4)
    a.update(change)
    table = torch.full((2, 4), 77, dtype=torch.int32, device="cuda")
    free, status = _i32(list(range(8))), _status()
    o = B.page_slots(_i32(a["n_kv"]), _i32(a["n_new"]), table, free, _i32([a["n_free"]]), page_size=16, n_rows=10, n_keep=_i32(a["n_keep"]), status=status)
    assert status.item() == B.SLED_ERR_ARG
    assert o.n_kv.tolist() == a["n_kv"] and o.n_free.item() == a["n_free"] and o.cu_q.tolist() == [0, 0, 0]
    assert o.positions.tolist() == [0] * 10 and o.slots.tolist() == [-1] * 10
    assert bool((table == 77).all()) and free.tolist() == list(range(8))


def test_places_refuse_what_the_binding_sees():
    i, t, f = _i32([1]), _i32([[0, 1]]), _i32([2, 3])
    for call in (lambda: B.page_slots(i, i, t, f, i, page_size=16, n_rows=-1), lambda: B.page_slots(i, i, t[0], f, i, page_size=16, n_rows=1),
                 lambda: B.page_slots(i, _i32([1, 2]), t, f, i, page_size=16, n_rows=1), lambda: B.page_slots(i, i.long(), t, f, i, page_size=16, n_rows=1),
                 lambda: B.page_slots(i, i, t, f, i, page_size=0, n_rows=1), lambda: B.page_slots(i, i.cpu(), t, f, i, page_size=16, n_rows=1),
                 lambda: B.page_slots(i, i, t, f, i, page_size=16, n_rows=1, out=(i, _i32([0, 0]), i.clone(), i.long(), i.clone()))):
        with pytest.raises(B.SledError) as e:
            call()
        assert e.value.code == B.SLED_ERR_ARG


# ------------------------------------------------------------------------------------------------------- rotary
def _rotary_check(q, k, positions, f, style, amplitude, inverse, **out):
    want = [None if x is None else S.rotary(x.cpu(), positions, f.numpy(), style == "halves", amplitude, inverse) for x in (q, k)]
    before = [None if x is None else x.clone() for x in (q, k)]
    got = B.rotary(q, k, _i32(positions), f.cuda(), style=style, amplitude=amplitude, inverse=inverse, **out)
    for x, was, y, w in zip((q, k), before, got, want):
        if x is None:
            assert y is None
            continue
        if y.data_ptr() != x.data_ptr():
            assert torch.equal(x, was)
        z = y.cpu().double()
        e = R.EPS[x.dtype]
        bad = (z - w[0]).abs() - (w[1] + e * (w[0].abs() + w[1]) + 1e-37)
        assert float(bad.max()) <= 0, float(bad.max())
        d = 2 * f.numel()
        assert torch.equal(y[..., d:], was[..., d:])
    return got


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("h,rot,hq,hk", [(128, 128, 32, 8), (64, 64, 4, 4), (64, 32, 5, 1), (128, 32, 8, 2), (96, 40, 3, 3), (6, 2, 2, 1), (10, 6, 3, 2),
                                         (256, 256, 7, 1), (512, 512, 2, 2), (80, 80, 1, 1), (2, 2, 40, 8), (136, 128, 2, 1)])
def test_rotary(h, rot, hq, hk, style, dtype):
    g = torch.Generator().manual_seed(h + rot)
    f, a = B.rotary_frequencies(rot, 1e4)
    for rows in (1, 3, 70):
        q, k = (torch.randn(rows, n, h, generator=g).to(dtype).cuda() for n in (hq, hk))
        positions = torch.randint(-100, 140000, (rows,), generator=g).tolist()
        _rotary_check(q, k, positions, f, style, a, rows == 3)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_rotary_of_a_long_chunk_in_slices_of_a_projection(style, dtype):
    g = torch.Generator().manual_seed(5)
    f, a = B.rotary_frequencies(64, 5e5, scaling=B.ROTARY_RAMP, factor=8.0, length=8192, low=1.0, high=32.0)
    x = torch.randn(2501, 8 + 2 * 2, 64, generator=g).to(dtype).cuda()
    positions = list(range(120000, 120000 + 2501))
    for inverse in (False, True):
        _rotary_check(x[:, :8], x[:, 8:10], positions, f, style, a, inverse)
    # in place, values untouched
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:].clone()
    want = B.rotary(q, k, _i32(positions), f.cuda(), style=style, amplitude=a)
    got = B.rotary(q, k, _i32(positions), f.cuda(), style=style, amplitude=a, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, 10:], v)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_rotary_of_any_strides(style, dtype):
    g = torch.Generator().manual_seed(6)
    f, a = B.rotary_frequencies(32, 1e4)
    base = torch.randn(40000, generator=g).to(dtype).cuda()
    positions = list(range(5, 45))
    crooked = base[3:3 + 40 * 99].view(40, 99)[:, :2 * 33].view(40, 2, 33)[:, :, :32]          # no address is a multiple of 16 bytes
    heads_first = base[:5 * 40 * 48].view(5, 40, 48).transpose(0, 1)                            # [rows, heads, h]: heads are far apart
    _rotary_check(crooked, heads_first[..., :32], positions, f, style, a, False)
    out = torch.zeros(5, 40, 48, dtype=dtype, device="cuda").transpose(0, 1)
    _rotary_check(heads_first, None, positions, f, style, a, True, q_out=out)
    shared = base[:40 * 32].view(40, 1, 32).expand(40, 4, 32)                                   # one head read four times
    _rotary_check(shared, base[:32].view(1, 1, 32).expand(40, 2, 32), positions, f, style, a, False)
    with pytest.raises(B.SledError):
        B.rotary(heads_first, None, _i32(positions), f.cuda(), q_out=base[:40 * 48].view(40, 1, 48).expand(40, 5, 48))


def test_far_positions_and_numbers_that_are_none():
    f, _ = B.rotary_frequencies(64, 5e5)
    g = torch.Generator().manual_seed(9)
    x = torch.randn(6, 3, 64, generator=g).cuda()
    positions = [0, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6 + 1, 16777217]
    _rotary_check(x, None, positions, f, "pairs", 1.0, False)
    x[1, 2, 5] = math.nan
    x[1, 0, 40] = math.inf
    y = B.rotary(x, None, _i32(positions), f.cuda(), style="pairs")[0]
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 2, 4:6] = bad[1, 0, 40:42] = True
    assert bool((~y.isfinite() <= bad).all()) and bool(y[1, 2, 4:6].isnan().all())


@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_the_gradient_of_rotary(style):
    """The call is linear in its input: differences are exact but for rounding, and the gradient is the transposed product."""
    g = torch.Generator().manual_seed(11)
    f, a = B.rotary_frequencies(48, 1e4, scaling=B.ROTARY_RAMP, factor=4.0, length=512, low=1.0, high=8.0)
    x, y = (torch.randn(9, 4, 64, generator=g).cuda() for _ in range(2))
    p = _i32([0, 1, 2, 3, 77, 1000, 1001, 5000, 123456])
    call = lambda t, inverse=False: B.rotary(t, None, p, f.cuda(), style=style, amplitude=a, inverse=inverse)[0]
    # the loss sum(y * rotary(x)) has the gradient rotary^T(y); its difference along any d is sum(y * rotary(d))
    grad = call(y, True).double()
    # an error of at most 2^-20 of the sizes on either side (see step_ref.rotary), 64 products a head
    for k in range(5):
        d = torch.randn(9, 4, 64, generator=g).cuda()
        lhs, rhs = (y.double() * (call(x + d).double() - call(x).double())).sum((1, 2)), (grad * d.double()).sum((1, 2))
        size = a * 2 * (y.double().abs().amax() * (x.double().abs() + d.double().abs()).sum((1, 2)) * 2)
        assert bool(((lhs - rhs).abs() <= size * 2.0 ** -20).all())
    back = call(call(x), True).double() / a ** 2        # turned back, but for the amplitude; dimensions behind 48 are copied
    assert float((back - x.double())[..., :48].abs().max()) <= 4 * float(x.abs().max()) * 2.0 ** -20


def test_rotary_refuses_what_the_binding_sees():
    q, p, f = torch.zeros(2, 3, 8, device="cuda"), _i32([0, 1]), torch.zeros(4, dtype=torch.float64, device="cuda")
    for call in (lambda: B.rotary(q, q, _i32([0]), f), lambda: B.rotary(q, q, p, f.float()), lambda: B.rotary(q, q, p, f, style="other"),
                 lambda: B.rotary(q, q.to(BF), p, f), lambda: B.rotary(q[0], None, p, f), lambda: B.rotary(q, q[:1], p, f),
                 lambda: B.rotary(q.transpose(1, 2), None, p, f[:1]), lambda: B.rotary(q, q, p, f, q_out=q[:, :2]), lambda: B.rotary(q.half(), None, p, f),
                 lambda: B.rotary(q, q, p, torch.zeros(5, dtype=torch.float64, device="cuda")), lambda: B.rotary(q, q, p, f.cpu()),
                 lambda: B.rotary(q, q, p, f, amplitude=math.nan)):
        with pytest.raises(B.SledError) as e:
            call()
        assert e.value.code == B.SLED_ERR_ARG


# ------------------------------------------------------------------------------------------------------- append
def _paged(lens, hkv, h, page, seed, spare=3):
    """(codes, scales, table, pages) of a cache whose pages hold anything, codes that are no numbers among them."""
    g = torch.Generator().manual_seed(seed)
    pages = [S.up(n, page) for n in lens]
    n_pages, cols = sum(pages) + spare, max([1] + pages)
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table, at = torch.full((len(lens), cols), -7, dtype=torch.int32), 0
    for i, p in enumerate(pages):
        table[i, :p] = order[at:at + p]
        at += p
    codes = torch.randint(0, 256, (n_pages, hkv, page, h), generator=g, dtype=torch.uint8).view(E4M3)
    scales = torch.exp2(torch.randint(-9, -4, (n_pages, hkv, page // 16), generator=g).float())
    return codes, scales, table


def _append_check(first, new, hkv, h, page, dtype, *, rows=None, seed=0, scales=None, shape_rows=None):
    lens = [a + b for a, b in zip(first, new)]
    made = [_paged(lens, hkv, h, page, seed + i) for i in range(2)]
    table = made[0][2]
    g = torch.Generator().manual_seed(seed + 5)
    k, v = rows or [(torch.randn(sum(new), hkv, h, generator=g) * torch.exp(2 * torch.randn(sum(new), 1, 1, generator=g))).to(dtype) for _ in range(2)]
    if scales is not None:
        made = [(c, scales.clone().expand_as(s).contiguous(), t) for c, s, t in made]
    dev = [(c.cuda(), s.cuda()) for c, s, _ in made]
    status = _status()
    dk, dv = (shape_rows or (lambda t: t.cuda()))(k), (shape_rows or (lambda t: t.cuda()))(v)
    for _ in range(2):      # a second time nothing changes any more
        B.append_keys(dk, dv, dev[0][0], dev[1][0], table.cuda(), _i32(lens), _cu(new), k_scale=dev[0][1], v_scale=dev[1][1], status=status)
        B.check_status(status)
    for x, (c, s, _), (dc, ds) in zip((k, v), made, dev):
        was, c, s, at = c.view(torch.uint8), c.double(), s.double(), 0
        touched = torch.zeros(c.shape, dtype=torch.bool)
        for i, (a, m) in enumerate(zip(first, new)):
            if m:
                S.append(x[at:at + m], c, s, table[i], a + m, a, page)
                for y in range(a // 16 * 16, a + m):
                    touched[table[i, y // page], :, y % page] = True
            at += m
        got = dc.cpu()
        assert torch.equal(torch.where(touched, torch.zeros_like(was), got.view(torch.uint8)), torch.where(touched, torch.zeros_like(was), was))
        gd = got.double()
        assert torch.equal(gd.isnan() & touched, c.isnan() & touched)
        differ = touched & (gd != c) & ~c.isnan()
        assert not bool(differ.any()), (int(differ.sum()), gd[differ][:5], c[differ][:5])
        assert torch.equal(ds.cpu().double(), s)
    return dev


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h,page", [(128, 16), (64, 32), (32, 48), (128, 256), (32, 16)])
def test_append_in_8_bits(h, page, dtype):
    first = [0, 1, 15, 16, 17, 40, 0, 100, 47, 64, 5]
    new = [1, 1, 1, 1, 20, 0, 70, 9, 2, 16, 3]
    _append_check(first, new, 3, h, page, dtype, seed=h + page)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_prompts_in_8_bits(dtype):
    _append_check([0, 333, 0], [3000, 500, 1], 2, 128, 16, dtype)
    _append_check([3] * 40, [70] * 40, 1, 64, 16, dtype)


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_long_prompts_in_8_bits(dtype, h):
    _append_check([0, 333, 0, 7, 50], [3100, 500, 1, 2900, 700], 1, h, 16, dtype, seed=h)


@pytest.mark.parametrize("new", [[4100, 2000, 1, 900], [3, 5, 4, 6] * 60, [1] * 700])
def test_append_as_they_are_for_few_and_many_rows(new):
    g = torch.Generator().manual_seed(3)
    first = [17, 0, 5, 40] * (len(new) // 4)
    lens = [a + b for a, b in zip(first, new)]
    _, _, table = _paged(lens, 2, 64, 16, 4)
    cache = torch.randn(sum(S.up(n, 16) for n in lens) + 3, 2, 16, 64, generator=g).to(BF)
    rows = [torch.randn(sum(new), 2, 64, generator=g).to(BF) for _ in range(2)]
    dev = [cache.cuda(), cache.cuda()]
    B.append_keys(rows[0].cuda(), rows[1].cuda(), dev[0], dev[1], table.cuda(), _i32(lens), _cu(new))
    for x, d in zip(rows, dev):
        c, at = cache.clone(), 0
        for i, (a, m) in enumerate(zip(first, new)):
            slot = torch.arange(a, a + m)
            c[table[i, slot // 16].long(), :, slot % 16] = x[at:at + m]
            at += m
        assert torch.equal(d.cpu(), c)


def test_append_to_many_requests():
    rng = random.Random(3)
    first = [rng.randint(0, 40) for _ in range(1200)]
    _append_check(first, [rng.choice([0, 1, 1, 2, 5]) for _ in first], 1, 32, 16, BF)


def test_append_of_zeros_tiny_huge_and_numbers_that_are_none():
    rows = torch.zeros(6 * 16, 1, 32)
    rows[16:32] = 2.0 ** -133 * torch.arange(16 * 32).view(16, 1, 32)
    rows[32:48] = 3.0e38 * torch.linspace(-1, 1, 16 * 32).view(16, 1, 32)
    rows[48:64] = torch.randn(16, 1, 32, generator=torch.Generator().manual_seed(1))
    rows[50, 0, 3], rows[55, 0, 7], rows[60, 0, 1] = math.nan, math.inf, -math.inf
    rows[64:80] = math.nan
    rows[80:96] = 448 * 2.0 ** torch.arange(-15, 1).view(16, 1, 1) * torch.tensor([1.0, -1.0] * 16)      # a largest of exactly 448 times a power of two
    for dtype in (F32, BF):
        x = rows.to(dtype)
        _append_check([0], [96], 1, 32, 16, dtype, rows=(x, x))
        _append_check([10], [96], 1, 32, 16, dtype, rows=(x, x))


@pytest.mark.parametrize("scale", [0.3, 1e-20, 1.0, 2.0 ** -126, 7.7, 1e20])
def test_append_beside_scales_of_any_size(scale):
    # blocks whose scale is larger than their new rows need keep it, whatever number it is; quotients are of 32 bits then
    _append_check([5, 8, 0, 19], [3, 20, 7, 1], 2, 64, 16, BF, scales=torch.full((1, 1, 1), scale))
    _append_check([5, 8, 0, 19], [3, 20, 7, 1], 2, 64, 16, F32, scales=torch.full((1, 1, 1), scale))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_from_slices(dtype):
    def apart(t):
        wide = torch.full((t.shape[0], 2 * t.shape[1] * t.shape[2] + 1), math.nan, dtype=dtype, device="cuda")
        part = wide[:, 1:1 + t.shape[1] * t.shape[2]].view(t.shape) if t.shape[0] == 1 else wide[:, 1:1 + t.shape[1] * t.shape[2]].unflatten(1, t.shape[1:])
        part.copy_(t)
        return part
    _append_check([7, 0], [12, 300], 2, 128, 16, dtype, shape_rows=apart)
    aligned = lambda t: torch.cat([t, t], 1).cuda()[:, :t.shape[1]]
    _append_check([7, 0], [12, 300], 2, 128, 16, dtype, shape_rows=aligned)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h,page", [(128, 16), (64, 64), (32, 48)])
def test_append_as_they_are(h, page, dtype):
    first, new = [0, 1, 15, 40, 0, 100], [1, 1, 20, 0, 3000, 9]
    lens = [a + b for a, b in zip(first, new)]
    _, _, table = _paged(lens, 2, h, page, 1)
    g = torch.Generator().manual_seed(2)
    n_pages = sum(S.up(n, page) for n in lens) + 3
    caches = [torch.randn(n_pages, 2, page, h, generator=g).to(dtype) for _ in range(2)]
    rows = [torch.randn(sum(new), 2, h, generator=g).to(dtype) for _ in range(2)]
    rows[0][3] = math.nan
    dev = [c.cuda() for c in caches]
    B.append_keys(rows[0].cuda(), rows[1].cuda(), dev[0], dev[1], table.cuda(), _i32(lens), _cu(new))
    for c, x, d in zip(caches, rows, dev):
        at = 0
        for i, (a, m) in enumerate(zip(first, new)):
            for j in range(m):
                c[table[i, (a + j) // page], :, (a + j) % page] = x[at + j]
            at += m
        ints = torch.int16 if dtype is BF else torch.int32
        assert torch.equal(d.cpu().view(ints), c.view(ints))


def test_append_leaves_wrong_requests_out():
    k = torch.ones(5, 1, 32, dtype=BF, device="cuda")
    for n_kv, cu, table, wrote in (([3, 40], [0, 3, 5], [[0, 1], [2, 3]], [0]), ([3, 1], [0, 3, 5], [[0, 1], [2, 3]], [0]),
                                   ([3, 2], [0, 3, 9], [[0, 1], [2, 3]], [0]), ([3, 2], [0, 3, 5], [[0, 1], [4, 3]], [0]),
                                   ([3, 2], [0, 3, 5], [[-1, 1], [2, 3]], [2]), ([3, 2], [2, 1, 3], [[0, 1], [2, 3]], [])):
        codes, scales, status = torch.zeros(4, 1, 16, 32, device="cuda").to(E4M3), torch.full((4, 1, 1), 5.0, device="cuda"), _status()
        c2, s2 = codes.clone(), scales.clone()
        B.append_keys(k, k, codes, c2, _i32(table), _i32(n_kv), _i32(cu), k_scale=scales, v_scale=s2, status=status)
        assert status.item() == B.SLED_ERR_ARG
        for c, s in ((codes, scales), (c2, s2)):
            assert [p for p in range(4) if bool((c[p].float() != 0).any()) or s[p].item() != 5.0] == wrote, (n_kv, cu, table)


def test_append_refuses_what_the_binding_sees():
    k = torch.zeros(2, 2, 32, device="cuda")
    c, s, t, n, cu = torch.zeros(3, 2, 16, 32, device="cuda").to(E4M3), torch.ones(3, 2, 1, device="cuda"), _i32([[0]]), _i32([2]), _i32([0, 2])
    call = lambda k=k, v=k, c=c, w=c, cu=cu, ks=s, vs=s: B.append_keys(k, v, c, w, t, n, cu, k_scale=ks, v_scale=vs)
    call()
    for bad in (dict(k=k[:, :1]), dict(k=k[..., :16]), dict(k=k.half()), dict(v=k.to(BF)), dict(v=k[:1]), dict(ks=None), dict(vs=None), dict(ks=s[:2]),
                dict(ks=s.double()), dict(cu=_i32([0, 1, 2])), dict(c=c.float(), w=c.float()), dict(c=c.to(BF), w=c.to(BF), ks=None, vs=None),
                dict(w=c.float()), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=k.cpu()), dict(ks=s.cpu())):
        with pytest.raises(B.SledError) as e:
            call(**bad)
        assert e.value.code == B.SLED_ERR_ARG


# ---------------------------------------------------------------------------------------------------- attention
def _tree(rng, m, roots=False):
    return [-1] + [rng.choice([-1] * roots + list(range(max(0, j - 5), j))) for j in range(1, m)]


def _coded_cache(lens, hkv, h, page, seed, whole=False, spread=0.0):
    """Codes and scales of K and V with every request's pages scattered; slots without keys are no numbers, neither are the scales of
    blocks without any."""
    k, v, table, n_kv = R.make_cache(lens, hkv, h, F32, page, seed)
    out = []
    g = torch.Generator().manual_seed(seed + 9)
    for x in (k, v):
        if spread:
            x = x * torch.exp2((spread * torch.randn(x.shape[0], hkv, page // 16, 1, 1, generator=g)).round()).expand(-1, -1, -1, 16, 1).reshape(x.shape[0], hkv, page, 1)
        empty = x.isnan().view(x.shape[0], hkv, page // 16, -1).all(-1)
        c, s = S.coded(x, whole)
        s[empty] = math.nan
        out += [c, s]
    return (*out, table, n_kv)


def _scaled_check(lens, q_len, hq, hkv, h, *, parents=None, page=16, scale=None, seed=0, cache=None, q=None, chunk=None):
    kc, ks, vc, vs, table, n_kv = cache or _coded_cache(lens, hkv, h, page, seed)
    if q is None:
        q = torch.randn(sum(q_len), hq, h, generator=torch.Generator().manual_seed(seed + 1)).to(BF)
    status = _status()
    lse = torch.full((sum(q_len), hq), 7.0, device="cuda")
    flat = None if parents is None else _i32(sum(parents, []))
    kwargs = {} if scale is None else {"scale": scale}
    out = B.attention_tree(q.cuda() if chunk is None else chunk(q), kc.cuda(), vc.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len), flat, lse=lse, status=status,
                           k_scale=ks.cuda(), v_scale=vs.cuda(), **kwargs)
    B.check_status(status)
    out, lse = out.cpu().double(), lse.cpu().double()
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, page) for c, s in ((kc, ks), (vc, vs)))
        see = R.tree_mask(None if parents is None else parents[i], m, n)
        # bounds as for 16-bit caches: scores of 32-bit sums (two more products, by the block's scale and the query's), numerators rounded to 16 bits
        o, l, p, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, see, scale or h ** -0.5, BF)
        bad = (out[at:at + m] - o).abs() - d_o
        assert not bool((bad > 0).any() | bad.isnan().any()), (i, n, m, float(bad.max()))
        got_l = lse[at:at + m]
        assert torch.equal(torch.isinf(got_l), torch.isinf(l))
        fine = ~torch.isinf(l)
        assert bool(((got_l - l).abs()[fine] <= d_l[fine]).all()), (i, float((got_l - l).abs()[fine].max()))
        at += m
    return out, lse


GEOMETRIES = [(32, 8, 128), (32, 8, 64), (8, 2, 128), (6, 2, 32), (5, 5, 128), (16, 1, 64), (7, 1, 128), (40, 1, 128), (3, 3, 32)]


@pytest.mark.parametrize("hq,hkv,h", GEOMETRIES)
def test_scaled_trees(hq, hkv, h):
    rng = random.Random(hq * 1000 + h)
    lens = [1, 2, 17, 16, 15, 63, 64, 65, 130, 9, 700, 33, 1025]
    q_len = [1, 1, 3, 16, 4, 2, 1, 8, 30, 9, 7, 12, 5]
    _scaled_check(lens, q_len, hq, hkv, h, parents=[_tree(rng, m, roots=True) for m in q_len])


@pytest.mark.parametrize("hq,hkv,h", GEOMETRIES[:6])
def test_scaled_chains(hq, hkv, h):
    _scaled_check([5, 0, 300, 64, 2000, 129], [5, 0, 200, 1, 3, 64], hq, hkv, h)


@pytest.mark.parametrize("hq,hkv,h", GEOMETRIES[:7])
def test_scaled_single_tokens(hq, hkv, h):
    _scaled_check([1, 15, 16, 17, 64, 100, 1000, 5, 4097], [1] * 9, hq, hkv, h)


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("page", [32, 64, 128, 256, 48])
def test_scaled_other_page_sizes(page, h):
    rng = random.Random(page)
    q_len = [4, 1, 9]
    _scaled_check([page * 3 + 5, page, 777], q_len, 8, 2, h, parents=[_tree(rng, m) for m in q_len], page=page)


@pytest.mark.parametrize("h", [32, 64, 128])
def test_scaled_largest_trees(h):
    rng = random.Random(4)
    q_len = [128, 127, 65, 1]
    _scaled_check([128, 1000, 400, 90], q_len, 8, 2, h, parents=[_tree(rng, 128, True), [-1] + list(range(126)), [-1] * 65, [-1]])
    _scaled_check([5000] * 3, [64] * 3, 32, 8, h, parents=[_tree(rng, 64) for _ in range(3)])


def test_scaled_one_long_context_and_many_short_ones():
    rng = random.Random(5)
    _scaled_check([40011], [3], 8, 2, 128, parents=[[-1, 0, 0]])
    lens = [rng.randint(1, 90) for _ in range(300)]
    q_len = [rng.randint(1, min(n, 3)) for n in lens]
    _scaled_check(lens, q_len, 8, 2, 64, parents=[_tree(rng, m) for m in q_len])


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("wide", [1, 12])
def test_scaled_unused_nodes_and_those_that_hang_on_them(wide, h):
    parents = [[-1, -2, 1, 0, 3], [-2, -2, -2], [-1, 0, -2, 2, 3, 1, -1], [-2]]
    out, lse = _scaled_check([40, 3, 100, 1], [5, 3, 7, 1], 8 * wide, 2, h, parents=parents)
    empty = [1, 2, 5, 6, 7, 10, 11, 12, 15]
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())


@pytest.mark.parametrize("wide", [1, 12])
def test_scaled_keys_that_a_row_does_not_see_may_be_anything(wide):
    # node 1 of 3 holds no number as key and value: nodes 0 and 2 do not see it, its own row is no number
    lens, q_len, parents = [150, 70], [3, 1], [[-1, 0, 0], [-1]]
    hq = 8 * wide
    kc, ks, vc, vs, table, n_kv = _coded_cache(lens, 2, 64, 16, 3)
    for c in (kc, vc):
        c.view(torch.uint8)[table[0, 148 // 16], :, 148 % 16] = 0xff
    q = torch.randn(4, hq, 64, generator=torch.Generator().manual_seed(1)).to(BF)
    lse = torch.empty(4, hq, device="cuda")
    out = B.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len), _i32([-1, 0, 0, -1]), lse=lse, k_scale=ks.cuda(),
                           v_scale=vs.cuda()).cpu().double()
    clean = [c.double().nan_to_num(0).float().to(E4M3) for c in (kc, vc)]
    at = 0
    for i, m in enumerate(q_len):
        kk, vv = (R.keys_of(S.values(c, s), table[i], lens[i], 16) for c, s in zip(clean, (ks, vs)))
        o, l, _, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(parents[i], m, lens[i]), 0.125, BF)
        for j in range(m):
            if (i, j) == (0, 1):
                assert bool(out[at + j].isnan().all()) and bool(lse[at + j].isnan().all())
                continue
            assert bool(((out[at + j] - o[j]).abs() <= d_o[j]).all()) and bool(((lse[at + j].cpu().double() - l[j]).abs() <= d_l[j]).all())
        at += m


@pytest.mark.parametrize("wide", [1, 12])
def test_scaled_values_that_are_no_numbers_reach_the_rows_that_see_them(wide):
    lens, q_len = [150, 70, 40], [3, 1, 5]
    hq = 8 * wide
    kc, ks, vc, vs, table, n_kv = _coded_cache(lens, 2, 64, 16, 3)
    vc.view(torch.uint8)[table[0, 149 // 16], 0, 149 % 16, 7] = 0x7f      # seen by the last token of request 0 only, dimension 7 of head 0
    vc.view(torch.uint8)[table[1, 0], 1, 3, 9] = 0xff                     # seen by request 1
    q = torch.randn(9, hq, 64, generator=torch.Generator().manual_seed(1)).to(BF)
    out = B.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len), k_scale=ks.cuda(), v_scale=vs.cuda()).cpu()
    want = torch.zeros(9, hq, 64, dtype=torch.bool)
    want[2, :hq // 2, 7] = True
    want[3, hq // 2:, 9] = True
    assert torch.equal(out.isnan(), want)


@pytest.mark.parametrize("wide", [1, 12])
@pytest.mark.parametrize("spread", [3.0, 8.0])
def test_scaled_blocks_of_very_different_scales(spread, wide):
    lens, q_len = [1, 200, 1000, 3000], [1, 4, 9, 1]
    cache = list(_coded_cache(lens, 2, 128, 16, 11, whole=True, spread=spread))
    cache[1] = torch.where(cache[1].isnan(), cache[1], cache[1].clamp_max(0.02))      # scores stay where exponentials say something
    _scaled_check(lens, q_len, 8 * wide, 2, 128, cache=cache)
    cache[3] = cache[3] * 2.0 ** 90
    _scaled_check(lens, q_len, 8 * wide, 2, 128, cache=cache)


@pytest.mark.parametrize("wide", [1, 12])
def test_scaled_scales_of_zero_and_below(wide):
    lens, q_len = [200, 90], [4, 1]
    cache = list(_coded_cache(lens, 2, 64, 16, 12))
    cache[1][::2] *= -1
    cache[3][::3] *= 0
    cache[3][1::3] *= -1
    _scaled_check(lens, q_len, 8 * wide, 2, 64, cache=cache)
    cache[3] *= 0
    out, _ = _scaled_check(lens, q_len, 8 * wide, 2, 64, cache=cache)
    assert bool((out == 0).all())


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("hq", [2, 12, 40, 200])
def test_scaled_values_of_nothing_under_the_largest_scores(hq, h):
    """What is left of a result when its largest probabilities meet values of 0, in a block beside the others."""
    lens, q_len = [200, 90, 40], [4, 1, 7]
    cache = list(_coded_cache(lens, 2, h, 16, 12, whole=True, spread=2.0))
    cache[3] = torch.where(cache[1] > cache[1].nan_to_num(0).quantile(0.7), 0.0, cache[3])
    _scaled_check(lens, q_len, hq, 2, h, cache=cache)
    cache[3] = cache[3] * 2.0 ** -100
    _scaled_check(lens, q_len, hq, 2, h, cache=cache)


@pytest.mark.parametrize("wide", [1, 12])
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** -14, 1e-3, 300.0, 2.0 ** 60])
def test_scaled_queries_of_any_size(size, wide):
    lens, q_len = [200, 90], [4, 1]
    q = (torch.randn(5, 8 * wide, 128, generator=torch.Generator().manual_seed(3)) * size).to(BF)
    q[1] = 0
    _scaled_check(lens, q_len, 8 * wide, 2, 128, q=q, scale=min(0.1, 0.1 / size) if size < 2.0 ** 60 else 2.0 ** -64)


def test_scaled_queries_of_large_spread():
    lens, q_len = [200, 90], [4, 1]
    g = torch.Generator().manual_seed(4)
    q = (torch.randn(5, 8, 128, generator=g) * torch.exp2(torch.randint(-12, 8, (5, 8, 128), generator=g).float())).to(BF)
    _scaled_check(lens, q_len, 8, 2, 128, q=q, scale=1e-3)


@pytest.mark.parametrize("h", [64, 128])
def test_scaled_queries_and_outputs_in_slices(h):
    lens, q_len = [200, 90, 33], [40, 1, 9]
    for pad in (2, 6, 16):       # elements: what the kernels may ask of alignment differs
        chunk = lambda q: torch.cat([q.flatten(1), torch.zeros(q.shape[0], pad, dtype=BF)], 1).cuda()[:, :q.shape[1] * h].unflatten(1, (q.shape[1], h))
        _scaled_check(lens, q_len, 8, 2, h, chunk=chunk)
    kc, ks, vc, vs, table, n_kv = _coded_cache(lens, 2, h, 16, 0)
    q = torch.randn(50, 8, h, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    args = (kc.cuda(), vc.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len))
    wide = torch.full((52, 8 * h + 6), 3.0, dtype=BF, device="cuda")
    got = B.attention_tree(q, *args, k_scale=ks.cuda(), v_scale=vs.cuda(), out=wide[1:51, 2:2 + 8 * h].unflatten(1, (8, h)))
    want = B.attention_tree(q, *args, k_scale=ks.cuda(), v_scale=vs.cuda())
    assert (got.double() - want.double()).abs().max() <= 2.0 ** -7 * want.double().abs().max()
    got.fill_(3.0)
    assert bool((wide == 3.0).all())


def test_scaled_rows_of_nobody_are_left_alone_and_wrong_requests_left_out():
    lens, q_len = [100, 50, 60], [2, 3, 1]
    kc, ks, vc, vs, table, n_kv = _coded_cache(lens, 2, 64, 16, 0)
    q = torch.randn(9, 8, 64).to(BF).cuda()
    call = lambda n_kv, cu, table, st, out, lse: B.attention_tree(q, kc.cuda(), vc.cuda(), table.cuda(), n_kv, cu, k_scale=ks.cuda(), v_scale=vs.cuda(),
                                                                 out=out, lse=lse, status=st)
    def fresh():
        return torch.full((9, 8, 64), 5.0, dtype=BF, device="cuda"), torch.full((9, 8), 5.0, device="cuda")
    out, lse = fresh()
    st = _status()
    call(n_kv.cuda(), _i32([1, 3, 6, 7]), table, st, out, lse)
    B.check_status(st)
    assert bool((out[[0, 7, 8]] == 5).all()) and bool((lse[[0, 7, 8]] == 5).all()) and not bool((lse[1:7] == 5).any())
    for bad in (_i32([100, 2, 60]), _i32([100, 5000, 60])):
        o2, l2 = fresh()
        st = _status()
        call(bad, _i32([1, 3, 6, 7]), table, st, o2, l2)
        assert st.item() == B.SLED_ERR_ARG
        assert bool((l2[3:6] == 5).all()) and torch.equal(o2[1:3], out[1:3]) and torch.equal(o2[6], out[6])
    wrong = table.clone()
    wrong[1, 0] = 10 ** 6
    o2, l2 = fresh()
    st = _status()
    call(n_kv.cuda(), _i32([1, 3, 6, 7]), wrong, st, o2, l2)
    assert st.item() == B.SLED_ERR_ARG and torch.equal(o2[1:3], out[1:3]) and torch.equal(o2[6], out[6])
    st = _status()
    B.attention_tree(q[:130 % 9 + 2], kc.cuda(), vc.cuda(), table[:1].cuda(), _i32([100]), _i32([0, 3]), _i32([-1, 5, -1, -1, -1, -1]), k_scale=ks.cuda(),
                     v_scale=vs.cuda(), status=st)
    assert st.item() == B.SLED_ERR_ARG      # a parent that is no earlier node


# Units of up to 256 rows are for batches of many tiles; how many there may be is what the table has columns for.
def _many_columns(cache):
    kc, ks, vc, vs, table, n_kv = cache
    wide = torch.full((table.shape[0], 4096), -9, dtype=table.dtype)
    wide[:, :table.shape[1]] = table
    return kc, ks, vc, vs, wide, n_kv


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(64, 2), (40, 1), (48, 3)])
def test_scaled_units_of_256_rows(hq, hkv, h):
    rng = random.Random(h + hq)
    lens = [64, 1, 17, 300, 0, 1025, 129, 700]
    q_len = [13, 1, 17, 30, 0, 8, 9, 7]
    cache = _many_columns(_coded_cache(lens, hkv, h, 16, h))
    _scaled_check(lens, q_len, hq, hkv, h, cache=cache, parents=[_tree(rng, m, roots=True) if m else [] for m in q_len])
    _scaled_check(lens, q_len, hq, hkv, h, cache=cache)
    parents = [[-2] + [-1] * (m - 1) if m else [] for m in q_len]            # the first row of every request sees nothing
    out, lse = _scaled_check(lens, q_len, hq, hkv, h, cache=cache, parents=parents)
    at = [sum(q_len[:i]) for i, m in enumerate(q_len) if m]
    assert bool((out[at] == 0).all()) and bool((lse[at] == -math.inf).all())


@pytest.mark.parametrize("h", [64, 128])
def test_scaled_prompts_in_units_of_256_rows(h):
    lens, q_len = [500, 333, 70, 128], [300, 333, 1, 128]
    _scaled_check(lens, q_len, 8, 2, h, cache=_many_columns(_coded_cache(lens, 2, h, 16, h)))


@pytest.mark.parametrize("columns", [lambda c: c, _many_columns])
@pytest.mark.parametrize("h", [64, 128])
def test_scaled_codes_that_are_no_numbers_in_large_units(h, columns):
    """Keys and values of a node that others do not see, under units of 128 and of 256 rows; scales of zero, below and far apart."""
    lens, q_len, parents, hq = [150, 70], [20, 9], [[-1] + [0] * 19, [-1] + [0] * 8], 64
    cache = list(columns(_coded_cache(lens, 2, h, 16, 3, whole=True, spread=3.0)))
    cache[3][1::3] *= -1
    cache[3][::5] *= 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        for c in (cache[0], cache[2]):
            c.view(torch.uint8)[cache[4][i, (n - 2) // 16], :, (n - 2) % 16] = 0xff          # node m - 2
    kc, ks, vc, vs, table, n_kv = cache
    q = torch.randn(29, hq, h, generator=torch.Generator().manual_seed(1)).to(BF)
    lse = torch.empty(29, hq, device="cuda")
    out = B.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len), _i32(sum(parents, [])), lse=lse, k_scale=ks.cuda(),
                           v_scale=vs.cuda()).cpu().double()
    clean = [c.double().nan_to_num(0).float().to(E4M3) for c in (kc, vc)]
    at = 0
    for i, m in enumerate(q_len):
        kk, vv = (R.keys_of(S.values(c, s), table[i], lens[i], 16) for c, s in zip(clean, (ks, vs)))
        o, l, _, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(parents[i], m, lens[i]), h ** -0.5, BF)
        for j in range(m):
            if j == m - 2:
                assert bool(out[at + j].isnan().all()) and bool(lse[at + j].isnan().all())
                continue
            assert bool(((out[at + j] - o[j]).abs() <= d_o[j]).all()) and bool(((lse[at + j].cpu().double() - l[j]).abs() <= d_l[j]).all())
        at += m


@pytest.mark.parametrize("columns", [lambda c: c, _many_columns])
def test_scaled_rows_of_nobody_in_large_units(columns):
    lens, q_len, hq = [100, 50, 60], [12, 9, 10], 64
    kc, ks, vc, vs, table, n_kv = (x.cuda() for x in columns(_coded_cache(lens, 2, 128, 16, 0)))
    q = torch.randn(40, hq, 128, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    cu = _i32([2, 14, 23, 33])
    def call(table, n_kv):
        out, lse, st = torch.full((40, hq, 128), 5.0, dtype=BF, device="cuda"), torch.full((40, hq), 5.0, device="cuda"), _status()
        B.attention_tree(q, kc, vc, table, n_kv, cu, k_scale=ks, v_scale=vs, out=out, lse=lse, status=st)
        return out, lse, st.item()
    out, lse, st = call(table, n_kv)
    assert st == 0
    nobody = [0, 1] + list(range(33, 40))
    assert bool((out[nobody] == 5).all()) and bool((lse[nobody] == 5).all()) and not bool((lse[2:33] == 5).any())
    o, l, st = call(table, _i32([100, 8, 60]))            # fewer keys than rows
    assert st == B.SLED_ERR_ARG and bool((l[14:23] == 5).all())
    assert torch.equal(o[2:14], out[2:14]) and torch.equal(o[23:33], out[23:33])
    wrong = table.clone()
    wrong[1, 0] = kc.shape[0]
    o, l, st = call(wrong, n_kv)
    assert st == B.SLED_ERR_ARG and torch.equal(o[2:14], out[2:14]) and torch.equal(o[23:33], out[23:33])


@pytest.mark.parametrize("hq,hkv,h,rows,columns", [(32, 8, 128, 1, 0), (6, 2, 32, 2, 0), (8, 2, 64, 4, 0), (32, 8, 128, 7, 0), (16, 2, 32, 30, 0), (32, 8, 128, 30, 0),
                                                   (64, 2, 64, 12, 4096)])
def test_scaled_results_do_not_depend_on_where_pages_lie(hq, hkv, h, rows, columns):
    """Bit for bit, several times: pages in order and scattered arrive at different times."""
    rng = random.Random(h + rows)
    lens = [rng.randint(30000, 60000), 5, rng.randint(1, 9000), rng.randint(1, 9000), 64, rng.randint(30000, 60000)]
    q_len = [min(n, rng.randint(max(1, rows // 2), rows)) for n in lens]
    pages = [S.up(n, 16) for n in lens]
    n_pages = sum(pages)
    g = torch.Generator(device="cuda").manual_seed(rows)
    codes = [torch.randint(0, 126, (n_pages, hkv, 16, h), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2)]
    scales = [torch.rand(n_pages, hkv, 1, device="cuda", generator=g) * x for x in (2e-4, 1.0)]
    q = torch.randn(sum(q_len), hq, h, device="cuda", generator=g).to(BF)
    want = None
    for order in [torch.arange(n_pages, device="cuda")] + [torch.randperm(n_pages, device="cuda", generator=g) for _ in range(3)]:
        table, at = torch.zeros(len(lens), columns or max(pages), dtype=torch.int32, device="cuda"), 0
        for i, p in enumerate(pages):
            table[i, :p] = order[at:at + p]
            at += p
        to = torch.empty_like(order)
        to[order] = torch.arange(n_pages, device="cuda")
        c, s, status = [x[to].view(E4M3) for x in codes], [x[to] for x in scales], _status()
        for _ in range(3):
            out = B.attention_tree(q, *c, table, _i32(lens), _cu(q_len), k_scale=s[0], v_scale=s[1], status=status)
            want = out if want is None else want
            assert torch.equal(out, want)
        B.check_status(status)


@pytest.mark.parametrize("hq,hkv,h", [(8, 2, 128), (6, 2, 32), (32, 8, 64), (64, 2, 128)])
@pytest.mark.parametrize("batch,length,rows", [(1, 4100, 3), (1, 9000, 1), (12, 512, 4), (40, 300, 1), (100, 64, 2), (90, 65, 9), (3, 1000, 7), (20, 700, 1)])
def test_scaled_units_that_are_alike(batch, length, rows, hq, hkv, h):
    _scaled_check([length] * batch, [rows] * batch, hq, hkv, h, seed=batch + rows)


@pytest.mark.parametrize("columns", [lambda c: c, _many_columns])
def test_scaled_wide_units_that_are_alike(columns):
    for batch, length, rows in ((1, 2500, 40), (9, 300, 9), (30, 130, 20)):
        _scaled_check([length] * batch, [rows] * batch, 32, 2, 128, cache=columns(_coded_cache([length] * batch, 2, 128, 16, rows)))


def test_scaled_empty_batches():
    q = torch.zeros(0, 8, 64, dtype=BF, device="cuda")
    c, s = torch.zeros(3, 2, 16, 64, device="cuda").to(E4M3), torch.ones(3, 2, 1, device="cuda")
    assert B.attention_tree(q, c, c, _i32([[0]]), _i32([5]), _i32([0, 0]), k_scale=s, v_scale=s).shape == q.shape
    assert B.attention_tree(q, c, c, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), _i32([]), _i32([0]), k_scale=s, v_scale=s).shape == q.shape


def test_scaled_refuses_what_the_binding_sees():
    q = torch.zeros(2, 4, 32, dtype=BF, device="cuda")
    c, s, t, n, cu = torch.zeros(3, 2, 16, 32, device="cuda").to(E4M3), torch.ones(3, 2, 1, device="cuda"), _i32([[0]]), _i32([2]), _i32([0, 2])
    call = lambda q=q, c=c, ks=s, vs=s, **kw: B.attention_tree(q, c, c, t, n, cu, k_scale=ks, v_scale=vs, **kw)
    call()
    for bad in (dict(q=q.float()), dict(ks=None), dict(vs=None), dict(ks=s[:2]), dict(vs=s.double()), dict(c=c.to(BF)), dict(c=c.float()),
                dict(key_weights=torch.zeros(3, 2, 16, device="cuda")), dict(out=q), dict(lse=torch.zeros(2, 3, device="cuda")),
                dict(out=torch.zeros(2, 4, 32, device="cuda"))):
        with pytest.raises(B.SledError) as e:
            call(**bad)
        assert e.value.code == B.SLED_ERR_ARG


def test_scaled_captured_and_side_by_side():
    rng = random.Random(21)
    calls = []
    for seed, (q_len, hq) in enumerate((([3, 1, 9], 8), ([70, 60, 50], 32), ([1, 1, 1], 40))):
        lens = [300, 77, 1500]
        kc, ks, vc, vs, table, n_kv = (x.cuda() for x in _coded_cache(lens, 2, 128, 16, seed))
        q = torch.randn(sum(q_len), hq, 128, generator=torch.Generator().manual_seed(seed)).to(BF).cuda()
        par = _i32(sum((_tree(rng, m) for m in q_len), []))
        calls.append(lambda q=q, kc=kc, vc=vc, table=table, n_kv=n_kv, cu=_cu(q_len), par=par, ks=ks, vs=vs: B.attention_tree(
            q, kc, vc, table, n_kv, cu, par, k_scale=ks, v_scale=vs))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = c()
        graphs.append((g, o))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for st, (g, _), c in zip(streams, graphs, calls):
            with torch.cuda.stream(st):
                g.replay()
                mine = c()
                mine.record_stream(st)
    torch.cuda.synchronize()
    for w, (_, o) in zip(want, graphs):
        assert torch.equal(w, o)
    for st, c, w in zip(streams, calls, want):
        with torch.cuda.stream(st):
            assert torch.equal(c(), w)


@pytest.mark.parametrize("dtype", [E4M3, BF])
def test_caches_of_more_than_four_gigabytes(dtype):
    """Keys written to, and read from, the last pages of a cache whose offsets pass 32 bits, against the same ones in a small cache."""
    hkv, h, page, lens = 8, 128, 16, [50, 3]
    n_pages = (2 ** 32 + 2 ** 26) // (hkv * page * h)                    # elements
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(sum(lens), hkv, h, generator=g).to(BF).cuda() for _ in range(2))
    q = torch.randn(40 + 3, 32, h, generator=g).to(BF).cuda()
    outs = []
    for n, first in ((8, 0), (n_pages, n_pages - 8)):
        kc, vc = (torch.empty(n, hkv, page, h, dtype=dtype, device="cuda") for _ in range(2))
        scales = dict(k_scale=torch.ones(n, hkv, 1, device="cuda"), v_scale=torch.ones(n, hkv, 1, device="cuda")) if dtype == E4M3 else {}
        table = first + _i32([[7, 0, 3, 1], [5, -1, -1, -1]])
        B.append_keys(k, v, kc, vc, table, _i32(lens), _cu(lens), **scales)
        one = [] if dtype is BF else [B.attention_tree(q[:2], kc, vc, table, _i32(lens), _cu([1, 1]), **scales), B.attention_tree(q, kc, vc, table, _i32(lens), _cu([40, 3]), **scales)]
        outs.append(one + [x[table[0].long()].view(torch.uint8) for x in (kc, vc)] + [s[table[0].long()] for s in scales.values()])
        del kc, vc
    filled = [slice(0, 3), (slice(3, 4), slice(None), slice(0, 2))]      # slots without keys hold anything
    for a, b in zip(*outs):
        if a.dtype == torch.uint8:
            assert all(torch.equal(a[f], b[f]) for f in filled)
        else:
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------- the whole step
@pytest.mark.parametrize("bits", [8, 16])
def test_steps_in_a_row(bits):
    """A server's steps over a cache of its own: places, positions, keys, attention - prompts first, then drafts of which some are
    rejected -, with lengths that stay on the GPU; checked against attention over all the tokens so far in 64 bits."""
    rng = random.Random(bits)
    g = torch.Generator().manual_seed(bits)
    batch, hq, hkv, h, page, n_pages, cols = 5, 8, 2, 64, 16, 64, 20
    f, a = B.rotary_frequencies(h, 1e4, scaling=B.ROTARY_BANDS, factor=4.0, length=64, low=1.0, high=4.0)
    ctype = E4M3 if bits == 8 else BF
    kc, vc = (torch.full((n_pages, hkv, page, h), math.nan).to(ctype).cuda() for _ in range(2))
    scales = dict(k_scale=torch.full((n_pages, hkv, 1), math.nan, device="cuda"), v_scale=torch.full((n_pages, hkv, 1), math.nan, device="cuda")) if bits == 8 else {}
    table = torch.full((batch, cols), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda(), _i32([n_pages])
    n_kv, status = _i32([0] * batch), _status()
    past = [[[], []] for _ in range(batch)]        # what every request keeps: turned keys, values (rows of fp64)
    lens = [0] * batch
    for step in range(6):
        keep = [n if step < 2 else n - rng.randint(0, 3) for n in lens]
        new = [rng.randint(20, 60) if step == 0 else rng.randint(0, 6) for _ in range(batch)]
        rows = sum(new)
        p = B.page_slots(n_kv, _i32(new), table, free, n_free, page_size=page, n_rows=rows, n_keep=_i32(keep), status=status)
        x = torch.randn(rows, hq + 2 * hkv, h, generator=g).to(BF).cuda()
        q, k = B.rotary(x[:, :hq], x[:, hq:hq + hkv], p.positions, f.cuda(), style="halves", amplitude=a)
        B.append_keys(k, x[:, hq + hkv:], kc, vc, table, p.n_kv, p.cu_q, status=status, **scales)
        out = B.attention_tree(q, kc, vc, table, p.n_kv, p.cu_q, status=status, **scales)
        n_kv, n_free = p.n_kv, p.n_free
        B.check_status(status)
        positions = sum((list(range(c, c + m)) for c, m in zip(keep, new)), [])
        assert p.positions.tolist() == positions
        q64, _ = S.rotary(x[:, :hq].cpu(), positions, f.numpy(), True, a, False)
        k64, _ = S.rotary(x[:, hq:hq + hkv].cpu(), positions, f.numpy(), True, a, False)
        v64, at = x[:, hq + hkv:].cpu().double(), 0
        for i, (c, m) in enumerate(zip(keep, new)):
            past[i] = [past[i][0][:c] + list(k64[at:at + m]), past[i][1][:c] + list(v64[at:at + m])]
            lens[i] = c + m
            if m:
                kk, vv = (torch.stack(y).transpose(0, 1) for y in past[i])
                o = R.attend(q64[at:at + m], kk, vv, R.tree_mask(None, m, c + m), h ** -0.5, BF)[0]
                # 16 bits: queries, keys and values are off by 2^-8 of their size; 8 bits: keys and values by 2^-4 of theirs at most, and
                # in the root mean square by 2^-4 / sqrt(12) * 2 or less; a score of 64 such products, an average of such values
                rel = float((out[at:at + m].cpu().double() - o).norm() / o.norm())
                assert rel <= (0.15 if bits == 8 else 0.02), (step, i, rel)
            at += m
        # the slot map says where the keys went
        k_at = kc.float().transpose(1, 2).reshape(-1, hkv, h)[p.slots]
        if bits == 8:
            k_at = k_at * scales["k_scale"][..., 0].repeat_interleave(page, 0).view(n_pages * page, hkv)[p.slots][..., None]
            assert bool(((k_at - k.float()).abs() <= k.float().abs() * 2.0 ** -4 + k.float().abs().max() * 2.0 ** -9).all())
        else:
            assert torch.equal(k_at.to(BF), k)
    assert n_free.item() == n_pages - sum(S.up(n, page) for n in lens)


def test_a_captured_step_follows_the_lengths():
    batch, hq, hkv, h = 3, 8, 2, 128
    g = torch.Generator().manual_seed(2)
    kc, vc = (torch.zeros(40, hkv, 16, h).to(E4M3).cuda() for _ in range(2))
    ks, vs = (torch.ones(40, hkv, 1, device="cuda") for _ in range(2))
    table, free, n_free, n_kv = torch.full((batch, 12), -1, dtype=torch.int32, device="cuda"), _i32(list(range(40))), _i32([40]), _i32([0] * batch)
    x = torch.randn(batch, hq + 2 * hkv, h, generator=g).to(BF).cuda()
    f, a = B.rotary_frequencies(h, 1e4)
    f = f.cuda()
    new = _i32([1] * batch)
    def step():
        p = B.page_slots(n_kv, new, table, free, n_free, page_size=16, n_rows=batch)
        q, k = B.rotary(x[:, :hq], x[:, hq:hq + hkv], p.positions, f)
        B.append_keys(k, x[:, hq + hkv:], kc, vc, table, p.n_kv, p.cu_q, k_scale=ks, v_scale=vs)
        out = B.attention_tree(q, kc, vc, table, p.n_kv, p.cu_q, k_scale=ks, v_scale=vs)
        n_kv.copy_(p.n_kv)
        n_free.copy_(p.n_free)
        return out
    outs = []
    for _ in range(20):
        outs.append(step().clone())
    state = [t.clone() for t in (kc.view(torch.uint8), vc.view(torch.uint8), ks, vs, table, n_kv, n_free)]
    for t, v in ((table, -1), (n_kv, 0), (n_free, 40), (ks, 1), (vs, 1), (kc.view(torch.uint8), 0), (vc.view(torch.uint8), 0)):
        t.fill_(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for want in outs:
        graph.replay()
        assert torch.equal(out, want)
    for t, w in zip((kc.view(torch.uint8), vc.view(torch.uint8), ks, vs, table, n_kv, n_free), state):
        assert torch.equal(t, w)
