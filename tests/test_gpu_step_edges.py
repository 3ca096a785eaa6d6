"""Edges of a decoding step's operators over a caller's paged cache: places in pages of any size, keys beside
scales below 0, units of one tile in a row, value scales of any size, what is lost to the rounding of queries
and numerators, calls that wait."""
import math
import random
import threading
import time

import paged_ref as R
import pytest
import step_ref as S
import test_gpu_step as T
import torch

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------------- places
@pytest.mark.parametrize("page,cols", [(1 << 30, 1), (1_500_000_000, 1), (2 ** 31 - 1025, 1), (715_827_000, 3), (3000, 715_827), (1, 2_000_000)])
def test_places_in_pages_of_any_size(page, cols):
    """A request's keys and a page's slots together need more than 32 bits."""
    full = page * cols
    rng = random.Random(page)
    T._slots_case(rng, [full - 7, 0, 5], [full - 9, 0, 5], [9, 4, 0], page, cols=cols)
    T._slots_case(rng, [full, 0, full - page // 2], [0, 0, full - page // 2], [3, 12, page // 2 if page < 10 else 7], page, cols=cols, extra_rows=2)
    T._slots_case(rng, [0, full - 1], [0, full - 1], [2, 1], page, cols=cols, spare=0)
    T._slots_case(rng, [0, full - 1], [0, full - 1], [2, 1], page, cols=cols, spare=0, short=1)


# ---------------------------------------------------------------------------------------------------------- keys
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [-4.0, -0.3, -2.0 ** -9, -1e20])
def test_append_beside_scales_below_0(scale, dtype):
    """Attention reads scales below 0; older keys of such a block stay what they were."""
    page, h, first, new = 32, 64, [5, 20, 0], [3, 30, 9]
    lens = [a + b for a, b in zip(first, new)]
    kept = [T._paged(lens, 2, h, page, 7 + i) for i in range(2)]
    table = kept[0][2]
    g = torch.Generator().manual_seed(3)
    rows = [torch.randn(sum(new), 2, h, generator=g).to(dtype) for _ in range(2)]
    before = [(c.clone(), torch.full_like(s, scale)) for c, s, _ in kept]
    after = [(c.cuda(), s.cuda()) for c, s in before]
    status = T._status()
    B.append_keys(*(x.cuda() for x in rows), after[0][0], after[1][0], table.cuda(), T._i32(lens), T._cu(new), k_scale=after[0][1], v_scale=after[1][1],
                  status=status)
    B.check_status(status)
    for x, was, now in zip(rows, before, after):
        at = 0
        for i, (a, m) in enumerate(zip(first, new)):
            old, got, size = (R.keys_of(y, table[i], a + m, page) for y in (S.values(*was), S.values(now[0].cpu(), now[1].cpu()),
                                                                         now[1].cpu().double().abs().repeat_interleave(16, -1)))
            want = torch.cat([old[:, :a], x[at:at + m].double().transpose(0, 1)], 1)
            assert torch.equal(got[:, :a].isnan(), want[:, :a].isnan())
            # half a step of a code, or of the smallest code; quotients are of 32 bits
            off = (got - want).abs() - want.abs() * (2.0 ** -4 + 2.0 ** -20) - 2.0 ** -10 * size[..., None]
            assert bool((off.nan_to_num(0) <= 0).all())
            untouched = a // 16 * 16
            assert torch.equal(got[:, :untouched].nan_to_num(7), old[:, :untouched].nan_to_num(7))
            at += m


# ------------------------------------------------------------------------------- attention over a cache in 8 bits
@pytest.mark.parametrize("columns", [lambda c: c, T._many_columns])
@pytest.mark.parametrize("longest", [64, 200])
def test_many_units_of_one_tile(longest, columns):
    """Units of up to 128 rows with one tile each, one behind the other on every SM, alone and among others of two to four: the
    second group of rows of a block has no tile in them."""
    rng = random.Random(longest)
    lens = [rng.randint(5, longest) for _ in range(500)]
    q_len = [5] * len(lens)
    cache = columns(T._coded_cache(lens, 2, 64, 16, longest))
    out, lse = T._scaled_check(lens, q_len, 16, 2, 64, cache=cache, parents=[T._tree(rng, 5) for _ in lens])
    kc, ks, vc, vs, table, n_kv = (x.cuda() for x in cache)
    q = torch.randn(sum(q_len), 16, 64, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    status = T._status()
    first = B.attention_tree(q, kc, vc, table, n_kv, T._cu(q_len), k_scale=ks, v_scale=vs, status=status)
    for _ in range(100):
        again = B.attention_tree(q, kc, vc, table, n_kv, T._cu(q_len), k_scale=ks, v_scale=vs, status=status)
        assert torch.equal(first, again)
    B.check_status(status)


def test_stretches_that_take_longer_than_a_wait():
    """Four contexts of twelve million keys, the same 256 each time, to every SM: a quarter of a second each."""
    hq, h, n, batch = 40, 64, 48 * 1024 * 256, 4 * torch.cuda.get_device_properties(0).multi_processor_count
    kc, ks, vc, vs, where, _ = T._coded_cache([256], 1, h, 256, 2)
    q = torch.randn(1, hq, h, generator=torch.Generator().manual_seed(7)).to(BF)
    page_of = int(where[0, 0])
    kk, vv = (R.keys_of(S.values(c, s), where[0], 256, 256) for c, s in ((kc, ks), (vc, vs)))
    o, l, p, d_o, d_l, _ = R.attend(q, kk, vv, R.tree_mask(None, 1, 256), h ** -0.5, BF)
    # sums and outputs of a row: 16 keys at a time are added to what there is, an addition off by 2^-24
    rel = n // 16 * 2.0 ** -24
    spread = torch.einsum("mrn,rnd->mrd", p, vv.abs().repeat_interleave(hq, 0))
    table = torch.full((batch, n // 256), page_of, dtype=torch.int32, device="cuda")
    status, lse = T._status(), torch.zeros(batch, hq, device="cuda")
    out = B.attention_tree(q.cuda().expand(batch, -1, -1).contiguous(), kc.cuda(), vc.cuda(), table, T._i32([n] * batch), T._cu([1] * batch), lse=lse,
                           k_scale=ks.cuda(), v_scale=vs.cuda(), status=status)
    B.check_status(status)
    assert bool(((out.cpu().double() - o).abs() <= d_o + 2 * rel * spread).all())
    assert bool(((lse.cpu().double() - (l + math.log(n // 256))).abs() <= d_l + rel).all())


def _run(cache, q_len, q, parents=None, scale=0.0):
    kc, ks, vc, vs, table, n_kv = (x.cuda() for x in cache)
    status = T._status()
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = B.attention_tree(q.cuda(), kc, vc, table, n_kv, T._cu(q_len), parents, scale=scale, lse=lse, k_scale=ks, v_scale=vs, status=status)
    B.check_status(status)
    return out.cpu().double(), lse.cpu().double()


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("hq", [2, 12, 40, 200])
@pytest.mark.parametrize("power", [-126, -120, -112, -100, -60, 60, 110])
def test_value_scales_of_any_size(power, hq, h):
    """All value scales the same power of two; results are compared times its inverse, so that the bound's absolute part says nothing."""
    lens, q_len = [200, 90, 40], [4, 1, 7]
    kc, ks, vc, vs, table, n_kv = T._coded_cache(lens, 2, h, 16, 12, whole=True)
    if power > 100:                  # sums of exponentials times values stay in fp32
        vc = (vc.double().nan_to_num(0) / 448).to(E4M3)
    one = torch.where(vs.isnan(), vs, 1.0)
    q = torch.randn(sum(q_len), hq, h, generator=torch.Generator().manual_seed(5)).to(BF)
    out, lse = _run((kc, ks, vc, one * 2.0 ** power, table, n_kv), q_len, q)
    out = out * 2.0 ** -power
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, 16) for c, s in ((kc, ks), (vc, one)))
        o, l, _, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(None, m, n), h ** -0.5, BF)
        d_o += 2.0 ** (-134 - power)             # half a step of the smallest results, 2^-133
        assert bool(((out[at:at + m] - o).abs() <= d_o).all()), (i, float(((out[at:at + m] - o).abs() / d_o).max()))
        assert bool(((lse[at:at + m] - l).abs() <= d_l).all())
        at += m


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("hq", [2, 12, 40, 200])
@pytest.mark.parametrize("sharp", [0.0, 1.0, 8.0, 30.0])
def test_value_scales_far_apart(sharp, hq, h):
    """Value scales 2^-126 .. 2^100 and zeros, block by block, under scores from flat to far apart."""
    lens, q_len = [200, 90, 700], [4, 1, 3]
    kc, ks, vc, vs, table, n_kv = T._coded_cache(lens, 2, h, 16, 51, whole=True)
    g = torch.Generator().manual_seed(52)
    vs = torch.where(vs.isnan(), vs, torch.exp2(torch.randint(-126, 101, vs.shape, generator=g).float()))
    vs = torch.where(torch.rand(vs.shape, generator=g) < 0.2, vs * 0, vs)
    q = (torch.randn(sum(q_len), hq, h, generator=g) * sharp).to(BF)
    out, lse = _run((kc, ks, vc, vs, table, n_kv), q_len, q)
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, 16) for c, s in ((kc, ks), (vc, vs)))
        o, l, p, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(None, m, n), h ** -0.5, BF)
        wide = lambda x: x.abs().repeat_interleave(hq // 2, 0)
        numerators = p * wide(R.keys_of(vs.double().repeat_interleave(16, -1), table[i], n, 16))
        codes = wide(R.keys_of(vc.double(), table[i], n, 16))
        # numerators are off by 2^-11 of each (in the bound with 2^-8), or by 2^-32 of the row's largest; a weight below 2^-111 of the
        # largest may count as less
        d_o += torch.einsum("mrn,rnd->mrd", (2.0 ** -32 * numerators.amax(-1, keepdim=True)).expand_as(p), codes)
        d_o += torch.einsum("mrn,rnd->mrd", torch.where(p < 2.0 ** -111 * p.amax(-1, keepdim=True), p, 0), wide(vv))
        assert bool(((out[at:at + m] - o).abs() <= d_o).all()), (i, float(((out[at:at + m] - o).abs() / d_o).max()))
        assert bool(((lse[at:at + m] - l).abs() <= d_l).all())
        at += m


@pytest.mark.parametrize("hq", [2, 12, 40, 200])
@pytest.mark.parametrize("gap", [60, 100, 118, 124, 131, 160, 400])
def test_values_of_nothing_under_scores_far_above_the_others(gap, hq):
    """The first block's keys have the largest scores by 2^gap, values of 0 and the smallest scale, the others' values are large: what
    the others weigh, down to 2^-111 of the largest, is exact; below, they count as no more than they are."""
    lens, q_len, h = [90, 40], [4, 1], 64
    kc, ks, vc, vs, table, n_kv = T._coded_cache(lens, 2, h, 16, 3, whole=True)
    kc, vc, vs = torch.full(kc.shape, -1.0).to(E4M3), vc.clone(), torch.full(vs.shape, 2.0 ** 30)
    ks = torch.ones(ks.shape)
    for i in range(len(lens)):
        kc[table[i, 0]] = torch.ones(()).to(E4M3)
        vc.view(torch.uint8)[table[i, 0]] = 0
        vs[table[i, 0]] = 2.0 ** -126
    scale = gap * math.log(2) / (2 * h)          # scores +- gap ln(2) / 2
    q = torch.ones(sum(q_len), hq, h).to(BF)
    out, lse = _run((kc, ks, vc, vs, table, n_kv), q_len, q, scale=scale)
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, 16) for c, s in ((kc, ks), (vc, vs)))
        see = R.tree_mask(None, m, n)
        o, l, p, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, see, scale, BF)
        weight = torch.where(p < 2.0 ** -111 * p.amax(-1, keepdim=True), p, 0)
        d_o += torch.einsum("mrn,rnd->mrd", weight, vv.abs().repeat_interleave(hq // 2, 0))
        assert bool(((out[at:at + m] - o).abs() <= d_o).all()), (i, float(((out[at:at + m] - o).abs() / d_o).max()))
        assert bool(((lse[at:at + m] - l).abs() <= d_l).all())
        at += m


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("hq", [4, 24, 80])
def test_numerators_are_rounded_by_no_more_than_said(hq, h):
    """Keys in pairs of nearly the same score and opposite values: what is left is small beside what was added up, so that it shows the
    numerators' rounding, 2^-11 of each, and not the results' own.  (Rounded to bf16 they would be off by up to 2^-8.)"""
    lens, q_len = [16, 8, 32, 24], [1] * 4
    kc, ks, vc, vs, table, n_kv = T._coded_cache(lens, 2, h, 16, 31, whole=True)
    k8, v8 = kc.view(torch.uint8).clone(), vc.view(torch.uint8).clone()
    k8[:, :, 1::2], v8[:, :, 1::2] = k8[:, :, ::2], v8[:, :, ::2] ^ 0x80
    k8[:, :, 1::2, 0] = torch.where(k8[:, :, ::2, 0] & 0x7f == 0, k8[:, :, ::2, 0], k8[:, :, ::2, 0] - 1)       # a code nearer to 0
    kc, vc = k8.view(E4M3), v8.view(E4M3)
    q = torch.randn(sum(q_len), hq, h, generator=torch.Generator().manual_seed(5)).to(BF)
    out, _ = _run((kc, ks, vc, vs, table, n_kv), q_len, q)
    for i, n in enumerate(lens):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, 16) for c, s in ((kc, ks), (vc, vs)))
        o, _, p, d_o, _, _ = R.attend(q[i:i + 1], kk, vv, R.tree_mask(None, 1, n), h ** -0.5, BF)
        spread = torch.einsum("mrn,rnd->mrd", p, vv.abs().repeat_interleave(hq // 2, 0))
        d_o += (2.0 ** -11 - 2.0 ** -8) * spread          # numerators in fp16, or 2^-32 of the largest, which is less here
        assert bool(((out[i] - o[0]).abs() <= d_o[0]).all()), (i, float(((out[i] - o[0]).abs() / d_o[0]).max()))


@pytest.mark.parametrize("h", [32, 64, 128])
@pytest.mark.parametrize("hq", [4, 24, 80])
@pytest.mark.parametrize("ratio", [20, 30, 34, 37, 45])
def test_queries_with_one_element_far_above_the_others(ratio, hq, h):
    """The largest element meets codes of 0, so that scores are what the others make of them: those are off by 2^-39 of the largest at most
    where they are below 2^-31 of it, and exact elsewhere."""
    lens, q_len = [100, 40, 200], [1, 3, 2]
    kc, ks, vc, vs, table, n_kv = T._coded_cache(lens, 2, h, 16, 41, whole=True)
    kc = kc.view(torch.uint8).clone()
    kc[..., 3] = 0
    kc = kc.view(E4M3)
    q = torch.randn(sum(q_len), hq, h, generator=torch.Generator().manual_seed(6)).to(BF)
    q[..., 3] = 2.0 ** ratio
    out, lse = _run((kc, ks, vc, vs, table, n_kv), q_len, q)
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(S.values(c, s), table[i], n, 16) for c, s in ((kc, ks), (vc, vs)))
        o, l, p, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(None, m, n), h ** -0.5, BF)
        mine = q[at:at + m].double()
        off = torch.where(mine.abs() < 2.0 ** (ratio - 31), 2.0 ** (ratio - 39), 0).clamp_max(mine.abs())      # of an element; no more than itself
        d_s = torch.einsum("mgrd,gnd->mgrn", off.view(m, 2, hq // 2, h), kk.abs()).amax(-1).reshape(m, hq) * h ** -0.5
        spread = torch.einsum("mrn,rnd->mrd", p, vv.abs().repeat_interleave(hq // 2, 0))
        assert bool(((lse[at:at + m] - l).abs() <= d_l + d_s).all())
        assert bool(((out[at:at + m] - o).abs() <= d_o + torch.expm1(2 * d_s)[..., None] * spread).all())
        at += m


# ---------------------------------------------------------------------------------------------------------- calls
@pytest.mark.parametrize("name", ["page_slots", "rotary", "append_keys", "attention"])
def test_other_threads_run_while_a_launch_waits(name):
    """A stream's queue that is full makes a launch wait; the interpreter's other threads go on meanwhile."""
    i, table = T._i32([1]), T._i32([[0, 1]])
    cache, scale = torch.zeros(3, 2, 16, 64, device="cuda").to(E4M3), torch.ones(3, 2, 1, device="cuda")
    rows, free = torch.zeros(1, 2, 64, dtype=BF, device="cuda"), T._i32([2])
    values, value_scale, out = cache.clone(), scale.clone(), torch.empty_like(rows)
    slots = B.page_slots(i, i, table, free, T._i32([1]), page_size=16, n_rows=1)
    frequencies, n_free = B.rotary_frequencies(64)[0].cuda(), T._i32([1])
    cu = T._cu([1])
    call = {"page_slots": lambda: B.page_slots(i, i, table, free, n_free, page_size=16, n_rows=1, out=slots),
            "rotary": lambda: B.rotary(rows, None, i, frequencies, q_out=out),
            "append_keys": lambda: B.append_keys(rows, rows, cache, values, table, i, cu, k_scale=scale, v_scale=value_scale),
            "attention": lambda: B.attention_tree(rows, cache, values, table, i, cu, k_scale=scale, v_scale=value_scale, out=out)}[name]
    call()
    torch.cuda.synchronize()
    ticks, done = [], threading.Event()

    def tick():
        while not done.is_set():
            ticks.append(time.perf_counter())
            time.sleep(0.001)

    other = threading.Thread(target=tick)
    other.start()
    begin = time.perf_counter()
    torch.cuda._sleep(int(1.2e9))            # cycles: 0.6 s and more
    for _ in range(4000):
        call()
    end = time.perf_counter()
    done.set()
    other.join()
    torch.cuda.synchronize()
    assert end - begin > 0.4                 # the queue was full
    seen = [begin] + [t for t in ticks if begin <= t <= end] + [end]
    assert max(b - a for a, b in zip(seen, seen[1:])) < 0.2
