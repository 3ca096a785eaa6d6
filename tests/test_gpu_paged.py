"""Operators over a paged cache against 64-bit statements of them (tests/paged_ref.py).  Slots that hold no key are NaN in
every cache here, and table entries behind a request's last page lie outside the pool, unless a test says otherwise."""
import math
import random

import paged_ref as R
import pytest
import torch

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _tree(rng, m, roots=False):
    return [-1] + [rng.choice([-1] * roots + list(range(max(0, j - 5), j))) for j in range(1, m)]


def _queries(q_len, hq, h, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(sum(q_len), hq, h, generator=g).to(dtype)


def _cu(q_len):
    cu = [0]
    for m in q_len:
        cu.append(cu[-1] + m)
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def _check_attention(lens, q_len, hq, hkv, h, dtype, *, parents=None, page=16, weigh=False, scale=None, seed=0, garbage=float("nan"),
                     cache=None):
    """Runs the operator and compares out, lse and (weigh) the weights of every key."""
    k, v, table, n_kv = cache or R.make_cache(lens, hkv, h, dtype, page, seed, garbage=garbage)
    q = _queries(q_len, hq, h, dtype, seed + 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.full((sum(q_len), hq), 7.0, device="cuda")
    w0 = torch.rand(k.shape[:3], generator=torch.Generator().manual_seed(seed + 2))
    w = w0.cuda()
    flat = None if parents is None else torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda")
    kwargs = {} if scale is None else {"scale": scale}
    out = B.attention_tree(q.cuda(), k.cuda(), v.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len), flat, lse=lse, status=status,
                           key_weights=w if weigh else None, **kwargs)
    B.check_status(status)
    out, lse, w = out.cpu().double(), lse.cpu().double(), w.cpu().double()
    want_w, tol_w = w0.double().clone(), w0.double() * 2.0 ** -23
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(x, table[i], n, page) for x in (k, v))
        see = R.tree_mask(None if parents is None else parents[i], m, n)
        o, l, p, d_o, d_l, rel_p = R.attend(q[at:at + m], kk, vv, see, scale or h ** -0.5, dtype)
        bad = (out[at:at + m] - o).abs() - d_o
        assert not bool((bad > 0).any() | bad.isnan().any()), (i, n, m, float(bad.max()))
        got_l = lse[at:at + m]
        assert torch.equal(torch.isinf(got_l), torch.isinf(l))
        fine = ~torch.isinf(l)
        assert bool(((got_l - l).abs()[fine] <= d_l[fine]).all()), (i, float((got_l - l).abs()[fine].max()))
        if weigh:
            per = p.view(m, hkv, hq // hkv, n).sum((0, 2))
            off = (p * rel_p[..., None]).view(m, hkv, hq // hkv, n).sum((0, 2))
            for b in range((n + page - 1) // page):
                c = min(page, n - b * page)
                want_w[table[i, b], :, :c] += per[:, b * page:b * page + c]
                # the sum of the rows and its addition are rounded too
                tol_w[table[i, b], :, :c] += off[:, b * page:b * page + c] + per[:, b * page:b * page + c] * (m * hq // hkv + 2) * 2.0 ** -24
        at += m
    if weigh:
        assert bool(((w - want_w).abs() <= tol_w).all()), float(((w - want_w).abs() - tol_w).max())
    return out, lse


GEOMETRIES = [(32, 8, 128, BF), (32, 8, 64, BF), (8, 2, 128, BF), (4, 4, 64, F32), (8, 2, 128, F32), (6, 2, 32, F32), (6, 2, 32, BF),
              (5, 5, 128, BF), (16, 1, 64, BF), (7, 1, 128, F32), (40, 1, 128, BF)]


@pytest.mark.parametrize("hq,hkv,h,dtype", GEOMETRIES)
@pytest.mark.parametrize("weigh", [False, True])
def test_trees(hq, hkv, h, dtype, weigh):
    rng = random.Random(hq * 1000 + h)
    lens = [1, 2, 17, 16, 15, 63, 64, 65, 130, 9, 700, 33, 1025]
    q_len = [1, 1, 3, 16, 4, 2, 1, 8, 30, 9, 7, 12, 5]
    _check_attention(lens, q_len, hq, hkv, h, dtype, parents=[_tree(rng, m, roots=True) for m in q_len], weigh=weigh)


@pytest.mark.parametrize("hq,hkv,h,dtype", GEOMETRIES[:6])
def test_chains(hq, hkv, h, dtype):
    _check_attention([5, 0, 300, 64, 2000, 129], [5, 0, 200, 1, 3, 64], hq, hkv, h, dtype, weigh=True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [32, 64, 128, 256, 48])
def test_other_page_sizes(page, dtype):
    rng = random.Random(page)
    q_len = [4, 1, 9]
    _check_attention([page * 3 + 5, page, 777], q_len, 8, 2, 64, dtype, parents=[_tree(rng, m) for m in q_len], page=page, weigh=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_largest_trees(dtype):
    rng = random.Random(4)
    q_len = [128, 127, 65, 1]
    _check_attention([128, 1000, 400, 90], q_len, 8, 2, 128, dtype, parents=[_tree(rng, 128, True), [-1] + list(range(126)), [-1] * 65, [-1]],
                     weigh=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_long_context_and_many_short_ones(dtype):
    rng = random.Random(5)
    _check_attention([20011], [3], 8, 2, 128, dtype, parents=[[-1, 0, 0]], weigh=True)
    lens = [rng.randint(1, 90) for _ in range(300)]
    q_len = [rng.randint(1, min(n, 3)) for n in lens]
    _check_attention(lens, q_len, 8, 2, 64, dtype, parents=[_tree(rng, m) for m in q_len], weigh=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_unused_nodes_and_those_that_hang_on_them(dtype):
    parents = [[-1, -2, 1, 0, 3], [-2, -2, -2], [-1, 0, -2, 2, 3, 1, -1], [-2]]
    out, lse = _check_attention([40, 3, 100, 1], [5, 3, 7, 1], 8, 2, 64, dtype, parents=parents, weigh=True)
    empty = [1, 2, 5, 6, 7, 10, 11, 12, 15]
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_keys_that_a_row_does_not_see_may_be_anything(dtype, what):
    # node 1 of 3 holds no finite key or value: nodes 0 and 2 do not see it, its own row is not finite
    lens, q_len, parents = [150, 70], [3, 1], [[-1, 0, 0], [-1]]
    k, v, table, n_kv = R.make_cache(lens, 2, 64, dtype, seed=3)
    for x in (k, v):
        x[table[0, 148 // 16], :, 148 % 16] = what
    q = _queries(q_len, 8, 64, dtype, 1)
    lse = torch.empty(4, 8, device="cuda")
    out = B.attention_tree(q.cuda(), k.cuda(), v.cuda(), table.cuda(), n_kv.cuda(), _cu(q_len),
                           torch.tensor([-1, 0, 0, -1], dtype=torch.int32, device="cuda"), lse=lse).cpu().double()
    at = 0
    for i, m in enumerate(q_len):
        kk, vv = (R.keys_of(torch.nan_to_num(x.float(), 0.0, 0.0, 0.0), table[i], lens[i], 16) for x in (k, v))
        o, l, _, d_o, d_l, _ = R.attend(q[at:at + m], kk, vv, R.tree_mask(parents[i], m, lens[i]), 0.125, dtype)
        for j in range(m):
            if (i, j) != (0, 1):
                assert bool(((out[at + j] - o[j]).abs() <= d_o[j]).all()) and bool(((lse[at + j].cpu() - l[j]).abs() <= d_l[j]).all())
        at += m
    if what != what:
        assert bool(out[1].isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_at_the_end_of_the_range(dtype):
    # one key far above all others, scores of thousands, and a cache of equal keys
    for make in (lambda k: k.mul_(40), lambda k: k.zero_(), lambda k: k[..., ::3, :].mul_(100)):
        cache = R.make_cache([200, 90], 2, 64, dtype, seed=7, garbage=0.0)
        make(cache[0])
        _check_attention([200, 90], [4, 2], 8, 2, 64, dtype, parents=[[-1, 0, 0, 1], [-1, 0]], cache=cache, seed=7, weigh=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scale_strides_and_rows_of_nobody(dtype):
    _check_attention([77, 5], [3, 2], 8, 2, 64, dtype, parents=[[-1, 0, 1], [-1, 0]], scale=0.31)
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([77, 5], 2, 64, dtype, seed=0))
    wide = torch.randn(9, 12, 64, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()    # q, k and v heads of one projection
    q = wide[:, :8]
    parents = torch.tensor([-1, 0, 1, -1, 0, 5, -9, 99, 3], dtype=torch.int32, device="cuda")     # four rows belong to nobody
    cu = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    big = torch.full((9, 10, 64), 5.0, dtype=dtype, device="cuda")
    lse = torch.full((9, 8), 5.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    big_table = torch.full((2, table.shape[1] + 9), 1 << 30, dtype=torch.int32, device="cuda")
    big_table[:, :table.shape[1]] = table
    got = B.attention_tree(q, k, v, big_table[:, :table.shape[1]], n_kv, cu, parents, out=big[:, :8], lse=lse, status=status)
    B.check_status(status)
    same = B.attention_tree(q[:5].contiguous(), k, v, table, n_kv, cu, parents[:5].contiguous())
    assert got.data_ptr() == big.data_ptr() and torch.equal(got[:5], same)
    assert bool((big[5:] == 5).all()) and bool((big[:, 8:] == 5).all()) and bool((lse[5:] == 5).all())


def test_results_are_the_same_twice_and_in_any_batch_slot_within_rounding():
    rng = random.Random(8)
    lens, q_len = [500, 3000, 90], [6, 9, 3]
    parents = [_tree(rng, m) for m in q_len]
    a = _check_attention(lens, q_len, 32, 8, 128, BF, parents=parents, weigh=True)
    b = _check_attention(lens, q_len, 32, 8, 128, BF, parents=parents, weigh=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------------------------------- what only the GPU can see
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("fault", ["keys beyond the table", "fewer keys than rows", "negative keys", "rows beyond the call", "rows run backwards",
                                   "tree too large"])
def test_a_request_that_does_not_hold_together_is_left_out(fault, dtype):
    lens, q_len = [100, 40, 70], [4, 5, 3]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype, garbage=0.0))
    rows = 140
    q = _queries([rows], 4, 64, dtype, 3).cuda()
    parents = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    cu = _cu(q_len)
    good = B.attention_tree(q, k, v, table, n_kv, cu, parents, key_weights=torch.zeros(k.shape[:3], device="cuda"))
    near = lambda a, b: bool(((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-3).all())   # the work is shared out anew
    code = B.SLED_ERR_ARG
    if fault == "keys beyond the table":
        n_kv[1] = 16 * table.shape[1] + 1
    elif fault == "fewer keys than rows":
        n_kv[1] = 4
    elif fault == "negative keys":
        n_kv[1] = -3
    elif fault == "rows beyond the call":
        cu[2], cu[3] = rows + 1, rows + 2
    elif fault == "rows run backwards":
        cu[2] = 2
    else:
        cu[2], cu[3] = 4 + 129, 136
        table = torch.cat([table, table[:, :1].expand(3, 8)], 1).contiguous().clamp(0, k.shape[0] - 1)
        n_kv[1] = 130
        code = B.SLED_ERR_K_RANGE
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    weights = torch.zeros(k.shape[:3], device="cuda")
    B.attention_tree(q, k, v, table, n_kv, cu, parents, out=out, status=status, key_weights=weights)
    with pytest.raises(B.SledError) as e:
        B.check_status(status)
    assert e.value.code == code
    assert near(out[:4], good[:4])
    if fault not in ("rows beyond the call", "rows run backwards", "tree too large"):
        assert bool((out[4:9] == 3).all()) and near(out[9:12], good[9:12])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_outside_the_pool_and_parents_that_are_no_earlier_nodes(dtype):
    lens, q_len = [100, 40], [4, 5]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype, garbage=0.0))
    q = _queries(q_len, 4, 64, dtype, 3).cuda()
    parents = torch.tensor([-1, 0, 1, 0, -1, 0, 2, 7, -5], dtype=torch.int32, device="cuda")     # three nodes of the second request
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.attention_tree(q, k, v, table, n_kv, _cu(q_len), parents, status=status)
    assert status.item() == B.SLED_ERR_ARG
    assert bool((out[6:] == 0).all()) and bool((out[:6] != 0).any(-1).all())
    good = B.attention_tree(q, k, v, table, n_kv, _cu(q_len))
    for page in (k.shape[0], -1, 2 ** 31 - 1, -2 ** 31):
        status.zero_()
        wrong = table.clone()
        wrong[1, 1] = page
        w, w_good = torch.zeros(k.shape[:3], device="cuda"), torch.zeros(k.shape[:3], device="cuda")
        out = B.attention_tree(q, k, v, wrong, n_kv, _cu(q_len), status=status, key_weights=w)
        assert status.item() == B.SLED_ERR_ARG and torch.equal(out[:4], good[:4])
        B.attention_tree(q, k, v, table, n_kv, _cu(q_len), key_weights=w_good)
        others = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
        others[table[1, :3].long()] = False                                             # nobody else's weights are touched
        assert torch.equal(w[others], w_good[others])
        status.zero_()
        kk, vv, w = k.clone(), v.clone(), torch.rand(k.shape[:3], device="cuda")
        B.evict_keys(kk, vv, w.clone(), wrong, n_kv, 24, n_recent=4, status=status)     # the second request is left as it is
        assert status.item() == B.SLED_ERR_ARG and not torch.equal(kk, k)
        others = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
        others[table[0, :7].long()] = False
        assert torch.equal(kk[others], k[others]) and torch.equal(vv[others], v[others])
        status.zero_()
        bounds = torch.zeros(k.shape[0], 2, 2, 64, dtype=dtype, device="cuda")
        right = bounds.clone()
        B.block_bounds(k, wrong, n_kv, bounds, status=status)
        B.block_bounds(k, table, n_kv, right)
        right[table[1, 1].long()] = 0
        assert status.item() == B.SLED_ERR_ARG and torch.equal(bounds, right)
        status.zero_()
        B.attention_blocks(q, k, v, bounds, wrong, n_kv, _cu(q_len), n_blocks=2, status=status)
        assert status.item() == B.SLED_ERR_ARG


# ------------------------------------------------------------------------------------------------------------ eviction
def _check_eviction(lens, budget, sink, recent, *, hkv=2, h=64, dtype=BF, layers=2, page=16, seed=0, weights=None, separate=False, one_layer=False):
    k, v, table, n_kv = R.make_cache(lens, hkv, h, dtype, page, seed, layers=layers, garbage=2.0)
    w = torch.randn(k.shape[:4], generator=torch.Generator().manual_seed(seed + 9))
    if weights is not None:
        w = weights(w)
    gk, gv, gw = k.cuda(), v.cuda(), w.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    w_out = torch.full_like(gw, 77.0) if separate else None
    if one_layer:
        assert layers == 1
        B.evict_keys(gk[0], gv[0], gw[0], table.cuda(), n_kv.cuda(), budget, n_sink=sink, n_recent=recent, status=status,
                     key_weights_out=None if w_out is None else w_out[0])
    else:
        B.evict_keys(gk, gv, gw, table.cuda(), n_kv.cuda(), budget, n_sink=sink, n_recent=recent, status=status, key_weights_out=w_out)
    B.check_status(status)
    want_k, want_v = k.clone(), v.clone()
    want_w = torch.full_like(w, 77.0) if separate else w.clone()
    for i, n in enumerate(lens):
        place = [(int(table[i, x // page]), x % page) for x in range(n)]
        for layer in range(layers):
            for g in range(hkv):
                mine = [w[layer, p, g, s].item() for p, s in place]
                for x, y in enumerate(R.evicted(mine, n, budget, sink, recent)):
                    (p, s), (pp, ss) = place[x], place[y]
                    want_k[layer, p, g, s], want_v[layer, p, g, s] = k[layer, pp, g, ss], v[layer, pp, g, ss]
                    want_w[layer, p, g, s] = w[layer, pp, g, ss]
    # slots behind the kept keys are nobody's: only what holds a key, and pages of others, are compared
    live = torch.ones(k.shape[1], page, dtype=torch.bool)
    for i, n in enumerate(lens):
        for x in range(min(n, budget), n):
            live[table[i, x // page], x % page] = False
    pick = live[None, :, None].expand(w.shape)
    got_w = (w_out if separate else gw).cpu()
    assert torch.equal(gk.cpu()[pick], want_k[pick]) and torch.equal(gv.cpu()[pick], want_v[pick])
    assert torch.equal(got_w[pick].nan_to_num(123.0), want_w[pick].nan_to_num(123.0))
    if separate:
        assert bool((got_w[~pick] == 77).all()) and torch.equal(gw.cpu().nan_to_num(123.0), w.nan_to_num(123.0))


@pytest.mark.parametrize("budget,sink,recent", [(64, 4, 16), (1, 0, 0), (1, 1, 0), (1, 0, 1), (40, 40, 0), (40, 0, 40), (40, 20, 20), (37, 3, 30),
                                                (500, 4, 100), (100000, 4, 4), (199, 0, 1), (17, 1, 0)])
@pytest.mark.parametrize("separate", [False, True])
def test_eviction(budget, sink, recent, separate):
    _check_eviction([0, 1, 40, 41, 200, 64, 65, 700, 1300], budget, sink, recent, separate=separate)


@pytest.mark.parametrize("dtype,h,hkv,page", [(F32, 128, 2, 16), (F32, 32, 3, 16), (BF, 32, 1, 32), (BF, 128, 8, 64), (F32, 64, 2, 256)])
def test_eviction_of_other_caches(dtype, h, hkv, page):
    _check_eviction([300, 33, 1000, 129], 128, 4, 50, dtype=dtype, h=h, hkv=hkv, page=page)
    _check_eviction([300, 2000], 129, 3, 5, dtype=dtype, h=h, hkv=hkv, page=page, layers=1, one_layer=True)


@pytest.mark.parametrize("weights", [lambda w: torch.zeros_like(w), lambda w: (w * 2).round(), lambda w: torch.where(w > 1, float("nan"), w),
                                     lambda w: torch.where(w > 1, float("inf"), torch.where(w < -1, -float("inf"), w)),
                                     lambda w: torch.where(w > 0, 0.0, -0.0), lambda w: w * 1e-40, lambda w: -w.abs(),
                                     lambda w: torch.arange(w.shape[-1]).float().expand_as(w).contiguous()],
                         ids=["equal", "ties", "nan", "inf", "zeros of both signs", "subnormal", "negative", "rising"])
def test_eviction_by_odd_weights(weights):
    _check_eviction([500, 90, 260], 80, 4, 16, weights=weights)


def test_eviction_of_a_long_context():
    _check_eviction([40000, 100], 3001, 4, 700, layers=1, hkv=2, h=32)
    _check_eviction([40000], 39990, 4, 700, layers=1, hkv=1, h=32)


def test_eviction_twice_keeps_the_newest_last():
    # the second eviction knows the newest keys by their place: those appended since, and those of the first call before them
    hkv, h, page = 2, 64, 16
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([400], hkv, h, F32, page, seed=2, layers=1, garbage=0.0))
    at = lambda x: (0, int(table[0, x // page]), slice(None), x % page)
    for x in range(400):
        k[at(x)] = float(x)                # a key that says which token it is
    w = torch.rand(k.shape[:4], device="cuda")
    B.evict_keys(k, v, w, table, n_kv, 100, n_sink=2, n_recent=32)
    for x in range(100, 140):              # forty more tokens
        k[at(x)] = float(300 + x)
    n_kv.fill_(140)
    B.evict_keys(k, v, w, table, n_kv, 100, n_sink=2, n_recent=50)
    tokens = [[k[at(x)][g, 0].item() for x in range(100)] for g in range(hkv)]
    for t in tokens:
        assert t[:2] == [0, 1] and t[50:] == list(range(390, 440)) and len(set(t)) == 100


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_eviction_leaves_out_a_request_with_impossible_lengths(bad):
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([100, 90], 2, 64, BF, layers=1, garbage=0.0))
    w = torch.rand(k.shape[:4], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n_kv[0] = bad
    before = k.clone()
    B.evict_keys(k, v, w, table, n_kv, 40, status=status)
    assert status.item() == B.SLED_ERR_ARG
    mine = table[0, :7].long()
    assert torch.equal(k[0, mine], before[0, mine]) and not torch.equal(k, before)


# ------------------------------------------------------------------------------------------------------- bounds, blocks
@pytest.mark.parametrize("hq,hkv,h,dtype", GEOMETRIES[:7])
@pytest.mark.parametrize("page", [16, 64])
def test_bounds(hq, hkv, h, dtype, page):
    lens, first = [1, 16, 17, 300, 0, 1000, 64], [0, 3, 16, 250, 0, 0, 64]
    k, v, table, n_kv = R.make_cache(lens, hkv, h, dtype, page)
    for use_first in (False, True):
        got = torch.full((k.shape[0], hkv, 2, h), 9.0, dtype=dtype)
        want = got.clone()
        got = got.cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.block_bounds(k.cuda(), table.cuda(), n_kv.cuda(), got, status=status,
                       first=torch.tensor(first, dtype=torch.int32, device="cuda") if use_first else None)
        B.check_status(status)
        for i, n in enumerate(lens):
            for b in range(first[i] // page if use_first else 0, (n + page - 1) // page):
                if use_first and first[i] >= n:
                    continue
                x = k[table[i, b], :, :min(page, n - b * page)]
                want[table[i, b]] = torch.stack([x.amin(1), x.amax(1)], 1)
        assert torch.equal(got.cpu(), want)


def test_bounds_of_keys_that_are_no_numbers():
    k, _, table, n_kv = R.make_cache([40], 1, 64, BF, garbage=1.0)
    k[table[0, 1], 0, 3, 5] = float("nan")
    k[table[0, 0], 0, 2, 7] = float("inf")
    got = torch.zeros(k.shape[0], 1, 2, 64, dtype=BF, device="cuda")
    B.block_bounds(k.cuda(), table.cuda(), n_kv.cuda(), got)
    got = got.cpu()
    assert bool(got[table[0, 1], 0, :, 5].isnan().all()) and got[table[0, 0], 0, 1, 7] == float("inf") and int(got.isnan().sum()) == 2


def _check_blocks(lens, q_len, n_blocks, n_local, hq, hkv, h, dtype, page=16, seed=0, bounds=None, change=None):
    k, v, table, n_kv = R.make_cache(lens, hkv, h, dtype, page, seed)
    if change:
        change(k, v, table)
    q = _queries(q_len, hq, h, dtype, seed + 1)
    dev = [t.cuda() for t in (k, v, table, n_kv)]
    if bounds is None:
        bounds = torch.full((k.shape[0], hkv, 2, h), float("nan"), dtype=dtype, device="cuda")
        B.block_bounds(dev[0], dev[2], dev[3], bounds)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    blocks = torch.full((sum(q_len), hkv, n_blocks), -5, dtype=torch.int32, device="cuda")
    out = B.attention_blocks(q.cuda(), dev[0], dev[1], bounds, dev[2], dev[3], _cu(q_len), n_blocks=n_blocks, n_local=n_local,
                             blocks=blocks, status=status)
    B.check_status(status)
    plain = B.attention_blocks(q.cuda(), dev[0], dev[1], bounds, dev[2], dev[3], _cu(q_len), n_blocks=n_blocks, n_local=n_local)
    assert torch.equal(plain.nan_to_num(1.5), out.nan_to_num(1.5))
    out, blocks, bounds = out.cpu().double(), blocks.cpu(), bounds.cpu()
    t = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(x, table[i], n, page) for x in (k, v))
        for j in range(m):
            x = n - m + j
            own = x // page
            count = min(n_blocks, own + 1)
            got = blocks[t, :, :count]
            assert bool((blocks[t, :, count:] == -5).all())
            assert bool((got[:, 1:] > got[:, :-1]).all()) and bool((got >= 0).all()) and bool((got <= own).all())
            if own + 1 > n_blocks:
                early, want = own + 1 - n_local, n_blocks - n_local
                assert bool((got[:, want:] == torch.arange(early, own + 1)).all())
                b = bounds[table[i, :early].long()]
                s = R.block_scores(q[t], b, hkv)
                size = (q[t].double().abs().view(hkv, -1, 1, h) * b.double().abs().amax(2).transpose(0, 1)[:, None]).sum(-1).amax((1, 2))
                off = (2 * size * (2 * h + 8) * 2.0 ** -24)                    # two scores that are nearer than this may change places
                for g in range(hkv):
                    mine = got[g, :want].long()
                    rest = torch.ones(early, dtype=torch.bool)
                    rest[mine] = False
                    if want and bool(rest.any()):
                        assert s[g, mine].min() >= s[g, rest].max() - off[g], (i, j, g)
            see = torch.zeros(1, hkv, n, dtype=torch.bool)
            for g in range(hkv):
                for b in got[g].tolist():
                    see[0, g, b * page:min((b + 1) * page, x + 1)] = True
            o, _, _, d_o, _, _ = R.attend(q[t:t + 1], kk, vv, see, h ** -0.5, dtype)
            assert bool(((out[t] - o[0]).abs() <= d_o[0]).all()), (i, j, float(((out[t] - o[0]).abs() - d_o[0]).max()))
            t += 1
    return out


@pytest.mark.parametrize("hq,hkv,h,dtype", GEOMETRIES)
def test_blocks(hq, hkv, h, dtype):
    _check_blocks([1, 16, 17, 100, 400, 1200, 2500], [1, 2, 3, 1, 9, 2, 1], 12, 2, hq, hkv, h, dtype)


@pytest.mark.parametrize("n_blocks,n_local", [(1, 1), (2, 1), (2, 2), (7, 7), (33, 1), (100, 3), (64, 64)])
def test_block_counts(n_blocks, n_local):
    _check_blocks([900, 40, 161, 1600], [2, 1, 5, 1], n_blocks, n_local, 8, 2, 64, BF)


@pytest.mark.parametrize("page", [32, 64, 256, 48])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_blocks_of_other_sizes(page, dtype):
    _check_blocks([page * 20 + 3, page * 5, 7], [2, 1, 1], 6, 2, 8, 2, 64, dtype, page=page)


def test_blocks_of_a_long_context():
    _check_blocks([50000], [2], 40, 4, 8, 2, 128, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_block_choice_among_equals_and_numbers_that_are_none(dtype):
    # all scores equal: the lowest blocks; a block whose bounds are NaN comes first
    lens, hkv, h = [640], 2, 64
    q_len = [1]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, hkv, h, dtype, garbage=0.0))
    q = _queries(q_len, 4, h, dtype, 1).cuda()
    bounds = torch.ones(k.shape[0], hkv, 2, h, dtype=dtype, device="cuda")
    blocks = torch.zeros(1, hkv, 9, dtype=torch.int32, device="cuda")
    B.attention_blocks(q, k, v, bounds, table, n_kv, _cu(q_len), n_blocks=9, n_local=2, blocks=blocks)
    assert blocks[0].tolist() == [[0, 1, 2, 3, 4, 5, 6, 38, 39]] * 2
    bounds[table[0, 20].long(), 1] = float("nan")
    B.attention_blocks(q, k, v, bounds, table, n_kv, _cu(q_len), n_blocks=9, n_local=2, blocks=blocks)
    assert blocks[0].tolist() == [[0, 1, 2, 3, 4, 5, 6, 38, 39], [0, 1, 2, 3, 4, 5, 20, 38, 39]]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_enough_blocks_are_full_attention(dtype):
    lens, q_len = [300, 77, 16], [5, 1, 16]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype))
    q = _queries(q_len, 8, 64, dtype, 1).cuda()
    bounds = torch.zeros(k.shape[0], 2, 2, 64, dtype=dtype, device="cuda")
    a = B.attention_blocks(q, k, v, bounds, table, n_kv, _cu(q_len), n_blocks=19)
    b = B.attention_tree(q, k, v, table, n_kv, _cu(q_len))
    assert float((a.double() - b.double()).abs().max()) <= (2 ** -7 if dtype == BF else 1e-5) * float(b.abs().max())


# ------------------------------------------------------------------------------------- streams, graphs, devices, together
def _decode_setup(dtype=BF):
    lens, q_len = [900, 130, 47], [3, 1, 4]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 128, dtype, garbage=0.0))
    q = _queries(q_len, 8, 128, dtype, 1).cuda()
    bounds = torch.zeros(k.shape[0], 2, 2, 128, dtype=dtype, device="cuda")
    parents = torch.tensor([-1, 0, 0, -1, -1, 0, 1, 1], dtype=torch.int32, device="cuda")
    return k, v, table, n_kv, q, bounds, parents, _cu(q_len)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_into_a_graph_and_replayed_with_other_inputs(dtype):
    k, v, table, n_kv, q, bounds, parents, cu = _decode_setup(dtype)
    w = torch.zeros(k.shape[:3], device="cuda")

    def step():
        a = B.attention_tree(q, k, v, table, n_kv, cu, parents, key_weights=w)
        B.block_bounds(k, table, n_kv, bounds)
        return a, B.attention_blocks(q, k, v, bounds, table, n_kv, cu, n_blocks=8, n_local=2)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = step()
    for new in ((900, 130, 47), (700, 100, 20), (16, 3, 4)):
        n_kv.copy_(torch.tensor(new, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, device="cuda").to(dtype))
        w.zero_()
        graph.replay()
        got = [t.clone() for t in (a, b, w)]
        w.zero_()
        want = step() + (w,)
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_on_a_stream_of_its_own_behind_other_work():
    k, v, table, n_kv, q, bounds, parents, cu = _decode_setup()
    want = B.attention_tree(q, k, v, table, n_kv, cu, parents)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.randn(2000, 2000, device="cuda") @ torch.randn(2000, 2000, device="cuda")
        late.copy_(q)                            # the queries are there only when the work before them is done
        got = B.attention_tree(late, k, v, table, n_kv, cu, parents)
    side.synchronize()
    assert torch.equal(got, want)


def test_two_streams_at_once():
    k, v, table, n_kv, q, bounds, parents, cu = _decode_setup()
    B.block_bounds(k, table, n_kv, bounds)
    want = (B.attention_tree(q, k, v, table, n_kv, cu, parents), B.attention_blocks(q, k, v, bounds, table, n_kv, cu, n_blocks=5))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(30):
        for s, g, f in zip(streams, got, (lambda: B.attention_tree(q, k, v, table, n_kv, cu, parents),
                                          lambda: B.attention_blocks(q, k, v, bounds, table, n_kv, cu, n_blocks=5))):
            with torch.cuda.stream(s):
                g.append(f())
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)


def test_a_conversation_under_a_budget():
    """As a server would use them: a prompt's cache, draft trees verified with weights kept, the accepted path's keys put in
    place, eviction when the budget is passed, sparse attention with the bounds kept up - all against 64 bits."""
    rng = random.Random(11)
    hq, hkv, h, page, budget = 8, 2, 64, 16, 96
    lens = [90, 80]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([160, 160], hkv, h, BF, page, seed=4, garbage=0.0))
    n_kv.copy_(torch.tensor(lens, dtype=torch.int32))
    w = torch.zeros(k.shape[:3], device="cuda")
    bounds = torch.zeros(k.shape[0], hkv, 2, h, dtype=BF, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ref_w = w.cpu().double()
    slot = lambda i, x: (int(table[i, x // page]), slice(None), x % page)
    g = torch.Generator().manual_seed(6)
    for step in range(12):
        m = [rng.randint(1, 9), rng.randint(1, 9)]
        parents = [_tree(rng, x) for x in m]
        n_kv += torch.tensor(m, dtype=torch.int32, device="cuda")             # the trees' keys are written behind the cache
        for i in range(2):
            for j in range(m[i]):
                x = lens[i] + j
                k[slot(i, x)] = torch.randn(hkv, h, generator=g).to(BF).cuda()
                v[slot(i, x)] = torch.randn(hkv, h, generator=g).to(BF).cuda()
                w[slot(i, x)] = 0
        q = torch.randn(sum(m), hq, h, generator=g).to(BF)
        ref_w = w.cpu().double()
        out = B.attention_tree(q.cuda(), k, v, table, n_kv, _cu(m), torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda"),
                               key_weights=w, status=status).cpu().double()
        ck, cv, ct, at = k.cpu(), v.cpu(), table.cpu(), 0
        for i in range(2):
            n = lens[i] + m[i]
            kk, vv = (R.keys_of(x, ct[i], n, page) for x in (ck, cv))
            o, _, p, d_o, _, rel = R.attend(q[at:at + m[i]], kk, vv, R.tree_mask(parents[i], m[i], n), h ** -0.5, BF)
            assert bool(((out[at:at + m[i]] - o).abs() <= d_o).all())
            per = p.view(m[i], hkv, -1, n).sum((0, 2))
            for x in range(n):
                got, want = w[slot(i, x)].cpu().double(), ref_w[slot(i, x)] + per[:, x]
                assert bool(((got - want).abs() <= (float(rel.max()) + 2.0 ** -18) * want + 1e-30).all())
            # the path to a random node is accepted: its keys close up behind the cache
            path, a = [], rng.randrange(m[i])
            while a >= 0:
                path.append(a)
                a = parents[i][a]
            for d, a in enumerate(reversed(path)):
                for x in (k, v, w):
                    x[slot(i, lens[i] + d)] = x[slot(i, lens[i] + a)].clone()
            lens[i] += len(path)
            at += m[i]
        n_kv.copy_(torch.tensor(lens, dtype=torch.int32))
        if max(lens) > budget:
            before = (k.cpu(), w.cpu())
            B.evict_keys(k, v, w, table, n_kv, budget, n_sink=2, n_recent=16, status=status)
            for i in range(2):
                for gg in range(hkv):
                    come = R.evicted([before[1][slot(i, x)][gg].item() for x in range(lens[i])], lens[i], budget, 2, 16)
                    for x, y in enumerate(come):
                        assert torch.equal(k[slot(i, x)][gg].cpu(), before[0][slot(i, y)][gg])
            lens = [min(n, budget) for n in lens]
            n_kv.copy_(torch.tensor(lens, dtype=torch.int32))
        B.block_bounds(k, table, n_kv, bounds, status=status)
        one = torch.randn(2, hq, h, generator=g).to(BF)
        blocks = torch.full((2, hkv, 3), -1, dtype=torch.int32, device="cuda")
        got = B.attention_blocks(one.cuda(), k, v, bounds, table, n_kv, _cu([1, 1]), n_blocks=3, blocks=blocks, status=status).cpu().double()
        ck, cv = k.cpu(), v.cpu()
        for i in range(2):
            kk, vv = (R.keys_of(x, ct[i], lens[i], page) for x in (ck, cv))
            see = torch.zeros(1, hkv, lens[i], dtype=torch.bool)
            for gg in range(hkv):
                for b in blocks[i, gg].tolist():
                    see[0, gg, b * page:(b + 1) * page] = True
            o, _, _, d_o, _, _ = R.attend(one[i:i + 1], kk, vv, see, h ** -0.5, BF)
            assert bool(((got[i] - o[0]).abs() <= d_o[0]).all())
    B.check_status(status)
