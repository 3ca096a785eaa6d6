"""Operators over a paged cache where numbers, lengths or tables are unusual, against the 64-bit statements of tests/paged_ref.py."""
import math
import random
import threading

import paged_ref as R
import pytest
import torch
from test_gpu_paged import BF, F32, _cu, _queries, _tree

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _close(got, want, tol):
    """Equal where the wanted values are no finite numbers, within tol elsewhere."""
    odd = ~torch.isfinite(want)
    fine = (got - want).abs() <= tol
    assert bool(torch.where(odd, (got == want) | (got.isnan() & want.isnan()), fine).all()), \
        (int((odd & ~((got == want) | (got.isnan() & want.isnan()))).sum()), float((got - want)[~odd].abs().sub(tol[~odd]).max()))


def _widened(table, columns):
    """The same table with `columns` columns; those behind the requests' pages lie outside the pool."""
    wide = torch.full((table.shape[0], columns), 1 << 30, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    return wide


def _check_call(cache, q, lens, q_len, parents=None, *, columns=0, weigh=True):
    """Runs sled_attention_tree on a cache and queries that may hold anything, and compares out, lse and weights."""
    k, v, table, n_kv = cache
    hkv, page, h = k.shape[1:]
    hq = q.shape[1]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.full((sum(q_len), hq), 7.0, device="cuda")
    w0 = torch.rand(k.shape[:3], generator=torch.Generator().manual_seed(5))
    w = w0.cuda()
    flat = None if parents is None else torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda")
    gpu_table = (_widened(table, columns) if columns else table).cuda()
    out = B.attention_tree(q.cuda(), k.cuda(), v.cuda(), gpu_table, n_kv.cuda(), _cu(q_len), flat, lse=lse, status=status,
                           key_weights=w if weigh else None)
    B.check_status(status)
    out, lse, w = out.cpu().double(), lse.cpu().double(), w.cpu().double()
    want_w, tol_w = w0.double().clone(), w0.double() * 2.0 ** -23
    at = 0
    for i, (n, m) in enumerate(zip(lens, q_len)):
        kk, vv = (R.keys_of(x, table[i], n, page) for x in (k, v))
        see = R.tree_mask(None if parents is None else parents[i], m, n)
        o, l, p, d_o, d_l, rel = R.attend(q[at:at + m], kk, torch.where(torch.isfinite(vv), vv, 0), see, h ** -0.5, q.dtype)
        # values that are no numbers reach the rows that see them, and no others
        seen = p.view(m, hkv, hq // hkv, n) > 0
        for what, value in ((vv == INF, INF), (vv == -INF, -INF), (vv.isnan(), NAN)):
            hit = torch.einsum("mgrn,gnd->mgrd", seen.double(), what.double()).reshape(m, hq, h) > 0
            o = o + torch.where(hit, value, 0.0)
        _close(out[at:at + m], o, d_o)
        _close(lse[at:at + m], l, d_l)
        per = p.view(m, hkv, hq // hkv, n).sum((0, 2))
        off = (p * rel.nan_to_num()[..., None]).view(m, hkv, hq // hkv, n).sum((0, 2))
        for b in range((n + page - 1) // page):
            c = min(page, n - b * page)
            want_w[table[i, b], :, :c] += per[:, b * page:b * page + c]
            # the sum of the rows and its addition are rounded too
            tol_w[table[i, b], :, :c] += off[:, b * page:b * page + c] + per[:, b * page:b * page + c] * (m * hq // hkv + 2) * 2.0 ** -24
        at += m
    if weigh:
        _close(w, want_w, tol_w)
    return out


# (query heads, nodes a request, table columns): weights from kept scores, by tcgen05 (bf16), and without kept scores
PATHS = [(8, 5, 0), (8, 40, 0), (8, 5, 300000)]


@pytest.mark.parametrize("what", [NAN, INF, -INF])
@pytest.mark.parametrize("hq,m,columns", PATHS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_of_unused_nodes_may_be_anything(dtype, hq, m, columns, what):
    """A batch padded with unused nodes: what their queries hold reaches neither results nor weights."""
    lens, q_len = [400, 70, 129], [m, m, m]
    rng = random.Random(m)
    parents = [_tree(rng, m) for _ in q_len]
    parents[0][m - 2] = parents[1][2] = -2
    parents[2] = [-2] * m                                   # a request without any used node
    q = _queries(q_len, hq, 64, dtype, 3)
    for i in range(3):
        for j, row in enumerate(R.tree_mask(parents[i], m, lens[i])):
            if not bool(row.any()):
                q[i * m + j] = what
    _check_call(R.make_cache(lens, 2, 64, dtype, seed=2), q, lens, q_len, parents, columns=columns)


@pytest.mark.parametrize("hq,m,columns", PATHS)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("chain", [False, True])
def test_a_row_that_is_no_number_weighs_only_on_the_keys_it_sees(dtype, hq, m, columns, chain):
    lens, q_len = [400, 70], [m, m]
    rng = random.Random(m)
    parents = None if chain else [[-1] * m, _tree(rng, m)]
    q = _queries(q_len, hq, 64, dtype, 3)
    q[1, 3, 9] = NAN                                        # second node of the first request, one head
    _check_call(R.make_cache(lens, 2, 64, dtype, seed=2), q, lens, q_len, parents, columns=columns)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_of_trees_where_the_scores_are_too_many_to_keep(dtype):
    lens, q_len = [100, 37, 16], [9, 5, 1]
    _check_call(R.make_cache(lens, 2, 64, dtype, seed=6), _queries(q_len, 8, 64, dtype, 7), lens, q_len,
                [[-1, 0, 0, -2, 3, 1, 5, -1, 7], [-1, 0, 1, 0, 3], [-1]], columns=300000)


# --------------------------------------------------------------------------------- units of 256 rows (paged_tc_kernel<H, 2>)
def _wide_columns(q_len, group, hkv, page=16):
    """Columns of a page table with which a call takes the kernel of 256-row units: 32 of its tiles to an SM."""
    rows = sum(q_len) * group // len(q_len)
    assert rows > 128
    tiles = 32 * torch.cuda.get_device_properties(0).multi_processor_count
    units = (rows + 127) // 256 * len(q_len) * hkv
    return ((tiles + units - 1) // units * 128 + page - 1) // page


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("lens,q_len", [([129, 300], [129, 130]), ([255, 1000, 400], [255, 1, 200]), ([256, 700], [256, 12]),
                                        ([257, 600, 90], [257, 128, 64]), ([512, 2000], [512, 3]), ([5000, 513, 30], [300, 513, 1])])
def test_units_of_256_rows_chains(lens, q_len, h):
    _check_call(R.make_cache(lens, 2, h, BF, seed=1), _queries(q_len, 2, h, BF, 2), lens, q_len, columns=_wide_columns(q_len, 1, 2))


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("hq", [8, 16])
def test_units_of_256_rows_trees(hq, h):
    """Requests on both sides of 128 and 256 rows, unused nodes, contexts that are cut into many shares."""
    rng = random.Random(hq + h)
    lens, q_len = [64, 300, 128, 90, 4000, 517, 33, 1500], [64, 65, 128, 3, 100, 32, 33, 127]
    parents = [_tree(rng, m, True) for m in q_len]
    for p in (parents[0], parents[2], parents[4], parents[7]):
        p[rng.randrange(len(p))] = -2
    parents[6] = [-2] * 33
    _check_call(R.make_cache(lens, 2, h, BF, seed=3), _queries(q_len, hq, h, BF, 4), lens, q_len, parents,
                columns=_wide_columns(q_len, hq // 2, 2))


@pytest.mark.parametrize("what", [NAN, INF, -INF])
@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_values_of_nodes_that_are_no_numbers(h, what, wide):
    """They reach the rows that see them and no others, in units of 128 and of 256 rows, whole and cut ones."""
    rng = random.Random(9)
    lens, q_len = [64, 300, 2500, 40], [64, 65, 100, 3]
    parents = [_tree(rng, m, True) for m in q_len]
    cache = R.make_cache(lens, 2, h, BF, seed=3)
    for i, j in ((0, 20), (1, 0), (1, 64), (2, 50), (3, 1)):
        x = lens[i] - q_len[i] + j
        cache[1][cache[2][i, x // 16], j % 2, x % 16, 5 + j % h // 2] = what
    x = lens[1] - q_len[1] - 2                              # and one of the keys that everybody sees, in a tile with nodes
    cache[1][cache[2][1, x // 16], 1, x % 16, h - 1] = what
    _check_call(cache, _queries(q_len, 8, h, BF, 4), lens, q_len, parents, columns=_wide_columns(q_len, 4, 2) if wide else 0)


@pytest.mark.parametrize("h", [64, 128])
def test_requests_on_both_sides_of_128_rows(h):
    """Small requests among large ones, 128 rows or less on average: the narrow kernel, with units of full and of few rows."""
    rng = random.Random(h + 1)
    q_len = [rng.choice([8] * 6 + [64, 33, 128]) for _ in range(40)]
    lens = [rng.randint(m, 2500) for m in q_len]
    assert 24 < sum(q_len) * 4 / 40 <= 128 and max(q_len) == 128
    _check_call(R.make_cache(lens, 2, h, BF, seed=5), _queries(q_len, 8, h, BF, 6), lens, q_len, [_tree(rng, m, True) for m in q_len])


# ------------------------------------------------------------------------------------------------------- bounds, choice
@pytest.mark.parametrize("dtype", [BF, F32])
def test_bounds_without_new_keys_are_left_alone(dtype):
    lens, first = [20, 20, 20, 33, 16, 47], [20, 25, 100, 32, 16, 47]
    k, _, table, n_kv = R.make_cache(lens, 2, 64, dtype)
    got = torch.full((k.shape[0], 2, 2, 64), 9.0, dtype=dtype)
    want = got.clone()
    got = got.cuda()
    B.block_bounds(k.cuda(), table.cuda(), n_kv.cuda(), got, first=torch.tensor(first, dtype=torch.int32, device="cuda"))
    x = k[table[3, 2], :, :1]                               # only the fourth request has a key there: its 33rd
    want[table[3, 2]] = torch.stack([x.amin(1), x.amax(1)], 1)
    assert torch.equal(got.cpu(), want)


def _check_choice(q, bounds, hkv, h, dtype, n_blocks=9, n_local=2):
    """One token over 40 blocks whose bounds are given; the choice by the definition, in 64 bits."""
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([640], hkv, h, dtype, garbage=0.0))
    mine = torch.zeros(k.shape[0], hkv, 2, h, dtype=dtype, device="cuda")
    mine[table[0].long()] = bounds.cuda()
    blocks = torch.full((1, hkv, n_blocks), -1, dtype=torch.int32, device="cuda")
    B.attention_blocks(q.cuda(), k, v, mine, table, n_kv, _cu([1]), n_blocks=n_blocks, n_local=n_local, blocks=blocks)
    blocks = blocks.cpu().long()
    early, want = 40 - n_local, n_blocks - n_local
    s = R.block_scores(q[0], bounds[:early], hkv)
    finite = torch.where(torch.isfinite(bounds), bounds, 0)[:early].double().abs().amax(2).transpose(0, 1)[:, None]
    size = (q[0].double().abs().nan_to_num(0, 0, 0).view(hkv, -1, 1, h) * finite).sum(-1).amax((1, 2))
    off = 2 * size * (2 * h + 8) * 2.0 ** -24               # two scores that are nearer than this may change places
    s = torch.where(s.isnan(), 3e300, torch.where(s == INF, 2e300, torch.where(s == -INF, -2e300, s)))
    for g in range(hkv):
        got = blocks[g * 0, g, :want]
        rest = torch.ones(early, dtype=torch.bool)
        rest[got] = False
        assert bool((got[1:] > got[:-1]).all()) and s[g, got].min() >= s[g, rest].max() - off[g], (g, got.tolist(), s[g].topk(want).indices.sort().values.tolist())
        edge = s[g, got].min()                              # among equals that are no finite numbers, the lowest blocks
        if float(edge.abs()) > 1e300:
            equal = (s[g] == edge).nonzero().flatten()
            taken = got[s[g, got] == edge]
            assert torch.equal(taken, equal[:len(taken)])


@pytest.mark.parametrize("dtype,h", [(BF, 64), (BF, 128), (BF, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("hq", [2, 8])
@pytest.mark.parametrize("which", ["high", "low", "both", "many"])
def test_scores_of_infinite_bounds(dtype, h, hq, which):
    """An infinite bound counts with the queries whose sign meets it, and with no others."""
    g = torch.Generator().manual_seed(h + hq)
    x = torch.randn(40, 2, 2, h, generator=g).sort(2).values.to(dtype)
    q = torch.randn(1, hq, h, generator=g).to(dtype)
    q[..., 7], q[..., 8] = -q[..., 7].abs() - 0.1, q[..., 8].abs() + 0.1
    if which == "high":
        x[11, :, 1, 7] = INF                                # a query component below 0 meets the low bound
    elif which == "low":
        x[11, :, 0, 8] = -INF
    elif which == "both":
        x[11, 0, 1, 7] = x[12, 1, 1, 8] = INF               # the second one is met
        x[13, :, 0, 7] = -INF                               # and so is this
    else:
        x[:, :, 1, 7] = INF
        x[::3, :, 0, 8] = -INF
    _check_choice(q, x, 2, h, dtype)


@pytest.mark.parametrize("dtype,h", [(BF, 64), (BF, 128), (BF, 32), (F32, 64)])
@pytest.mark.parametrize("what", [NAN, INF, -INF])
def test_choice_of_queries_that_are_no_numbers(dtype, h, what):
    g = torch.Generator().manual_seed(h)
    x = torch.randn(40, 2, 2, h, generator=g).sort(2).values.to(dtype)
    x[20, :, 0, 3] = x[30, :, 1, 3] = 0                     # infinity times 0 is no number
    q = torch.randn(1, 8, h, generator=g).to(dtype)
    q[0, 1, 3] = what                                       # one head of the first KV head
    _check_choice(q, x, 2, h, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_choice_among_more_blocks_than_stay_in_shared_memory(dtype):
    lens, hkv, h = [70000], 1, 64
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, hkv, h, dtype, garbage=0.0))
    q = _queries([1], 2, h, dtype, 1).cuda()
    bounds = torch.ones(k.shape[0], hkv, 2, h, dtype=dtype, device="cuda")
    own = (70000 - 1) // 16
    for n_blocks, better in ((4110, []), (4110, [4300, 4350]), (30, [10, 4095, 4096, 4097, 4371]), (4000, [4100])):
        b = bounds.clone()
        for x in better:                                    # every score term of these is at least as large
            b[table[0, x].long(), :, 0], b[table[0, x].long(), :, 1] = -2.0, 2.0
        blocks = torch.full((1, hkv, n_blocks), -1, dtype=torch.int32, device="cuda")
        out = B.attention_blocks(q, k, v, b, table, n_kv, _cu([1]), n_blocks=n_blocks, n_local=2, blocks=blocks)
        equal = [x for x in range(own - 1) if x not in better][:n_blocks - 2 - len(better)]
        want = sorted(equal + better) + [own - 1, own]
        assert blocks[0, 0].tolist() == want
        kk, vv = (R.keys_of(x.cpu(), table[0].cpu(), 70000, 16) for x in (k, v))
        see = torch.zeros(1, hkv, 70000, dtype=torch.bool)
        for x in want:
            see[..., x * 16:(x + 1) * 16] = True
        o, _, _, d_o, _, _ = R.attend(q.cpu(), kk, vv, see, h ** -0.5, dtype)
        _close(out.cpu().double(), o, d_o)


# -------------------------------------------------------------------------------------------------- arguments, batches
@pytest.mark.parametrize("dtype", [BF, F32])
def test_batches_of_nothing(dtype):
    k, v = (torch.zeros(4, 2, 16, 64, dtype=dtype, device="cuda") for _ in range(2))
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    status, w, bounds = ints(1), torch.ones(4, 2, 16, device="cuda"), torch.ones(4, 2, 2, 64, dtype=dtype, device="cuda")
    # no requests; requests without keys and a table without columns
    for table, n_kv, cu in ((ints(0, 5), ints(0), ints(1)), (ints(0, 0), ints(0), ints(1)), (ints(3, 0), ints(3), ints(4))):
        for rows in (0, 2):
            q = torch.zeros(rows, 8, 64, dtype=dtype, device="cuda")
            out = torch.full_like(q, 5.0)
            B.attention_tree(q, k, v, table, n_kv, cu, out=out, key_weights=w, status=status)
            B.attention_blocks(q, k, v, bounds, table, n_kv, cu, n_blocks=4, out=out, status=status)
            assert bool((out == 5).all())
        B.evict_keys(k, v, w, table, n_kv, 8, n_recent=2, status=status)
        B.block_bounds(k, table, n_kv, bounds, status=status)
    B.check_status(status)
    assert bool((w == 1).all()) and bool((bounds == 1).all())


def test_integers_of_any_shape_that_can_be_read():
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([12, 9], 2, 64, BF, seed=1))
    q = _queries([1, 1], 8, 64, BF, 2).cuda()
    want = B.attention_tree(q, k, v, table, n_kv, _cu([1, 1]))
    assert table.shape[1] == 1
    tall = torch.stack([table[:, 0], table[:, 0] + 1000], 0).t()[:, :1]          # one column, whose stride says nothing
    assert tall.stride() == (1, 2)
    status = torch.zeros((), dtype=torch.int32, device="cuda")
    assert torch.equal(B.attention_tree(q, k, v, tall, n_kv, _cu([1, 1]), status=status), want)
    B.check_status(status)
    n_kv[0] = 17
    B.attention_tree(q, k, v, table, n_kv, _cu([1, 1]), status=status)
    with pytest.raises(B.SledError):
        B.check_status(status)
    for wrong in (torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")):
        with pytest.raises(B.SledError):
            B.attention_tree(q, k, v, table, n_kv, _cu([1, 1]), status=wrong)
    with pytest.raises(B.SledError):
        B.block_bounds(k, table, n_kv, torch.zeros(k.shape[0], 2, 2, 64, dtype=BF, device="cuda"),
                       first=torch.zeros((), dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_requests_in_another_order(dtype):
    rng = random.Random(8)
    lens, q_len, parents = [500, 3000, 90, 64], [6, 9, 3, 30], None
    parents = [_tree(rng, m) for m in q_len]
    k, v, table, n_kv = R.make_cache(lens, 2, 128, dtype, seed=4)
    q = _queries(q_len, 8, 128, dtype, 5)
    rows, at = [], 0
    for m in q_len:
        rows.append(list(range(at, at + m)))
        at += m
    _check_call((k, v, table, n_kv), q, lens, q_len, parents)
    for order in ([3, 1, 0, 2], [1, 2, 3, 0]):
        pick = lambda x: [x[i] for i in order]
        _check_call((k, v, table[order], n_kv[order]), q[sum(pick(rows), [])], pick(lens), pick(q_len), pick(parents))


@pytest.mark.parametrize("n,group", [(300000, 1), (3000, 4)])
def test_long_chains_with_values_that_are_no_numbers(n, group):
    """A whole prompt as one chain: a value that is no number reaches the rows behind it, and takes the others no time to
    go round (in the long one a wait of the kernel would run out otherwise)."""
    h, page = 128, 256
    k, v, table, n_kv = R.make_cache([n], 1, h, BF, page, seed=7)
    for x, d, what in ((20, 3, NAN), (n // 2, 70, INF), (n - 2, 90, -INF)):
        v[table[0, x // page], 0, x % page, d] = what
    q = _queries([n], group, h, BF, 8)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros(n, group, device="cuda")
    out = B.attention_tree(q.cuda(), k.cuda(), v.cuda(), table.cuda(), n_kv.cuda(), _cu([n]), lse=lse, status=status)
    B.check_status(status)
    kk, vv = (R.keys_of(x, table[0], n, page) for x in (k, v))
    for j in (0, 19, 20, 21, 127, 128, 129, 1000, n // 2 - 1, n // 2, n // 2 + 1, n - 200, n - 3, n - 2, n - 1):
        see = torch.ones(1, j + 1, dtype=torch.bool)
        o, l, p, d_o, d_l, _ = R.attend(q[j:j + 1], kk[:, :j + 1], torch.where(torch.isfinite(vv[:, :j + 1]), vv[:, :j + 1], 0), see, h ** -0.5, BF)
        for x, d, what in ((20, 3, NAN), (n // 2, 70, INF), (n - 2, 90, -INF)):
            if x <= j:
                o[..., d] = what
        _close(out[j:j + 1].cpu().double(), o, d_o)
        _close(lse[j:j + 1].cpu().double(), l, d_l)


def test_calls_from_two_host_threads():
    """Each thread on a stream of its own, from the process's first calls of these shapes on."""
    sets = []
    for seed, (hq, h, dtype, m) in enumerate([(8, 128, BF, 3), (8, 64, BF, 40), (4, 32, F32, 5), (8, 128, F32, 2)]):
        lens, q_len = [500, 90], [m, m]
        k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, h, dtype, seed=seed, garbage=0.0))
        q = _queries(q_len, hq, h, dtype, seed).cuda()
        bounds = torch.zeros(k.shape[0], 2, 2, h, dtype=dtype, device="cuda")
        sets.append((q, k, v, table, n_kv, _cu(q_len), bounds))
    torch.cuda.synchronize()

    def calls(s):
        q, k, v, table, n_kv, cu, bounds = s
        w, mine = torch.zeros(k.shape[:3], device="cuda"), torch.zeros_like(bounds)
        a = B.attention_tree(q, k, v, table, n_kv, cu, key_weights=w)
        B.block_bounds(k, table, n_kv, mine)
        b = B.attention_blocks(q, k, v, mine, table, n_kv, cu, n_blocks=5)
        kk, vv, ww = k.clone(), v.clone(), w.clone()
        B.evict_keys(kk, vv, ww, table, n_kv, 60, n_recent=8)
        return a, w, mine, b, kk, vv, ww

    got, wrong, start = {}, [], threading.Barrier(2)

    def run(name):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                got[name] = [[calls(s) for s in sets] for _ in range(10)]
                torch.cuda.current_stream().synchronize()
        except Exception as e:      # noqa: BLE001 - the main thread reports it
            wrong.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    want = [calls(s) for s in sets]
    for rounds in got.values():
        for results in rounds:
            for x, y in zip(results, want):
                assert all(torch.equal(a, b) for a, b in zip(x, y))


@pytest.mark.parametrize("hq,m,columns", PATHS + [(8, 70, 0)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("chain", [False, True])
def test_keys_that_are_no_numbers_and_weights(dtype, hq, m, columns, chain):
    """Rows that see such a key are no numbers, nor are the weights of the keys that those rows see; all others are untouched."""
    rng = random.Random(m)
    lens, q_len = [400, 90, 300], [m, m, 1]
    parents = None if chain else [_tree(rng, m, True), _tree(rng, m), [-1]]
    cache = R.make_cache(lens, 2, 64, dtype, seed=2)
    for i, j, g in ((0, 2, 0), (0, m - 1, 1), (1, m - 2, 0)):
        x = lens[i] - m + j
        cache[0][cache[2][i, x // 16], g, x % 16, 11] = NAN
    _check_call(cache, _queries(q_len, hq, 64, dtype, 3), lens, q_len, parents, columns=columns)
