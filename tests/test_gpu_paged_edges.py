"""Calls of the operators over a paged cache at the edges of what their documentation allows."""
import random

import paged_ref as R
import pytest
import torch
from test_gpu_paged import BF, F32, _check_attention, _check_blocks, _check_eviction, _cu, _queries, _tree

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv", [(6, 2), (5, 1), (24, 1)])
def test_many_rows_of_groups_that_divide_no_power_of_two(hq, hkv):
    rng = random.Random(hq)
    q_len = [40, 60, 33]
    _check_attention([300, 70, 1000], q_len, hq, hkv, 64, BF, parents=[_tree(rng, m) for m in q_len], weigh=True)


@pytest.mark.parametrize("page", [32, 48, 112, 256])
@pytest.mark.parametrize("h", [64, 128])
def test_many_rows_over_other_pages(page, h):
    rng = random.Random(page)
    q_len = [40, 1, 128]
    _check_attention([page * 5 + 3, page, 1111], q_len, 8, 2, h, BF, parents=[_tree(rng, m, True) for m in q_len], page=page, weigh=True)


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("lo,hi", [(26, 128), (100, 300)])
def test_many_short_contexts_of_many_rows(lo, hi, h):
    """Blocks that go through many units of one or two tiles each."""
    rng = random.Random(lo + h)
    lens = [rng.randint(lo, hi) for _ in range(90)]
    q_len = [rng.randint(20, min(n, 32)) for n in lens]
    _check_attention(lens, q_len, 32, 8, h, BF, parents=[_tree(rng, m, True) for m in q_len], weigh=True)


def test_long_chains():
    _check_attention([700, 1025, 300], [300, 1, 300], 8, 2, 128, BF, weigh=True)


@pytest.mark.parametrize("m", [3, 40])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_queries_and_results_that_are_only_aligned_to_a_word(m, dtype):
    rng = random.Random(m)
    lens, q_len = [400, 90], [m, m]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype, seed=3))
    parents = torch.tensor(sum((_tree(rng, m) for _ in q_len), []), dtype=torch.int32, device="cuda")
    q = _queries(q_len, 8, 64, dtype, 4).cuda()
    want = B.attention_tree(q, k, v, table, n_kv, _cu(q_len), parents)
    words = 4 // q.element_size()

    def shifted():
        room = torch.full((2 * m * (8 * 64 + words) + words,), 9.0, dtype=dtype, device="cuda")
        return room, room[words:].view(2 * m, 8 * 64 + words)[:, :512].unflatten(1, (8, 64))

    _, sq = shifted()
    sq.copy_(q)
    room, out = shifted()
    got = B.attention_tree(sq, k, v, table, n_kv, _cu(q_len), parents, out=out)
    # another kernel may serve it: both are right within their bounds, which test_trees checks
    tol = 2.0 ** -7 if dtype is BF else 2.0 ** -18
    assert bool(((got.float() - want.float()).abs() <= tol * (1 + want.float().abs())).all())
    assert bool((room[:words] == 9).all()) and bool((room[words:].view(2 * m, -1)[:, 512:] == 9).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_where_the_scores_of_all_rows_are_too_many_to_keep(dtype):
    lens, q_len = [100, 37], [4, 2]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype, seed=6))
    q = _queries(q_len, 8, 64, dtype, 7).cuda()
    wide = torch.full((2, 300000), 1 << 30, dtype=torch.int32, device="cuda")    # 6 rows x 8 heads x 4.8 M keys
    wide[:, :table.shape[1]] = table
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    w, w_wide = (torch.zeros(k.shape[:3], device="cuda") for _ in range(2))
    out = B.attention_tree(q, k, v, table, n_kv, _cu(q_len), key_weights=w)
    out_wide = B.attention_tree(q, k, v, wide, n_kv, _cu(q_len), key_weights=w_wide, status=status)
    B.check_status(status)
    assert torch.equal(out, out_wide)
    # scores are sums of 64 products, sum |q k| <= 100 here, in either order: off by 64 * 2^-24 * 100 / 8 each, lse likewise; both
    # move a weight by 2^-13.4 of itself at most, and 32 terms are summed
    assert bool(((w - w_wide).abs() <= 2.0 ** -12 * w + 2.0 ** -30).all()) and abs(float(w.sum()) - 48) < 0.05


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pools_of_more_than_two_to_the_31_elements(dtype):
    rng = random.Random(2)
    lens, q_len, hkv, h = [300, 45], [30, 5], 8, 128
    parents = torch.tensor(sum((_tree(rng, m) for m in q_len), []), dtype=torch.int32, device="cuda")
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, hkv, h, dtype, seed=8))
    n_small, n_big = k.shape[0], 2 ** 31 // (hkv * 16 * h) + 40
    big = [torch.empty(n_big, hkv, 16, h, dtype=dtype, device="cuda") for _ in range(2)]
    for x, y in zip(big, (k, v)):
        x[-n_small:] = y
    far = torch.where((table >= 0) & (table < n_small), table + (n_big - n_small), table)
    q, q1 = _queries(q_len, 32, h, dtype, 9).cuda(), _queries([2, 1], 32, h, dtype, 10).cuda()
    w, w_far = torch.zeros(k.shape[:3], device="cuda"), torch.zeros(n_big, hkv, 16, device="cuda")
    for rows, lens_q, p in ((q, q_len, parents), (q1, [2, 1], None)):
        a = B.attention_tree(rows, k, v, table, n_kv, _cu(lens_q), p, key_weights=w)
        b = B.attention_tree(rows, *big, far, n_kv, _cu(lens_q), p, key_weights=w_far)
        assert torch.equal(a, b) and torch.equal(w, w_far[-n_small:]) and bool((w_far[:-n_small] == 0).all())
    bounds = torch.zeros(n_small, hkv, 2, h, dtype=dtype, device="cuda")
    bounds_far = torch.zeros(n_big, hkv, 2, h, dtype=dtype, device="cuda")
    B.block_bounds(k, table, n_kv, bounds)
    B.block_bounds(big[0], far, n_kv, bounds_far)
    assert torch.equal(bounds, bounds_far[-n_small:])
    assert torch.equal(B.attention_blocks(q1, k, v, bounds, table, n_kv, _cu([2, 1]), n_blocks=5),
                       B.attention_blocks(q1, *big, bounds_far, far, n_kv, _cu([2, 1]), n_blocks=5))
    B.evict_keys(k, v, w, table, n_kv, 40, n_sink=2, n_recent=8)
    B.evict_keys(*big, w_far, far, n_kv, 40, n_sink=2, n_recent=8)
    for x, y in zip(big + [w_far], (k, v, w)):
        assert torch.equal(x[-n_small:].nan_to_num(3.0), y.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_chosen_blocks_of_requests_whose_rows_overlap_are_checked(dtype):
    """Rows 4 .. 7 belong to two requests: the first one finds the choice that was made for the other, and entries of nobody."""
    lens = [2000, 500, 500, 60]
    k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, dtype, garbage=0.0))
    q = _queries([12], 8, 64, dtype, 3).cuda()
    good = B.attention_blocks(q[:8].contiguous(), k, v, *_bounds(k, table, n_kv), table[:1], n_kv[:1], _cu([8]), n_blocks=20)
    cu = torch.tensor([0, 8, 4, 4, 12], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    blocks = torch.full((12, 2, 20), 1 << 30, dtype=torch.int32, device="cuda")
    out = B.attention_blocks(q, k, v, *_bounds(k, table, n_kv), table, n_kv, cu, n_blocks=20, blocks=blocks, status=status)
    with pytest.raises(B.SledError):
        B.check_status(status)
    near = (out[:4].float() - good[:4].float()).abs() <= 2.0 ** -7 * good[:4].float().abs() + 1e-3    # the work is shared out anew
    assert bool(near.all())


def _bounds(k, table, n_kv):
    bounds = torch.zeros(k.shape[0], k.shape[1], 2, k.shape[3], dtype=k.dtype, device="cuda")
    B.block_bounds(k, table, n_kv, bounds)
    return (bounds,)


@pytest.mark.parametrize("page", [48, 112])
def test_eviction_and_bounds_of_pages_that_are_no_power_of_two(page):
    _check_eviction([page * 6 + 1, 70, page * 9, 0], 71, 3, 20, page=page, layers=3, separate=True)
    k, v, table, n_kv = R.make_cache([page * 3 + 5, page], 2, 64, BF, page, garbage=float("inf"))
    got = _bounds(k.cuda(), table.cuda(), n_kv.cuda())[0].cpu()
    for i, n in enumerate([page * 3 + 5, page]):
        for b in range((n + page - 1) // page):
            keys = k[table[i, b], :, :min(page, n - b * page)]
            assert torch.equal(got[table[i, b], :, 0], keys.amin(1)) and torch.equal(got[table[i, b], :, 1], keys.amax(1))


def test_results_in_the_place_of_the_queries_are_refused():
    k, v, table, n_kv = (t.cuda() for t in R.make_cache([30], 2, 64, BF))
    q = _queries([2], 8, 64, BF, 1).cuda()
    with pytest.raises(B.SledError) as e:
        B.attention_tree(q, k, v, table, n_kv, _cu([2]), out=q)
    assert e.value.code == B.SLED_ERR_ARG


def test_two_graphs_with_workspaces_of_their_own_replayed_at_once():
    calls = []
    for seed in (1, 2):
        rng = random.Random(seed)
        lens, q_len = [900 * seed, 200], [30, 4]
        k, v, table, n_kv = (t.cuda() for t in R.make_cache(lens, 2, 64, BF, seed=seed))
        q = _queries(q_len, 8, 64, BF, seed).cuda()
        parents = torch.tensor(sum((_tree(rng, m) for m in q_len), []), dtype=torch.int32, device="cuda")
        args = (q, k, v, table, n_kv, _cu(q_len), parents)
        w = torch.zeros(k.shape[:3], device="cuda")
        want = B.attention_tree(*args, key_weights=w)
        out = torch.empty_like(want)
        got_w = torch.zeros_like(w)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            got_w.zero_()
            B.attention_tree(*args, out=out, key_weights=got_w)
        calls.append((graph, stream, out, want, got_w, w, args))
    for _ in range(20):
        for graph, stream, out, *_ in calls:
            with torch.cuda.stream(stream):
                out.zero_()
                graph.replay()
    torch.cuda.synchronize()
    for _, _, out, want, got_w, w, _ in calls:
        assert torch.equal(out, want) and torch.equal(got_w, w)


@pytest.mark.parametrize("n_blocks", [3, 4000])
def test_blocks_with_rows_of_no_request_and_requests_of_no_rows(n_blocks):
    _check_blocks([200, 33, 0, 1], [0, 3, 0, 1], n_blocks, 2, 8, 2, 64, BF)
