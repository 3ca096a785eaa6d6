"""The operators over a paged cache refuse what the host can see to be wrong, before any device is touched."""
import ctypes as C

import pytest
import torch

from paper_2506_09397_b200 import binding as B


def _kv(**change):
    kv = B.SledPagedKv(4096, 8192, B.SLED_BF16, 1, 10, 2, 16, 64, 256, 5, 5, 512, 3)
    for name, value in change.items():
        setattr(kv, name, value)
    return kv


def _tree(kv, *, q=4096, q_stride=256, cu=256, parents=0, rows=4, heads=4, scale=0.0, out=4096, out_stride=256, lse=0, weights=0,
          status=0, ws=0, ws_bytes=0):
    return B.lib().sled_attention_tree(C.byref(kv) if kv else None, q, q_stride, cu, parents, rows, heads, scale, out, out_stride,
                                       lse, weights, status, ws, ws_bytes, 0)


def _bytes(what, *args):
    n = C.c_int64(-1)
    assert getattr(B.lib(), what + "_workspace")(*args, C.byref(n)) == B.SLED_OK
    return n.value


BAD_CACHES = [dict(k=0), dict(k=4100), dict(v=8200), dict(dtype=2), dict(head_dim=96), dict(head_dim=0), dict(page_size=8),
              dict(page_size=24), dict(page_size=512), dict(page_size=0), dict(n_layers=0), dict(n_pages=0), dict(n_kv_heads=0),
              dict(n_reqs=-1), dict(table_cols=-1), dict(table_stride=4), dict(page_table=0), dict(n_kv=0), dict(n_kv=513),
              dict(n_pages=1 << 27), dict(table_cols=1 << 28, table_stride=1 << 28)]


@pytest.mark.parametrize("change", BAD_CACHES, ids=str)
def test_bad_caches_are_refused_by_every_operator(change):
    kv = _kv(**change)
    assert _tree(kv, ws=256, ws_bytes=1 << 60) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_tree_workspace(C.byref(kv), 4, 4, 0, C.byref(C.c_int64())) == B.SLED_ERR_ARG
    assert B.lib().sled_evict_keys(C.byref(kv), 256, 256, 32, 1, 1, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG
    assert B.lib().sled_evict_keys_workspace(C.byref(kv), C.byref(C.c_int64())) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_blocks(C.byref(kv), 256, 4096, 256, 256, 4, 4, 0.0, 4, 1, 4096, 256, 0, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_blocks_workspace(C.byref(kv), 4, 4, 4, C.byref(C.c_int64())) == B.SLED_ERR_ARG
    if "v" not in change:
        assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_ERR_ARG


def test_null_descriptions_are_refused():
    assert _tree(None) == B.SLED_ERR_ARG
    assert B.lib().sled_evict_keys(None, 256, 256, 32, 1, 1, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG
    assert B.lib().sled_block_bounds(None, 0, 256, 0, 0) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_blocks(None, 256, 4096, 256, 256, 4, 4, 0.0, 4, 1, 4096, 256, 0, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG


@pytest.mark.parametrize("change", [dict(q=0), dict(q=4097), dict(q=4098), dict(out=0), dict(out=4098), dict(cu=0), dict(cu=257),
                                    dict(rows=-1), dict(heads=0), dict(heads=3), dict(scale=-1.0), dict(scale=float("nan")),
                                    dict(scale=float("inf")), dict(q_stride=255), dict(q_stride=257), dict(out_stride=128),
                                    dict(out_stride=259), dict(parents=2), dict(lse=6), dict(weights=7), dict(status=1)], ids=str)
def test_bad_rows_are_refused(change):
    assert _tree(_kv(), **{**dict(ws=256, ws_bytes=1 << 60), **change}) == B.SLED_ERR_ARG


def test_a_layer_dimension_is_refused_where_it_means_nothing():
    kv = _kv(n_layers=2)
    assert _tree(kv, ws=256, ws_bytes=1 << 60) == B.SLED_ERR_ARG
    assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_blocks(C.byref(kv), 256, 4096, 256, 256, 4, 4, 0.0, 4, 1, 4096, 256, 0, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG
    assert _bytes("sled_evict_keys", C.byref(kv)) > 0


@pytest.mark.parametrize("budget,sink,recent,w,w_out", [(0, 0, 0, 256, 256), (-5, 0, 0, 256, 256), (8, -1, 0, 256, 256), (8, 0, -1, 256, 256),
                                                        (8, 5, 4, 256, 256), (8, 2147483647, 2147483647, 256, 256), (8, 1, 1, 0, 256),
                                                        (8, 1, 1, 256, 0), (8, 1, 1, 258, 258), (8, 1, 1, 256, 260), (8, 1, 1, 4096, 3840)])
def test_bad_evictions_are_refused(budget, sink, recent, w, w_out):
    # the last two: weights that overlap without being the same array
    assert B.lib().sled_evict_keys(C.byref(_kv()), w, w_out, budget, sink, recent, 0, 256, 1 << 60, 0) == B.SLED_ERR_ARG


@pytest.mark.parametrize("n_blocks,n_local,bounds,blocks", [(0, 1, 256, 0), (4, 0, 256, 0), (4, 5, 256, 0), (4, -1, 256, 0), (4, 1, 0, 0),
                                                            (4, 1, 264, 0), (4, 1, 256, 3)])
def test_bad_block_choices_are_refused(n_blocks, n_local, bounds, blocks):
    assert B.lib().sled_attention_blocks(C.byref(_kv()), bounds, 4096, 256, 256, 4, 4, 0.0, n_blocks, n_local, 4096, 256, blocks, 0, 256,
                                         1 << 60, 0) == B.SLED_ERR_ARG


def test_workspaces_that_are_too_small_or_crooked_are_refused():
    kv = _kv()
    need = _bytes("sled_attention_tree", C.byref(kv), 4, 4, 1)
    assert need > 0
    for ws, have in ((0, need), (256, need - 1), (264, need)):
        assert _tree(kv, weights=256, ws=ws, ws_bytes=have) == B.SLED_ERR_ARG
    need = _bytes("sled_evict_keys", C.byref(kv))
    for ws, have in ((0, need), (256, need - 1), (264, need)):
        assert B.lib().sled_evict_keys(C.byref(kv), 256, 256, 32, 1, 1, 0, ws, have, 0) == B.SLED_ERR_ARG
    need = _bytes("sled_attention_blocks", C.byref(kv), 4, 4, 4)
    for ws, have in ((0, need), (256, need - 1), (264, need)):
        assert B.lib().sled_attention_blocks(C.byref(kv), 256, 4096, 256, 256, 4, 4, 0.0, 4, 1, 4096, 256, 0, 0, ws, have, 0) == B.SLED_ERR_ARG


def test_empty_calls_need_no_device():
    kv = _kv()
    assert _tree(kv, rows=0, q=0, out=0, ws=256, ws_bytes=1 << 60) == B.SLED_OK
    assert _tree(_kv(n_reqs=0), ws=256, ws_bytes=1 << 60) == B.SLED_OK
    assert B.lib().sled_block_bounds(C.byref(_kv(table_cols=0)), 0, 256, 0, 0) == B.SLED_OK
    assert B.lib().sled_evict_keys(C.byref(_kv(n_reqs=0)), 256, 256, 32, 1, 1, 0, 0, 0, 0) == B.SLED_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
def test_without_a_device_the_calls_say_so():
    assert _tree(_kv(), ws=256, ws_bytes=1 << 60) == B.SLED_ERR_NO_DEVICE
    assert B.lib().sled_block_bounds(C.byref(_kv()), 0, 256, 0, 0) == B.SLED_ERR_NO_DEVICE


def test_the_binding_refuses_tensors_of_the_host():
    k = torch.zeros(4, 2, 16, 64)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(B.SledError) as e:
        B.block_bounds(k, i.view(1, 1), i, torch.zeros(4, 2, 2, 64))
    assert e.value.code == B.SLED_ERR_NO_DEVICE


def test_sizes_beyond_any_memory_are_refused_and_do_not_wrap_around():
    n = C.c_int64(-7)
    many = _kv(n_pages=1, n_kv_heads=65535, n_reqs=65535, table_cols=(1 << 27) - 128, table_stride=1 << 27)
    assert B.lib().sled_attention_blocks_workspace(C.byref(many), 2 ** 31 - 1, 65535, 2 ** 31 - 1, C.byref(n)) == B.SLED_ERR_ARG
    assert B.lib().sled_evict_keys_workspace(C.byref(_kv(n_layers=65535, n_pages=1, n_kv_heads=65535, n_reqs=65535, table_cols=(1 << 27) - 128,
                                                         table_stride=1 << 27)), C.byref(n)) == B.SLED_ERR_ARG
    assert n.value == -7
    assert B.lib().sled_evict_keys(C.byref(_kv(n_layers=65535, n_pages=1, n_kv_heads=65535, n_reqs=65535, table_cols=(1 << 27) - 128,
                                               table_stride=1 << 27)), 256, 256, 32, 1, 1, 0, 256, 2 ** 63 - 1, 0) == B.SLED_ERR_ARG
    # scores of this many (row, key) pairs are not kept: the workspace stays small
    assert _bytes("sled_attention_tree", C.byref(many), 2 ** 31 - 1, 1, 1) < 1 << 36
    # (row, head) pairs and the keys of a request are counted in 32 bits
    assert _tree(_kv(n_kv_heads=1), rows=2 ** 30, heads=4, ws=256, ws_bytes=1 << 60) == B.SLED_ERR_ARG
    assert _tree(_kv(table_cols=(1 << 27) - 1, table_stride=1 << 27), ws=256, ws_bytes=1 << 60) == B.SLED_ERR_ARG
