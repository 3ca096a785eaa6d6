"""Arguments of the operators over a paged cache: calls that have nothing to do need no arrays, numbers of more than 32 bits do
not arrive as smaller ones."""
import ctypes as C

import pytest
import torch

from paper_2506_09397_b200 import binding as B


@pytest.mark.parametrize("n_reqs,table_cols,page_table,n_kv", [(0, 5, 0, 0), (0, 0, 0, 0), (0, 5, 256, 0)])
def test_a_batch_of_no_requests(n_reqs, table_cols, page_table, n_kv):
    kv = B.SledPagedKv(4096, 8192, B.SLED_BF16, 1, 10, 2, 16, 64, page_table, table_cols, table_cols, n_kv, n_reqs)
    n = C.c_int64(-1)
    assert B.lib().sled_attention_tree_workspace(C.byref(kv), 4, 4, 1, C.byref(n)) == B.SLED_OK and n.value >= 0
    for rows, q in ((0, 0), (4, 4096)):
        assert B.lib().sled_attention_tree(C.byref(kv), q, 256, 256, 0, rows, 4, 0.0, q, 256, 0, 0, 0, 256, 1 << 60, 0) == B.SLED_OK
        assert B.lib().sled_attention_blocks(C.byref(kv), 256, q, 256, 256, rows, 4, 0.0, 4, 1, q, 256, 0, 0, 256, 1 << 60, 0) == B.SLED_OK
    assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_OK
    assert B.lib().sled_evict_keys(C.byref(kv), 256, 256, 32, 1, 1, 0, 0, 0, 0) == B.SLED_OK


def test_requests_without_keys_need_no_table():
    kv = B.SledPagedKv(4096, 8192, B.SLED_BF16, 1, 10, 2, 16, 64, 0, 0, 0, 512, 3)
    assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_OK
    assert B.lib().sled_evict_keys(C.byref(kv), 256, 256, 32, 1, 1, 0, 0, 0, 0) == B.SLED_OK
    kv.n_kv = 0                                             # but their lengths are looked at
    assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_ERR_ARG


@pytest.mark.parametrize("number", [2 ** 32 + 8, 2 ** 31, -2 ** 31 - 1, 2 ** 63 - 1])
def test_numbers_of_more_than_32_bits_are_refused(number):
    k = torch.zeros(4, 2, 16, 64)
    i = torch.zeros(1, dtype=torch.int32)
    evict = lambda **n: B.evict_keys(k, k, k[..., 0], i.view(1, 1), i, **{**dict(budget=8), **n})
    blocks = lambda **n: B.attention_blocks(k[0], k, k, k, i.view(1, 1), i, i, **{**dict(n_blocks=8), **n})
    for call in (lambda: evict(budget=number), lambda: evict(n_sink=number), lambda: evict(n_recent=number),
                 lambda: blocks(n_blocks=number), lambda: blocks(n_local=number)):
        with pytest.raises(B.SledError) as e:
            call()
        assert e.value.code == B.SLED_ERR_ARG
    with pytest.raises(B.SledError) as e:
        evict()
    assert e.value.code == B.SLED_ERR_NO_DEVICE
