"""Edges of a decoding step's operators over a caller's paged cache: units of one tile in a row."""
import math
import random

import pytest
import test_gpu_step as T
import torch

from paper_2506_09397_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


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
