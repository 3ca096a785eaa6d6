"""A decoding step's operators refuse what the host can see to be wrong, before any device is touched; frequencies of rotary
positions, which need no device."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2506_09397_b200 import binding as B


def _kv(**change):
    kv = B.SledPagedKv(4096, 8192, B.SLED_E4M3, 1, 10, 2, 16, 64, 256, 5, 5, 512, 3)
    for name, value in change.items():
        setattr(kv, name, value)
    return kv


def _slots(**change):
    a = dict(n_kv=4096, n_keep=0, n_new=8192, n_reqs=3, page=16, table=1 << 20, stride=5, cols=5, free=2 << 20, cap=10, n_free=3 << 20, n_kv_out=4 << 20,
             n_free_out=5 << 20, cu=6 << 20, positions=7 << 20, slots=8 << 20, rows=20, status=0)
    a.update(change)
    return B.lib().sled_page_slots(*a.values(), 0)


@pytest.mark.parametrize("change", [
    dict(n_kv=0), dict(n_new=0), dict(n_reqs=-1), dict(n_reqs=65536), dict(page=0), dict(page=-16), dict(table=0), dict(stride=4), dict(cols=-1),
    dict(free=0), dict(cap=-1), dict(n_free=0), dict(n_kv_out=0), dict(n_free_out=0), dict(cu=0), dict(rows=-1), dict(cols=1 << 28, stride=1 << 28),
    dict(n_kv=4097), dict(n_keep=2), dict(table=(1 << 20) + 2), dict(slots=(8 << 20) + 4), dict(status=3), dict(cu=(6 << 20) + 1),
    # outputs in the place of inputs or of each other
    dict(n_kv_out=4096), dict(n_kv_out=4100), dict(n_free_out=3 << 20), dict(cu=8192), dict(positions=8 << 20), dict(slots=1 << 20),
    dict(cu=2 << 20), dict(n_keep=4 << 20), dict(n_kv=1 << 20), dict(status=6 << 20)], ids=str)
def test_bad_places_are_refused(change):
    assert _slots(**change) == B.SLED_ERR_ARG


def _heads(**change):
    h = B.SledHeads(4096, 256, 64, 8192, 256, 64, 4)
    for name, value in change.items():
        setattr(h, name, value)
    return h


def _rotary(q, k=None, *, rows=3, h=64, dtype=B.SLED_F32, positions=256, freq=512, rot=64, pairs=0, amplitude=1.0, transpose=0):
    return B.lib().sled_rotary(None if q is None else C.byref(q), None if k is None else C.byref(k), rows, h, dtype, positions, freq, rot, pairs,
                               amplitude, transpose, 0)


@pytest.mark.parametrize("change", [dict(in_=0), dict(out=0), dict(in_=4098), dict(out=4097), dict(n_heads=-1), dict(n_heads=65536), dict(out_head=63),
                                    dict(out_row=255), dict(out_row=0), dict(out_head=0), dict(in_row=-1), dict(out_row=-256), dict(in_head=1 << 31),
                                    dict(out=4096, out_row=260), dict(out=4096, in_head=65)], ids=str)
def test_bad_heads_are_refused(change):
    assert _rotary(_heads(**change)) == B.SLED_ERR_ARG
    assert _rotary(_heads(), _heads(**change)) == B.SLED_ERR_ARG


@pytest.mark.parametrize("change", [dict(rows=-1), dict(h=0), dict(h=63, rot=62), dict(h=514), dict(rot=0), dict(rot=63), dict(rot=66), dict(dtype=2),
                                    dict(dtype=-1), dict(positions=0), dict(positions=258), dict(freq=0), dict(freq=516), dict(pairs=2),
                                    dict(amplitude=math.nan), dict(amplitude=math.inf), dict(rows=1 << 30)], ids=str)
def test_bad_rotations_are_refused(change):
    assert _rotary(_heads(), **change) == B.SLED_ERR_ARG
    assert _rotary(None) == B.SLED_ERR_ARG


def _append(kv, **change):
    a = dict(ks=256, vs=512, k=4096, k_stride=128, v=4096, v_stride=128, dtype=B.SLED_BF16, cu=256, rows=4, status=0)
    a.update(change)
    return B.lib().sled_append_keys(None if kv is None else C.byref(kv), *a.values(), 0)


def _attend(kv, **change):
    a = dict(ks=256, vs=512, q=4096, q_stride=256, cu=256, parents=0, rows=4, heads=4, scale=0.0, out=4096, out_stride=256, lse=0, status=0, ws=256,
             ws_bytes=1 << 60)
    a.update(change)
    return B.lib().sled_attention_scaled(None if kv is None else C.byref(kv), *a.values(), 0)


BAD_CACHES = [dict(k=0), dict(k=4100), dict(v=0), dict(v=8200), dict(dtype=3), dict(dtype=-1), dict(head_dim=96), dict(page_size=8), dict(page_size=24),
              dict(page_size=512), dict(n_layers=2), dict(n_pages=0), dict(n_kv_heads=0), dict(n_reqs=-1), dict(table_stride=4), dict(page_table=0),
              dict(n_kv=0), dict(n_pages=1 << 27), dict(table_cols=1 << 28, table_stride=1 << 28)]


@pytest.mark.parametrize("change", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(change):
    kv = _kv(**change)
    assert _append(kv) == B.SLED_ERR_ARG
    assert _attend(kv) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_scaled_workspace(C.byref(kv), 4, 4, C.byref(C.c_int64())) == B.SLED_ERR_ARG


@pytest.mark.parametrize("change", [dict(ks=0), dict(vs=0), dict(ks=258), dict(vs=3), dict(k=0), dict(v=0), dict(k=4097), dict(v=4097), dict(k_stride=127),
                                    dict(v_stride=127), dict(k_stride=1 << 50), dict(dtype=2), dict(dtype=B.SLED_F32, k=4098), dict(cu=0), dict(cu=258),
                                    dict(rows=-1), dict(status=2)], ids=str)
def test_bad_rows_of_keys_are_refused(change):
    assert _append(_kv(), **change) == B.SLED_ERR_ARG
    assert _append(None) == B.SLED_ERR_ARG


def test_scales_belong_to_caches_in_8_bits_and_rows_to_caches_of_their_type():
    for dtype in (B.SLED_F32, B.SLED_BF16):
        assert _append(_kv(dtype=dtype), dtype=dtype) == B.SLED_ERR_ARG
        assert _append(_kv(dtype=dtype), dtype=1 - dtype, ks=0, vs=0) == B.SLED_ERR_ARG
        assert _attend(_kv(dtype=dtype)) == B.SLED_ERR_ARG
    n = C.c_int64()
    for kv in (_kv(), _kv(page_size=32)):     # no other operator takes 8 bits
        assert B.lib().sled_attention_tree_workspace(C.byref(kv), 4, 4, 0, C.byref(n)) == B.SLED_ERR_ARG
        assert B.lib().sled_evict_keys_workspace(C.byref(kv), C.byref(n)) == B.SLED_ERR_ARG
        assert B.lib().sled_block_bounds(C.byref(kv), 0, 256, 0, 0) == B.SLED_ERR_ARG


@pytest.mark.parametrize("change", [dict(ks=0), dict(vs=0), dict(ks=2), dict(vs=6), dict(q=0), dict(q=4098), dict(out=0), dict(out=4098), dict(cu=0),
                                    dict(cu=257), dict(rows=-1), dict(heads=0), dict(heads=3), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                                    dict(q_stride=255), dict(q_stride=257), dict(out_stride=128), dict(out_stride=259), dict(parents=2), dict(lse=6),
                                    dict(status=1), dict(rows=1 << 30)], ids=str)
def test_bad_attention_rows_are_refused(change):
    assert _attend(_kv(), **change) == B.SLED_ERR_ARG
    assert _attend(None) == B.SLED_ERR_ARG


def test_workspaces_that_are_too_small_or_crooked_are_refused():
    n = C.c_int64(-1)
    assert B.lib().sled_attention_scaled_workspace(C.byref(_kv()), 4, 4, C.byref(n)) == B.SLED_OK and n.value >= 0
    if n.value:
        for ws, have in ((0, n.value), (256, n.value - 1), (264, n.value)):
            assert _attend(_kv(), ws=ws, ws_bytes=have) == B.SLED_ERR_ARG
    assert B.lib().sled_attention_scaled_workspace(C.byref(_kv()), 4, 4, None) == B.SLED_ERR_ARG


def test_empty_calls_need_no_device():
    assert _attend(_kv(), rows=0, q=0, out=0) == B.SLED_OK
    assert _attend(_kv(n_reqs=0)) == B.SLED_OK
    assert _attend(_kv(n_reqs=0, page_table=0, n_kv=0)) == B.SLED_OK
    assert _append(_kv(), rows=0, k=0, v=0) == B.SLED_OK
    assert _append(_kv(n_reqs=0)) == B.SLED_OK
    assert _rotary(_heads(in_=0, out=0), rows=0, positions=0) == B.SLED_OK
    assert _rotary(_heads(n_heads=0)) == B.SLED_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
def test_without_a_device_the_calls_say_so():
    assert _slots() == B.SLED_ERR_NO_DEVICE
    assert _slots(n_keep=9 << 20, positions=0, slots=0) == B.SLED_ERR_NO_DEVICE
    assert _rotary(_heads()) == B.SLED_ERR_NO_DEVICE
    assert _rotary(_heads(out=4096), _heads(n_heads=1, in_head=7, out_head=-3)) == B.SLED_ERR_NO_DEVICE     # one head: strides mean nothing
    assert _rotary(_heads(in_row=64, in_head=192, out_row=64, out_head=192)) == B.SLED_ERR_NO_DEVICE            # heads of rows
    assert _append(_kv()) == B.SLED_ERR_NO_DEVICE
    assert _attend(_kv()) == B.SLED_ERR_NO_DEVICE


def test_the_binding_refuses_tensors_of_the_host():
    i = torch.zeros(1, dtype=torch.int32)
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(4, 2, 1)
    rows = torch.zeros(1, 2, 64)
    for call in (lambda: B.page_slots(i, i, i.view(1, 1), i, i, page_size=16, n_rows=1),
                 lambda: B.rotary(rows, rows, i, torch.zeros(32, dtype=torch.float64)),
                 lambda: B.append_keys(rows, rows, k, k, i.view(1, 1), i, torch.zeros(2, dtype=torch.int32), k_scale=s, v_scale=s),
                 lambda: B.attention_tree(rows, k, k, i.view(1, 1), i, torch.zeros(2, dtype=torch.int32), k_scale=s, v_scale=s)):
        with pytest.raises(B.SledError) as e:
            call()
        assert e.value.code == B.SLED_ERR_NO_DEVICE


@pytest.mark.parametrize("number", [2 ** 32 + 16, 2 ** 31, -2 ** 31 - 1])
def test_numbers_of_more_than_32_bits_are_refused(number):
    i = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: B.page_slots(i, i, i.view(1, 1), i, i, page_size=number, n_rows=1),
                 lambda: B.page_slots(i, i, i.view(1, 1), i, i, page_size=16, n_rows=number), lambda: B.rotary_frequencies(number)):
        with pytest.raises(B.SledError) as e:
            call()
        assert e.value.code == B.SLED_ERR_ARG


# ---- frequencies
def _turns(f, length):
    return length * f / (2 * math.pi)


@pytest.mark.parametrize("d,theta", [(2, 1e4), (64, 1e4), (128, 5e5), (6, 3.5), (512, 1e6)])
def test_plain_and_linear_frequencies(d, theta):
    want = np.array([theta ** (-2 * i / d) for i in range(d // 2)])
    f, a = B.rotary_frequencies(d, theta)
    assert f.dtype is torch.float64 and f.shape == (d // 2,) and a == 1.0
    assert np.allclose(f.numpy(), want, rtol=1e-14)
    f, a = B.rotary_frequencies(d, theta, scaling=B.ROTARY_LINEAR, factor=4.0)
    assert np.allclose(f.numpy(), want / 4, rtol=1e-14) and a == 1.0


def test_a_raised_base_slows_the_lowest_frequency_by_the_factor():
    plain, _ = B.rotary_frequencies(64, 1e4)
    f, a = B.rotary_frequencies(64, 1e4, scaling=B.ROTARY_BASE, factor=8.0)
    assert f[0] == 1 and a == 1.0 and abs(f[-1] * 8 / plain[-1] - 1) < 1e-12
    r = f / plain
    assert bool((r[1:] < r[:-1]).all())


def test_bands_keep_high_frequencies_and_slow_low_ones_down():
    plain, _ = B.rotary_frequencies(128, 5e5)
    f, a = B.rotary_frequencies(128, 5e5, scaling=B.ROTARY_BANDS, factor=8.0, length=8192, low=1.0, high=4.0)
    seen = [0, 0, 0]
    for x, y in zip(plain.tolist(), f.tolist()):
        t = _turns(x, 8192)
        s = 1 if t > 4 else 0 if t < 1 else (t - 1) / 3
        seen[0 if s == 1 else 1 if s == 0 else 2] += 1
        assert abs(y / (x * (s + (1 - s) / 8)) - 1) < 1e-12
    assert a == 1.0 and min(seen) > 0


def test_a_ramp_along_the_pairs():
    d, theta, length = 128, 1e4, 4096
    plain, _ = B.rotary_frequencies(d, theta)
    f, a = B.rotary_frequencies(d, theta, scaling=B.ROTARY_RAMP, factor=16.0, length=length, low=1.0, high=32.0)
    assert abs(a - (0.1 * math.log(16) + 1)) < 1e-15
    # the pair that makes exactly 32 turns (1 turn) lies between two indices; the ramp begins (ends) at the lower (upper) one
    many, one = ([i for i in range(d // 2) if _turns(plain[i], length) >= t] for t in (32, 1))
    first, last = many[-1], one[-1] + 1
    for i, (x, y) in enumerate(zip(plain.tolist(), f.tolist())):
        s = 1 - min(max((i - first) / (last - first), 0), 1)
        assert abs(y / (x * (s + (1 - s) / 16)) - 1) < 1e-12, i
    assert B.rotary_frequencies(d, theta, scaling=B.ROTARY_RAMP, factor=0.5, length=length, high=32.0)[1] == 1.0


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=7), dict(theta=0.0), dict(theta=-1.0), dict(theta=math.nan), dict(theta=math.inf),
                                 dict(scaling=-1), dict(scaling=5), dict(scaling=1, factor=0.0), dict(scaling=1, factor=math.nan), dict(scaling=2, rot_dim=2, factor=2.0),
                                 dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, length=100.0, low=4.0, high=4.0),
                                 dict(scaling=3, factor=2.0, length=100.0, low=-1.0), dict(scaling=4, factor=2.0, length=100.0, low=0.0),
                                 dict(scaling=4, factor=2.0, length=100.0, theta=1.0), dict(scaling=4, factor=2.0, length=math.inf)], ids=str)
def test_bad_frequencies_are_refused(bad):
    a = dict(rot_dim=64, theta=1e4)
    a.update(bad)
    with pytest.raises(B.SledError) as e:
        B.rotary_frequencies(a.pop("rot_dim"), a.pop("theta"), **a)
    assert e.value.code == B.SLED_ERR_ARG
