"""Sequences that a reservation refused, in the calls that follow it in a step: what the oracle does, and what the library refuses, on the host."""
import ctypes as C

import numpy as np

import oracle as O
import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding
from test_attention_refusals import ONE, _call
from test_cache_refusals import _cache


def _full(page=4):
    """Two sequences of 12 positions in pages of 4, and one free page."""
    return O.Cache([[0, 1, 2, -1, -1], [3, 4, 5, -1, -1]], [12, 12], [1] * 6 + [0], page)


def test_a_cut_after_a_refused_reservation():
    cache = _full()
    src, dst, status = cache.reserve([5, 5])
    assert status == [512, 512] and cache.length == [12, 12]
    assert cache.truncate([2, 2], of=5, row_status=status) == [512, 512]
    assert cache.length == [12, 12] and cache.ref == [1] * 6 + [0] and cache.table == _full().table
    # ... one served, one not
    _, _, status = cache.reserve([4, 5])
    assert status == [0, 512] and cache.length == [16, 12]
    assert cache.truncate([1, 1], of=4, row_status=status) == [0, 512]
    assert cache.length == [13, 12]


def test_attention_for_a_refused_sequence():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 2, 2, 4)), rng.normal(size=(7, 4, 1, 4)), rng.normal(size=(7, 4, 1, 4))
    table = np.array(_full().table)
    a = O.paged_attention(q, k, v, table, [12, 12], 0.5)
    b = O.paged_attention(q, k, v, table, [12, 12], 0.5, row_status=[0, 512])
    assert np.array_equal(a[0][0], b[0][0]) and not b[0][1].any() and np.isneginf(b[1][1]).all() and b[2].tolist() == [0, 512]


def test_the_status_that_is_read_is_not_the_one_that_is_written():
    assert _call(row_status=ONE, scratch_bytes=1000) == 1 and "scratch" in P.last_error()          # (no status is written: nothing to clash)
    for at in (ONE, ONE + 4, ONE - 4):
        i, o = _structs()
        i.row_status, o.row_status = ONE, at
        assert binding.load_library().saki_paged_attention(C.byref(i), C.byref(o), ONE, 1 << 40, None) == 1 and "two arrays" in P.last_error()
    i, o = _structs()
    i.row_status, o.row_status = ONE, ONE + 8
    assert binding.load_library().saki_paged_attention(C.byref(i), C.byref(o), ONE, 1000, None) == 1 and "scratch" in P.last_error()
    assert binding.load_library().saki_cache_truncate(C.byref(_cache(B=0, row_status=ONE)), None, 0, -1, ONE, None) == 0


def _structs():
    i, o = binding.SakiAttnIn(), binding.SakiAttnOut()
    i.q = i.k_pages = i.v_pages = i.page_table = i.length = ONE
    i.B, i.Q, i.Hq, i.H, i.D, i.page_size, i.max_pages, i.n_pages, i.dtype, i.ld_table, i.scale = 2, 1, 8, 2, 64, 16, 4, 32, 1, 4, 0.125
    i.kp_page = i.vp_page = 16 * 2 * 64
    i.kp_pos = i.vp_pos = 2 * 64
    i.kp_head = i.vp_head = 64
    o.out = ONE
    return i, o
