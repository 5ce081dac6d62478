"""Which sequences a compaction flagged can be asked for."""
import pytest

import paper_2609_36601_b200 as P
from test_gpu_cache_pages import _int, _ref, _same
from test_gpu_paged_attention import DEV

pytestmark = pytest.mark.gpu


def test_flagged_sequences_are_named():
    P.check()
    cache = P.PageCache.empty(5, 3, 20, 4, DEV)
    P.cache_reserve(cache, _int([5, 9, 3, 12, 0]))
    P.cache_truncate(cache, _int([0, 9, 3, 12, 0]))
    cache.page_table[1, 1] = 20                               # outside the pool
    cache.length[3] = 13                                      # outside the table
    ref = _ref(cache)
    src, dst, moves, status = P.cache_compact(cache, return_status=True)
    want = ref.compact()
    assert [src.tolist(), dst.tolist(), int(moves), status.tolist()] == list(want) and status.tolist() == [0, 128, 0, 256, 0]
    _same(cache, ref)
    assert P.check() == 2
    assert len(P.cache_compact(cache)) == 3
    P.check()
