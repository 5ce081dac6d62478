"""Pages copied in pools of every layout that attention and cache_write take: after a fork, after compaction, and refused where elements overlap."""
import pytest
import torch

import paper_2609_36601_b200 as P
from test_gpu_attention_forms import LAYOUTS, _laid_out
from test_gpu_cache_pages import _int
from test_gpu_paged_attention import BF16, DEV, F32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("dtype,H,D,page", [(BF16, 2, 64, 16), (BF16, 1, 8, 5), (F32, 3, 36, 4), (BF16, 5, 3, 7), (F32, 1, 1, 1)])
def test_pages_are_copied_whole_and_nothing_else(how, dtype, H, D, page):
    g = torch.Generator(device=DEV).manual_seed(H + D)
    n_pages = 9
    rows = [torch.randn((n_pages, page, H, D), generator=g, device=DEV).to(dtype) for _ in range(2)]
    pools = [_laid_out(x.clone(), how) for x in rows]
    around = [torch.as_strided(p, (p.untyped_storage().nbytes() // p.element_size(),), (1,), 0) for p in pools]      # all of the memory, what lies between the pages too
    before = [a.clone() for a in around]
    src, dst = [3, 0, -1, 8, 5, 2], [1, 7, 6, 4, -1, 99]
    P.copy_pages(pools, _int(src), _int(dst))
    for x, p, a, b in zip(rows, pools, around, before):
        want = x.clone()
        for s, d in zip(src, dst):
            if 0 <= s < n_pages and 0 <= d < n_pages:
                want[d] = x[s]
        assert torch.equal(p, want)
        p.copy_(x)
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) and torch.equal(torch.isnan(a), torch.isnan(b))


@pytest.mark.parametrize("how", LAYOUTS)
def test_a_forked_cache_is_parted_and_compacted(how):
    """Sequences that share pages go their own ways, then the pages move to the front: attention sees the same in every layout."""
    B, H, D, page, n_pages = 3, 2, 64, 8, 40
    g = torch.Generator(device=DEV).manual_seed(3)
    cache = P.PageCache.empty(B, 10, n_pages, page, DEV)
    pools = [_laid_out(torch.zeros((n_pages, page, H, D), dtype=BF16, device=DEV), how) for _ in range(2)]
    k, v = (torch.randn((B, 21, H, D), generator=g, device=DEV).to(BF16) for _ in range(2))
    more = [torch.randn((B, 6, H, D), generator=g, device=DEV).to(BF16) for _ in range(2)]
    q = torch.randn((B, 1, 4, D), generator=g, device=DEV).to(BF16)
    P.cache_reserve(cache, 21)
    P.cache_write(cache, k, v, *pools)
    P.cache_fork(cache, _int([1, 1, 1]))
    src, dst, st = P.cache_reserve(cache, 6)
    assert int((src >= 0).sum()) == 2
    P.copy_pages(pools, src, dst)
    P.cache_write(cache, *more, *pools, st)
    P.cache_truncate(cache, _int([27, 0, 27]))
    for again in range(2):
        for p, old, new in zip(pools, (k, v), more):
            for b in (0, 2):
                want = torch.cat([old[1], new[b]])
                assert torch.equal(p[cache.page_table[b, :4].long()].flatten(0, 1)[:27], want)
        got = P.paged_attention(q, *pools, cache.page_table, cache.length)
        if again:
            assert all(torch.equal(a, b) for a, b in zip(got, first))
        first = got
        src, dst, moves = P.cache_compact(cache)
        P.copy_pages(pools, src, dst)
        assert again or int(moves) > 0
    assert P.check() == 0


def test_pages_whose_elements_overlap_are_refused():
    x = torch.zeros((4, 8, 1, 16), dtype=BF16, device=DEV)
    for bad in (x.expand(4, 8, 3, 16), torch.as_strided(x, (4, 3, 1, 16), (128, 8, 1, 1))):
        with pytest.raises(ValueError, match="overlap"):
            P.copy_pages([bad], _int([0]), _int([1]))
