"""The pages of a key-value cache (saki_cache_*): tables, lengths and counts against the integer oracle, one call at a time and in
long random sequences of calls; keys and values against copies of their own."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _same(cache, ref):
    assert cache.length.tolist() == ref.length
    assert cache.ref_count.tolist() == ref.ref
    assert cache.page_table.tolist() == ref.table


def _ref(cache):
    return O.Cache(cache.page_table.tolist(), cache.length.tolist(), cache.ref_count.tolist(), cache.page_size)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _counts(ref):
    """How often the tables hold each page."""
    got = [0] * len(ref.ref)
    for row, L in zip(ref.table, ref.length):
        for i in row[:ref.pages(L)]:
            got[i] += 1
    return got


@pytest.mark.parametrize("B,max_pages,n_pages,page", [(1, 3, 2, 1), (5, 7, 40, 4), (33, 9, 300, 16), (130, 5, 1000, 3), (1500, 3, 9000, 8)])
def test_random_sequences_of_calls(B, max_pages, n_pages, page):
    rng = np.random.default_rng(B + page)
    cache = P.PageCache.empty(B, max_pages, n_pages, page, DEV)
    ref = _ref(cache)
    for step in range(24):
        kind = rng.integers(0, 5)
        if kind <= 1:
            n = rng.integers(0, 2 * page + 1, B) if kind else np.full(B, rng.integers(0, page + 1))
            src, dst, st = P.cache_reserve(cache, _int(n) if kind else int(n[0]))
            want = ref.reserve([int(v) for v in n])
            assert [src.tolist(), dst.tolist(), st.tolist()] == [list(w) for w in want], step
        elif kind == 2:
            keep = [int(rng.integers(0, v + 1)) for v in ref.length]
            assert P.cache_truncate(cache, _int(keep)).tolist() == ref.truncate(keep)
        elif kind == 3:
            group = int(rng.integers(1, min(B, 9) + 1))
            parent = [int(v) for v in rng.integers(-1, group, B)]
            assert P.cache_fork(cache, _int(parent), group).tolist() == ref.fork(parent, group)
        else:
            src, dst, moves = P.cache_compact(cache)
            want = ref.compact()
            assert [src.tolist(), dst.tolist(), int(moves)] == list(want[:3])
        _same(cache, ref)
        assert _counts(ref) == ref.ref
    P.check()


def test_who_keeps_a_shared_last_page():
    """All holders go on: the first keeps the page.  One of them does not: all others copy.  No room for the last: it holds on."""
    page = 4
    for n_new, n_pages, expect in (([1, 1, 1], 8, [-1, 2, 3]), ([1, 0, 1], 8, [2, -1, 3]), ([1, 1, 1], 4, [2, 3, -1])):
        cache = P.PageCache.empty(3, 4, n_pages, page, DEV)
        P.cache_reserve(cache, _int([6, 0, 0]))
        P.cache_fork(cache, _int([0, 0, 0]))
        ref = _ref(cache)
        assert ref.ref[:2] == [3, 3]
        src, dst, st = P.cache_reserve(cache, _int(n_new))
        assert [src.tolist(), dst.tolist(), st.tolist()] == [list(x) for x in ref.reserve(n_new)]
        assert dst.tolist() == expect
        _same(cache, ref)
    assert P.check() == 1                       # the sequence without a page


def test_rows_that_are_flagged_stay_as_they_are():
    cache = P.PageCache.empty(6, 3, 9, 4, DEV)
    P.cache_reserve(cache, _int([5, 5, 5, 5, 0, 1]))
    P.check()
    cache.length[0], cache.length[1] = -3, 13                 # outside the table
    cache.page_table[2, 1] = 9                                # outside the pool
    ref = _ref(cache)
    src, dst, st = P.cache_reserve(cache, _int([1, 1, 1, -1, 13, 1]))
    assert [src.tolist(), dst.tolist(), st.tolist()] == [list(x) for x in ref.reserve([1, 1, 1, -1, 13, 1])]
    assert st.tolist() == [256, 256, 128, 256, 256, 0]
    _same(cache, ref)
    assert P.check() == 5
    keep = [0, 0, 1, 6, -1, 2]
    assert P.cache_truncate(cache, _int(keep)).tolist() == ref.truncate(keep) == [256, 256, 128, 256, 256, 0]
    _same(cache, ref)
    parent = [2, 6, -2, 3, 0, 5]
    assert P.cache_fork(cache, _int(parent)).tolist() == ref.fork(parent, 6)
    _same(cache, ref)
    cache.page_table[5, 0] = -7
    cache.length[3] = 1 << 30
    ref = _ref(cache)
    src, dst, moves = P.cache_compact(cache)
    want = ref.compact()
    assert [src.tolist(), dst.tolist(), int(moves)] == list(want[:3])
    _same(cache, ref)
    assert P.check() > 0


def test_commit_of_a_verified_block():
    """K + 1 positions in, the token in front of the draft and the accepted prefix stay."""
    K, page = 6, 4
    cache = P.PageCache.empty(5, 8, 64, page, DEV)
    P.cache_reserve(cache, _int([3, 4, 5, 8, 0]))
    ref = _ref(cache)
    P.cache_reserve(cache, K + 1)
    ref.reserve([K + 1] * 5)
    n_accept = [0, 6, 3, 2, 5]
    assert P.cache_truncate(cache, _int(n_accept), of=K + 1, keep_add=1).tolist() == [0] * 5
    ref.truncate([a + 1 for a in n_accept], K + 1)
    _same(cache, ref)
    assert cache.length.tolist() == [4, 11, 9, 11, 6]
    assert P.cache_truncate(cache, _int([0, 0, 0, 0, 0]), of=10).tolist() == [256, 0, 256, 0, 256]
    assert P.cache_truncate(cache, _int([2 ** 31 - 1] * 5), keep_add=2 ** 31 - 1).tolist() == [256] * 5
    P.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Q,H,D,page,head_major,odd", [(1, 1, 1, 8, 1, False, False), (3, 5, 2, 64, 4, True, False), (7, 2, 3, 36, 5, False, True),
                                                         (40, 17, 8, 128, 16, False, False)])
def test_write_and_copy(dtype, B, Q, H, D, page, head_major, odd):
    """Each position's keys and values land in its slot, and nothing else changes; pages are copied whole."""
    g = torch.Generator(device=DEV).manual_seed(B)
    n_pages = B * (-(-(Q + 9) // page)) + 3
    cache = P.PageCache.empty(B, -(-(Q + 9) // page), n_pages, page, DEV)
    P.cache_reserve(cache, torch.randint(0, 10, (B,), generator=g, device=DEV, dtype=torch.int32))
    shape = (n_pages, H, page, D) if head_major else (n_pages, page, H, D)
    pools = [torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(2)]
    kp, vp = [p.transpose(1, 2) if head_major else p for p in pools]
    wide = torch.randn((B, Q, 2, H, D + (1 if odd else 0)), generator=g, device=DEV).to(dtype)
    k, v = wide[:, :, 0, :, :D], wide[:, :, 1, :, :D]
    n_new = torch.randint(0, Q + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    _, _, st = P.cache_reserve(cache, n_new)
    assert st.tolist() == [0] * B
    want = [kp.clone(), vp.clone()]
    skip = B // 2                                    # a sequence that is passed over
    st[skip] = 512
    for b in range(B):
        n, L = int(n_new[b]), int(cache.length[b])
        for j in range(n):
            x = L - n + j
            i = int(cache.page_table[b, x // page])
            if b != skip:
                want[0][i, x % page], want[1][i, x % page] = k[b, j], v[b, j]
    P.cache_write(cache, k, v, kp, vp, st, n_new)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])
    P.cache_write(cache, k[:, :0], v[:, :0], kp, vp)
    src, dst = _int([0, n_pages, -1, 1 % n_pages]), _int([n_pages - 1, 0, 0, -5])
    P.copy_pages([kp, vp], src, dst)
    for w, p in zip(want, (kp, vp)):
        w[n_pages - 1] = w[0]
        assert torch.equal(p, w)


def test_write_passes_over_what_has_no_place():
    page, H, D = 4, 1, 8
    cache = P.PageCache.empty(5, 3, 8, page, DEV)
    P.cache_reserve(cache, _int([6, 6, 6, 6, 6]))
    P.check()
    cache.page_table[0, 1] = 8                       # outside the pool
    cache.length[1] = 13
    cache.length[2] = 1                              # fewer positions than new ones: the first ones have no place
    kp, vp = (torch.zeros(8, page, H, D, device=DEV) for _ in range(2))
    k = torch.ones(5, 2, H, D, device=DEV)
    P.cache_write(cache, k, 2 * k, kp, vp, n_new=_int([2, 2, 2, 3, -1]))
    want = torch.zeros(8, page, H, D, device=DEV)
    want[cache.page_table[2, 0], 0] = 1
    assert torch.equal(kp, want) and torch.equal(vp, 2 * want)


def test_many_pools_and_wide_strides():
    """More pools than one launch takes, pages that are views into something wider, sizes that are no multiple of 16 bytes."""
    g = torch.Generator(device=DEV).manual_seed(1)
    wide = [torch.randn((6, 2, 3, 1, 5), generator=g, device=DEV).to(torch.bfloat16) for _ in range(70)]
    pools = [w[:, 1] for w in wide]
    want = [w.clone() for w in wide]
    P.copy_pages(pools, _int([4, 0]), _int([1, 3]))
    for w, x in zip(want, wide):
        w[1, 1], w[3, 1] = w[4, 1], w[0, 1]
        assert torch.equal(w, x)


def test_offsets_beyond_32_bits():
    """Pools of more than 2^32 bytes, pages at their far end."""
    n_pages, page, H, D = 70000, 16, 8, 256            # 4.6 GB in bf16
    kp = torch.empty((n_pages, page, H, D), dtype=torch.bfloat16, device=DEV)
    cache = P.PageCache.empty(1, 2, n_pages, page, DEV)
    cache.ref_count[:n_pages - 2] = 1
    P.cache_reserve(cache, 20)
    assert cache.page_table.tolist() == [[n_pages - 2, n_pages - 1]]
    k = torch.randn(1, 20, H, D, device=DEV).to(torch.bfloat16)
    P.cache_write(cache, k, k, kp, kp)
    assert torch.equal(kp[n_pages - 2:].reshape(32, H, D)[:20], k[0])
    P.copy_pages([kp], _int([n_pages - 1]), _int([n_pages - 3]))
    assert torch.equal(kp[n_pages - 3, :4], k[0, 16:])


def test_captured_calls_replay():
    page = 4
    cache = P.PageCache.empty(4, 6, 40, page, DEV)
    P.cache_reserve(cache, 5)
    ref = _ref(cache)
    parent, keep = _int([1, 1, 0, 3]), _int([1, 2, 0, 3])
    P.cache_truncate(cache, _int([0, 0, 0, 0]), of=0)        # (the library is loaded and looked up)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.cache_fork(cache, parent)
        src, dst, st = P.cache_reserve(cache, 3)
        P.cache_truncate(cache, keep, of=3)
    for _ in range(3):
        graph.replay()
        ref.fork(parent.tolist(), 4)
        want = ref.reserve([3] * 4)
        ref.truncate(keep.tolist(), 3)
        assert [src.tolist(), dst.tolist(), st.tolist()] == [list(w) for w in want]
        _same(cache, ref)


def test_another_stream():
    """Calls on a stream of the caller's, outputs from its pool."""
    s = torch.cuda.Stream()
    cache = P.PageCache.empty(64, 8, 1000, 4, DEV)
    ref = _ref(cache)
    s.wait_stream(torch.cuda.current_stream())
    for n in (3, 5, 2):
        src, dst, st = P.cache_reserve(cache, n, stream=s)
        want = ref.reserve([n] * 64)
    s.synchronize()
    assert st.tolist() == want[2]
    _same(cache, ref)
