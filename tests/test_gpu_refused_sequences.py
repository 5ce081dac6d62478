"""Decoding steps on a pool without room for all sequences: those that cache_reserve refuses keep what was committed, through writing, attention and the
cut of the verified block; eager, and as one captured step that is replayed.  Tables against the integer oracle, attention against the float64 one
(tolerances: those of test_gpu_paged_attention, at its _check), refused rows exact."""
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding
from test_gpu_cache_pages import _int, _ref, _same
from test_gpu_paged_attention import BF16, DEV, F32, _check, _make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


@pytest.mark.parametrize("dtype,D,captured", [(BF16, 128, False), (BF16, 128, True), (BF16, 64, False), (F32, 32, False), (F32, 32, True)])
def test_a_step_with_a_full_pool(dtype, D, captured):
    B, K, page, H, G, max_pages, n_pages = 7, 4, 4, 2, 3, 12, 30
    g = torch.Generator(device=DEV).manual_seed(D)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
    cache = P.PageCache.empty(B, max_pages, n_pages, page, DEV)
    kp, vp = r(n_pages, page, H, D), r(n_pages, page, H, D)
    P.cache_reserve(cache, _int([12, 12, 16, 3, 0, 9, 7]))
    k, v, q = r(B, K + 1, H, D), r(B, K + 1, H, D), r(B, K + 1, H * G, D)
    n_accept = torch.zeros(B, dtype=torch.int32, device=DEV)

    def step():
        src, dst, st = P.cache_reserve(cache, K + 1)
        P.copy_pages([kp, vp], src, dst)
        P.cache_write(cache, k, v, kp, vp, st)
        table, length = cache.page_table.clone(), cache.length.clone()
        got = P.paged_attention(q, kp, vp, cache.page_table, cache.length, row_status=st)
        kept = P.cache_truncate(cache, n_accept, of=K + 1, keep_add=1, row_status=st)
        return st, table, length, got, kept

    graph = None
    if captured:
        before, pools = cache.meta.clone(), (kp.clone(), vp.clone())
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = step()
        cache.meta.copy_(before); kp.copy_(pools[0]); vp.copy_(pools[1])
        P.check()
    ref = _ref(cache)
    refused = 0
    for i in range(8):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        n_accept.copy_(torch.randint(0, K + 1, (B,), generator=g, device=DEV))
        pools = kp.clone(), vp.clone()
        if captured:
            graph.replay()
            st, table, length, got, kept = result
        else:
            st, table, length, got, kept = step()
        want = ref.reserve([K + 1] * B)
        assert st.tolist() == want[2]
        assert length.tolist() == ref.length and table.tolist() == ref.table
        for b in range(B):                                     # what the sequences before the block held is as it was, a refused sequence's altogether
            n = ref.length[b] - (0 if want[2][b] else K + 1)
            for x in range(n):
                at = ref.table[b][x // page], x % page
                assert torch.equal(kp[at], pools[0][at]) and torch.equal(vp[at], pools[1][at])
        keep = (st == 0)
        some = torch.nonzero(keep).flatten()
        if len(some):
            _check(q[some], kp, vp, table[some], length[some], got=[t[some] for t in got])
        gone = ~keep
        assert not got[0][gone].any() and torch.isneginf(got[1][gone]).all() and torch.equal(got[2], st)
        assert kept.tolist() == ref.truncate([a + 1 for a in n_accept.tolist()], K + 1, want[2])
        _same(cache, ref)
        n = int(gone.sum())
        refused += n
        # (a sequence that grew out of its table is refused as well; both count once in a step)
        assert P.check() == n
        if i == 4:                                             # one sequence ends: its pages serve the others
            ends = [0 if b == 2 else n for b, n in enumerate(ref.length)]
            P.cache_truncate(cache, _int(ends))
            ref.truncate(ends)
            _same(cache, ref)
    assert refused > 0


@pytest.mark.parametrize("dtype,Q,G,D,page", [(BF16, 1, 4, 128, 16), (BF16, 5, 4, 128, 16), (BF16, 1, 2, 64, 16), (BF16, 3, 2, 256, 16), (F32, 3, 2, 80, 16)])
def test_attention_passes_over_refused_sequences(dtype, Q, G, D, page):
    """Long refused sequences between short ones; lengths and pages of refused ones are not looked at."""
    lengths = [9000, 40, 300, 20000, Q, 129, 700]
    q, k, v, table, length = _make(7, Q, 2, G, D, page, lengths, dtype, Q + D)
    want = P.paged_attention(q, k, v, table, length)
    for st in ([0] * 7, [512, 0, 0, 256, 0, 128, 0], [512] * 7, [0, 0, 0, 0, 0, 0, 1 << 20]):
        bad = [b for b in range(7) if st[b]]
        t, n = table.clone(), length.clone()
        for b in bad:
            t[b], n[b] = -1, (1 << 30) if b % 2 else -5
        P.check()
        out, lse, got = P.paged_attention(q, k, v, t, n, row_status=_int(st))
        assert got.tolist() == st and P.check() == 0
        for b in range(7):
            if st[b]:
                assert not out[b].any() and torch.isneginf(lse[b]).all()
            else:
                # (cuts fall elsewhere: the same sums in another order)
                assert torch.allclose(lse[b], want[1][b], rtol=2.0 ** -20, atol=2.0 ** -20)
        ok = [b for b in range(7) if not st[b] and lengths[b] < 1000]
        if ok:
            _check(q[ok], k, v, table[ok], length[ok], got=[x[ok] for x in (out, lse, got)])


def test_the_cut_passes_over_refused_sequences():
    cache = P.PageCache.empty(5, 4, 20, 4, DEV)
    P.cache_reserve(cache, _int([6, 7, 8, 9, 0]))
    ref = _ref(cache)
    st = [0, 512, 0, 128, 256]
    assert P.cache_truncate(cache, _int([1, 1, 9, 1, 7]), of=3, row_status=_int(st)).tolist() == ref.truncate([1, 1, 9, 1, 7], 3, st) == [0, 512, 256, 128, 256]
    _same(cache, ref)
    assert P.check() == 1                                      # the one that was not refused before
    with pytest.raises(ValueError):
        P.cache_truncate(cache, _int([0] * 5), row_status=_int([0] * 4))
    with pytest.raises(ValueError):
        P.cache_truncate(cache, _int([0] * 5), row_status=torch.zeros(5, device=DEV))
    q, k, v, table, length = _make(2, 1, 1, 2, 64, 16, [20, 30], BF16, 1)
    with pytest.raises(ValueError):
        P.paged_attention(q, k, v, table, length, row_status=_int([0]))
    # in C the status that is read may be the one that is written
    import ctypes as C
    both = _int(st)
    c = binding.SakiCache()
    c.page_table, c.length, c.ref_count = cache.page_table.data_ptr(), cache.length.data_ptr(), cache.ref_count.data_ptr()
    c.B, c.max_pages, c.n_pages, c.page_size, c.ld_table, c.row_status = 5, 4, 20, 4, 4, both.data_ptr()
    keep = _int([0] * 5)
    torch.cuda.synchronize()
    assert binding.load_library().saki_cache_truncate(C.byref(c), keep.data_ptr(), 0, -1, both.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert both.tolist() == st and ref.truncate([0] * 5, None, st) == st
    _same(cache, ref)
