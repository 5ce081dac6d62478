"""Attention over a paged cache in the forms that decide which kernel runs and how it reads the pools: heads, rows, lengths of the tables, layouts; and the
give-up paths of its bounded waits, exercised without withholding anything (a limit of a few cycles runs out although the copies are on
their way).  Tolerances: those of test_gpu_paged_attention."""
import numpy as np
import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding
from test_gpu_paged_attention import BF16, DEV, F32, _check, _make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


# one token of few rows: heads up to 64, tables up to 256 positions, and one above; more rows, more tokens; heads at the ends of what a kernel takes
@pytest.mark.parametrize("Q,G,D,page,lengths,extra", [
    (1, 1, 8, 16, [100, 1], 3), (1, 4, 16, 8, [300, 17], 3), (1, 5, 24, 16, [129, 64], 3), (2, 5, 24, 16, [129, 2], 3),
    (1, 16, 64, 32, [700, 33], 3), (1, 17, 64, 32, [700, 33], 3), (1, 4, 128, 16, [200, 16], 3), (1, 4, 128, 16, [256, 240], 0), (1, 4, 128, 16, [257, 1], 0),
    (1, 16, 96, 8, [130, 9], 0), (1, 17, 96, 8, [130, 9], 0), (1, 33, 72, 24, [100, 50], 0), (2, 17, 128, 16, [400, 128], 0), (5, 13, 128, 16, [128, 129], 0),
    (32, 4, 64, 8, [300, 40], 0), (3, 20, 40, 8, [65, 3], 0)])
def test_heads_rows_and_tables(Q, G, D, page, lengths, extra):
    _check(*_make(len(lengths), Q, 2, G, D, page, lengths, BF16, Q + G + D, extra=extra, fill=float("nan")))


@pytest.mark.parametrize("window", [1, 200, 255, 256, 257])
def test_windows_beside_the_choice_of_a_kernel(window):
    args = _make(3, 1, 2, 4, 128, 16, [1500, 90, 700], BF16, window)
    _check(*args, window=window)
    _check(*args, window=window, sinks=20)


@pytest.mark.parametrize("D", [4, 12, 64, 68, 80, 96, 100, 128, 192])
@pytest.mark.parametrize("G,Q", [(3, 3), (4, 5), (9, 7)])
def test_f32_heads(D, G, Q):
    for page in (24, 5):
        _check(*_make(2, Q, 1, G, D, page, [211, Q], F32, D + G, fill=float("inf")))


def _laid_out(x, how):
    """x [n_pages, page, H, D], the same numbers in another order of memory."""
    n, page, H, D = x.shape
    if how == "pages":
        return x
    if how == "heads first":
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    if how == "heads outermost":
        return x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    if how == "heads outermost, pages apart":
        wide = torch.full((H, n, page + 8, D), float("nan"), dtype=x.dtype, device=x.device)
        wide[:, :, :page] = x.permute(2, 0, 1, 3)
        return wide[:, :, :page].permute(1, 2, 0, 3)
    if how == "heads apart":
        wide = torch.full((n, page, 2 * H, D), float("nan"), dtype=x.dtype, device=x.device)
        wide[:, :, ::2] = x
        return wide[:, :, ::2]
    if how == "rows apart":
        wide = torch.full((n, page, H, D + 8), float("nan"), dtype=x.dtype, device=x.device)
        wide[..., :D] = x
        return wide[..., :D]
    pos = torch.full((page, n, H, D), float("nan"), dtype=x.dtype, device=x.device)      # "positions outermost"
    pos[:] = x.permute(1, 0, 2, 3)
    return pos.permute(1, 0, 2, 3)


LAYOUTS = ["pages", "heads first", "heads outermost", "heads outermost, pages apart", "heads apart", "rows apart", "positions outermost"]


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("dtype,H,Q,D,page", [(BF16, 2, 1, 128, 16), (BF16, 1, 3, 128, 16), (BF16, 3, 3, 128, 8), (BF16, 3, 2, 128, 136), (BF16, 2, 1, 64, 16), (BF16, 2, 4, 80, 24), (F32, 2, 2, 80, 24)])
def test_layouts_of_the_pools(how, dtype, H, Q, D, page):
    q, k, v, table, length = _make(2, Q, H, 3, D, page, [400, 131], dtype, H + Q + D)
    a = _check(q, _laid_out(k, how), _laid_out(v, how), table, length)
    for other in ("pages", "heads first"):
        b = P.paged_attention(q, _laid_out(k, how), _laid_out(v, other), table, length)
        assert all(torch.equal(x, y) for x, y in zip(a, b))      # where the numbers lie does not change what is made of them


@pytest.mark.parametrize("dtype,Q,G,D,page", [(BF16, 1, 4, 128, 16), (BF16, 3, 4, 128, 16), (BF16, 7, 9, 64, 16), (BF16, 1, 4, 64, 16), (BF16, 1, 2, 256, 16),
                                              (BF16, 5, 9, 256, 16), (BF16, 4, 5, 128, 5), (F32, 3, 3, 80, 24), (F32, 9, 8, 64, 8)])
def test_expired_waits_flag_sequences_and_leave_the_library_usable(dtype, Q, G, D, page):
    lengths = [3000, Q, 700, 20000, 129, 4000]
    q, k, v, table, length = _make(6, Q, 2, G, D, page, lengths, dtype, Q + G + D, fill=float("nan"))
    P.check()
    want = P.paged_attention(q, k, v, table, length)
    torch.cuda.synchronize()
    assert P.check() == 0
    flush = torch.empty(320 << 20, dtype=torch.uint8, device=DEV)
    try:
        for limit in (2, 300, 3000):
            flush.fill_(1)
            torch.cuda.synchronize()
            assert P.set_wait_limit(limit) == 0
            out, lse, st = P.paged_attention(q, k, v, table, length)
            assert P.set_wait_limit(0) == limit
            flagged = P.check()                                 # synchronises: the kernels came back
            st = st.cpu().numpy().astype(np.uint32)
            assert np.all((st == 0) | (st == binding.ROW_TIMEOUT)) and flagged == int((st != 0).sum())
            assert limit > 2 or st.any(), "no wait ran out: the limit did not reach the kernel"
            for b in range(6):                                  # a head is right, or it was late and the sequence says so
                for h in range(2 * G):
                    for j in range(Q):
                        late = bool(torch.isneginf(lse[b, j, h]))
                        assert not late or st[b] != 0
                        x = torch.zeros_like(out[b, j, h]) if late else want[0][b, j, h]
                        assert torch.equal(out[b, j, h], x), (limit, b, j, h)
            again = P.paged_attention(q, k, v, table, length)
            assert P.check() == 0 and all(torch.equal(x, y) for x, y in zip(again, want))
    finally:
        P.set_wait_limit(0)


def test_two_streams_at_once_and_two_captured_calls():
    """Calls that run at the same time, and graphs whose replays follow one another in any order, do not share what they work in."""
    a = _make(8, 1, 2, 4, 128, 16, [9000, 1, 300, 128, 2000, 64, 65, 5000], BF16, 3)
    b = _make(4, 5, 2, 3, 64, 8, [700, 5, 4000, 130], BF16, 4)
    want = [P.paged_attention(*x) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, x in enumerate((a, b)):
            got[i].append(P.paged_attention(*x, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, y) for g in got[i] for x, y in zip(g, want[i]))
    graphs, outs = [], []
    for x in (a, b, a):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(P.paged_attention(*x))
        graphs.append(g)
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0)):
        for o in outs:
            for t in o:
                t.fill_(0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(order):
            assert all(torch.equal(x, y) for x, y in zip(outs[i], want[i % 2]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Q,G,D,page,lengths", [(1, 4, 128, 128, [500, 128]), (3, 4, 128, 256, [300, 700]), (2, 2, 64, 1000, [1500, 2]), (1, 2, 64, 4096, [5000, 4096]),
                                                (32, 64, 64, 16, [200, 32]), (32, 64, 128, 12, [70, 33])])
def test_large_pages_and_many_rows(dtype, Q, G, D, page, lengths):
    _check(*_make(2, Q, 1, G, D, page, lengths, dtype, Q + G + page, extra=1, fill=float("nan")))


@pytest.mark.parametrize("dtype,Q,D,page", [(BF16, 2, 128, 16), (BF16, 1, 128, 16), (BF16, 1, 64, 16), (BF16, 3, 64, 5), (F32, 2, 64, 16)])
@pytest.mark.parametrize("size", [1e10, 1e15, 1e17])
def test_scores_far_below_zero(dtype, Q, D, page, size):
    """Scores of -1e21 to -1e35, the same at all positions: the mean of the values, whatever the maximum was taken to be at first."""
    n = 700
    q, k, v, table, length = _make(2, Q, 2, 2, D, page, [n, 40], dtype, 5)
    q.fill_(size)
    k.fill_(-size)
    out, lse, st = P.paged_attention(q, k, v, table, length)
    assert int(st.abs().max()) == 0 and torch.isfinite(lse).all()
    for b in range(2):
        pages = table[b, :-(-int(length[b]) // page)].long()
        vb = v[pages].flatten(0, 1).double()
        for j in range(Q):
            m = int(length[b]) - Q + j + 1
            want = vb[:m].mean(0).repeat_interleave(2, 0)
            size_v = vb[:m].abs().mean(0).repeat_interleave(2, 0)
            half = torch.finfo(dtype).eps / 2
            # equal weights of 1 (exact in two terms), a sum of m values, one division, one rounding
            assert ((out[b, j].double() - want).abs() <= half * want.abs() + (m + 4) * 2.0 ** -23 * size_v).all()
