"""Attention over a paged cache with scores so large that the rounding of a score times log2(e) is no small thing: equal scores weigh the same in
every tile, piece and window, and scores that are apart by a little weigh what they should.

The numbers are chosen so that scores are exact in float32 (integers below 2^24 times a power of two, or the same number everywhere)."""
import numpy as np
import pytest
import torch

import paper_2609_36601_b200 as P
from test_gpu_paged_attention import BF16, DEV, F32, _make

pytestmark = pytest.mark.gpu
FORMS = [(BF16, 2, 128, 16), (BF16, 1, 128, 16), (BF16, 1, 64, 16), (BF16, 3, 64, 5), (BF16, 7, 64, 16), (F32, 2, 64, 16)]


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


def _rows(table, v, b, n, page):
    return v[table[b, :-(-n // page)].long()].flatten(0, 1)[:n].double()


@pytest.mark.parametrize("dtype,Q,D,page", FORMS)
@pytest.mark.parametrize("size", [300, 1000, 1500, 2000, 3000, 5000, 20000, 1e6])
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_scores(dtype, Q, D, page, size, sign):
    """The mean of the values that are seen, whatever the maximum was taken to be: over a window whose first tile is cut, over sequences whose last tile is a
    piece of its own, over short ones."""
    lengths = [700, 40, 129, 6000, 257, 1025]
    q, k, v, table, length = _make(6, Q, 2, 2, D, page, lengths, dtype, 5)
    q.fill_(size)
    k.fill_(sign * size)
    half = torch.finfo(dtype).eps / 2
    for window in (0, 130, 450):
        out, lse, st = P.paged_attention(q, k, v, table, length, window=window)
        assert int(st.abs().max()) == 0 and torch.isfinite(lse).all()
        for b, n in enumerate(lengths):
            vb = _rows(table, v, b, n, page)
            for j in range(Q):
                m = n - Q + j + 1
                lo = max(0, m - window) if window else 0
                want, size_v = vb[lo:m].mean(0).repeat_interleave(2, 0), vb[lo:m].abs().mean(0).repeat_interleave(2, 0)
                # equal weights, 2^-16 off in two bf16 terms (numerator and denominator); a power of two, 2^-22 off, wherever sums are brought to a new maximum;
                # a sum of m - lo values, one division, one rounding
                share = (2 * 2.0 ** -16 if dtype == BF16 else 2.0 ** -20) + 2.0 ** -20 + (m - lo + 4) * 2.0 ** -23
                err = (out[b, j].double() - want).abs()
                assert bool((err <= half * (1 + share) * want.abs() + share * size_v).all()), (window, b, j, float((err / size_v).max()))


@pytest.mark.parametrize("dtype,Q,D,page", FORMS)
@pytest.mark.parametrize("first,second", [(0, 8), (8, 0), (0, 3), (3, 0)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_that_are_close(dtype, Q, D, page, first, second, sign):
    """Two scores of some 2^23, `first` or `second` above: runs of one and the other, of 200 positions each.  With a scale of 1 / 8 they lie some 2^20 from 0, where
    a unit in the last place (an eighth) is 9 % of a weight, and e^1 or e^0.375 apart."""
    lengths = [700, 40, 6000, 1025]
    q, k, v, table, length = _make(4, Q, 2, 2, D, page, lengths, dtype, 6)
    q.zero_(); k.zero_()
    q[..., :32], q[..., 32] = 64.0, 1.0
    k[..., :31], k[..., 31] = sign * 4096.0, sign * 4032.0           # 64 (31 x 4096 + 4032): 2^23 - 4096
    for b, n in enumerate(lengths):
        for x in range(n):
            k[int(table[b, x // page]), x % page, :, 32] = float(second if (x // 200) % 2 else first)
    base = sign * 64 * (31 * 4096 + 4032)
    assert abs(base) + 8 < 2 ** 23
    out, lse, st = P.paged_attention(q, k, v, table, length, scale=0.125)
    assert int(st.abs().max()) == 0
    half = torch.finfo(dtype).eps / 2
    for b, n in enumerate(lengths):
        vb = _rows(table, v, b, n, page)
        s = torch.tensor([float(second if (x // 200) % 2 else first) for x in range(n)], dtype=torch.float64, device=DEV) / 8
        for j in range(Q):
            m = n - Q + j + 1
            w = torch.softmax(s[:m], 0)
            want = torch.einsum("x,xhd->hd", w, vb[:m]).repeat_interleave(2, 0)
            size = torch.einsum("x,xhd->hd", w, vb[:m].abs()).repeat_interleave(2, 0)
            # exponents: two scores are at most 8 / 8 log2(e) apart, times a constant rounded by 2^-24 of itself, rounded once more; the maxima's difference is exact.  The rest as above
            share = 2 * (2.0 ** -21 + (2.0 ** -16 if dtype == BF16 else 0)) + 2.0 ** -20 + (m + 4) * 2.0 ** -23
            err = (out[b, j].double() - want).abs()
            assert bool((err <= half * (1 + share) * want.abs() + share * size).all()), (b, j, float((err / size).max()))
            ll = base / 8 + float(torch.logsumexp(s[:m], 0))
            # the constant's rounding and the result's own, of 2^20; what the maximum's rounding took away is in the sum
            assert abs(float(lse[b, j, 0]) - ll) <= 3 * 2.0 ** -24 * abs(ll) + 2.0 ** -3


@pytest.mark.parametrize("dtype,Q,D,page", FORMS)
@pytest.mark.parametrize("scale", [1.0, 2.0, 4.0, 8.0])
@pytest.mark.parametrize("first,second", [(0, 1), (1, 0)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_a_step_apart(dtype, Q, D, page, scale, first, second, sign):
    """Scores of some 2^23 that are a unit, their own last place, apart: times 1 to 8 they lie up to 2^26 from 0, where float32 numbers are 8 apart, and weigh 2.7 to 3000 times
    what the lower ones do."""
    lengths = [700, 40, 6000, 1025]
    q, k, v, table, length = _make(4, Q, 2, 2, D, page, lengths, dtype, 7)
    q.zero_(); k.zero_()
    q[..., :32], q[..., 32] = 64.0, 1.0
    k[..., :31], k[..., 31] = sign * 4096.0, sign * 4032.0
    for b, n in enumerate(lengths):
        for x in range(n):
            k[int(table[b, x // page]), x % page, :, 32] = float(second if (x // 200) % 2 else first)
    base = sign * 64 * (31 * 4096 + 4032)
    out, lse, st = P.paged_attention(q, k, v, table, length, scale=scale)
    assert int(st.abs().max()) == 0
    half = torch.finfo(dtype).eps / 2
    for b, n in enumerate(lengths):
        vb = _rows(table, v, b, n, page)
        s = torch.tensor([float(second if (x // 200) % 2 else first) for x in range(n)], dtype=torch.float64, device=DEV) * scale
        for j in range(Q):
            m = n - Q + j + 1
            w = torch.softmax(s[:m], 0)
            want = torch.einsum("x,xhd->hd", w, vb[:m]).repeat_interleave(2, 0)
            size = torch.einsum("x,xhd->hd", w, vb[:m].abs()).repeat_interleave(2, 0)
            # exponents: 8 log2(e) apart at most, the constant rounded by 2^-24 of itself and each exponent (up to 24: what the maximum's rounding took away is below 8, the lower scores
            # 12 below) by 2^-24 of itself; powers of two 2^-22; the rest as above
            share = 2 * (24 * 2.0 ** -23 + 2.0 ** -21 + (2.0 ** -16 if dtype == BF16 else 0)) + 2.0 ** -20 + (m + 4) * 2.0 ** -23
            err = (out[b, j].double() - want).abs()
            assert bool((err <= half * (1 + share) * want.abs() + share * size).all()), (b, j, float((err / size).max()))
            ll = base * scale + float(torch.logsumexp(s[:m], 0))
            assert abs(float(lse[b, j, 0]) - ll) <= 4 * 2.0 ** -24 * abs(ll)
