"""Bounded waits of the attention kernels that run out part of the way: the warps that share a worker's tiles give up on the same segment, and every row
that was given up on is told.  A limit of two to a few thousand cycles runs out although the copies are on their way; nothing is withheld."""
import numpy as np
import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding
from test_gpu_paged_attention import BF16, DEV, F32, _make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


# one, two, four and eight warps a worker; pages by TMA and by plain loads; the kernel on tcgen05
@pytest.mark.parametrize("dtype,Q,G,D,page", [(BF16, 1, 4, 64, 16), (BF16, 1, 2, 256, 16), (BF16, 3, 9, 256, 16), (BF16, 8, 8, 256, 16), (BF16, 16, 8, 256, 5),
                                              (F32, 1, 2, 64, 16), (F32, 4, 6, 80, 16), (F32, 7, 8, 64, 5), (F32, 16, 8, 64, 16), (BF16, 7, 4, 128, 16)])
def test_rows_given_up_on_are_told(dtype, Q, G, D, page):
    H = 2
    lengths = [Q + (61 * i) % 211 for i in range(160)] + [9000, 5000]      # many segments a worker, and some that several share
    q, k, v, table, length = _make(len(lengths), Q, H, G, D, page, lengths, dtype, Q + G + D, fill=float("nan"))
    want = P.paged_attention(q, k, v, table, length)
    assert P.check() == 0
    flush = torch.empty(320 << 20, dtype=torch.uint8, device=DEV)
    ran_out = 0
    try:
        for limit in (2, 20, 60, 120, 250, 400, 550, 700, 850, 1000, 1200, 1500, 2000, 2500, 3000, 4000, 6000):
            flush.fill_(1)
            torch.cuda.synchronize()
            P.set_wait_limit(limit)
            out, lse, st = P.paged_attention(q, k, v, table, length)
            assert P.set_wait_limit(0) == limit
            flagged = P.check()                                 # synchronises: the kernels came back
            st = st.cpu().numpy().astype(np.uint32)
            assert np.all((st == 0) | (st == binding.ROW_TIMEOUT)) and flagged == int((st != 0).sum())
            late = torch.isneginf(lse)                          # [B, Q, Hq]
            told = torch.from_numpy(st != 0).to(DEV)
            assert not (late & ~told[:, None, None]).any()
            assert torch.equal(torch.where(late[..., None], torch.zeros_like(out), want[0]), out)
            assert torch.equal(torch.where(late, lse, want[1]), lse)
            by_head = late.view(len(lengths), Q, H, G)          # (rows of a key head that are worked on together are late together: up to 128 of them)
            if Q * G <= 16 or (dtype == F32 and Q * G <= 128) or D == 256:
                whole = by_head.any(1).any(-1)
                assert torch.equal(by_head.all(1).all(-1), whole)
            ran_out += int(told.sum())
        again = P.paged_attention(q, k, v, table, length)
        assert P.check() == 0 and all(torch.equal(x, y) for x, y in zip(again, want))
    finally:
        P.set_wait_limit(0)
    assert ran_out > 0


@pytest.mark.parametrize("dtype,Q,G,D", [(BF16, 1, 4, 128), (BF16, 7, 4, 128), (BF16, 2, 2, 64), (BF16, 1, 2, 64), (F32, 1, 2, 64)])
def test_the_limit_is_a_tiles_not_a_sequences(dtype, Q, G, D):
    """Eight sequences of four million positions on pages that they share: a worker has more than a thousand tiles of one, milliseconds of work, under a limit of a
    quarter of a millisecond, some hundred times what a tile takes."""
    page, n_pages, n = 128, 64, 1 << 22
    g = torch.Generator(device=DEV).manual_seed(D)
    q = torch.randn((8, Q, G, D), generator=g, device=DEV).to(dtype)
    k, v = (torch.randn((n_pages, page, 1, D), generator=g, device=DEV).to(dtype) for _ in range(2))
    table = torch.randint(0, n_pages, (8, n // page), generator=g, device=DEV, dtype=torch.int32)
    length = torch.tensor([n - 5 * b for b in range(8)], dtype=torch.int32, device=DEV)
    want = P.paged_attention(q, k, v, table, length)
    assert P.check() == 0
    try:
        P.set_wait_limit(500000)
        got = P.paged_attention(q, k, v, table, length)
        assert P.set_wait_limit(0) == 500000
    finally:
        P.set_wait_limit(0)
    assert P.check() == 0 and int(got[2].abs().max()) == 0
    assert all(torch.equal(a, b) for a, b in zip(got, want))
