"""Attention over a paged cache: values that are not finite at positions that only some of a block's queries see, in runs of short sequences, where
a worker takes up the next sequence while the products of the one before are under way.  Exact: what such a value does not reach has the bits of
the call with a number in its place (weights of 0 add nothing), what it reaches is not finite."""
import pytest
import torch

import paper_2609_36601_b200 as P
from test_gpu_paged_attention import BF16, DEV, F32, _make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


@pytest.mark.parametrize("dtype,Q,G,D,page", [(BF16, 4, 4, 128, 16), (BF16, 7, 4, 128, 16), (BF16, 7, 2, 64, 8), (BF16, 16, 4, 128, 16), (BF16, 3, 2, 256, 16), (F32, 3, 3, 80, 16)])
def test_short_sequences_one_behind_the_other(dtype, Q, G, D, page):
    B, H = 700, 2
    lengths = [Q + (97 * b) % (300 if b % 3 else 125) for b in range(B)]
    q, k, v, table, length = _make(B, Q, H, G, D, page, lengths, dtype, Q + D)
    want, lse, _ = P.paged_attention(q, k, v, table, length)
    strange = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=dtype, device=DEV)
    reached = torch.zeros((B, Q, H * G, D), dtype=torch.bool, device=DEV)
    v = v.clone()
    for b, n in enumerate(lengths):
        for i in range((b * 7) % 4):                         # none, one, two or three of them: behind query j0 - 1, the last positions most
            j0 = Q - 1 - (b + i) % min(Q, 3) if b % 5 else 1
            x, h, col = n - Q + j0, (b + i) % H, (b * 5 + i * 17) % D
            v[int(table[b, x // page]), x % page, h, col] = strange[(b + i) % 3]
            reached[b, j0:, h * G:(h + 1) * G, col] = True
    assert int(reached.any(-1).any(-1).any(-1).sum()) > B // 2
    for _ in range(25):
        out, again, st = P.paged_attention(q, k, v, table, length)
        assert not torch.isfinite(out[reached]).any()
        assert torch.equal(torch.where(reached, want, out), want) and torch.equal(again, lse) and int(st.abs().max()) == 0
    assert P.check() == 0
