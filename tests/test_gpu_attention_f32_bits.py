"""How many bits float32 attention keeps: single positions, where the log-sum-exp is one product and the output one value."""
import pytest
import torch

import paper_2609_36601_b200 as P
from test_gpu_paged_attention import DEV, F32

pytestmark = pytest.mark.gpu


def _single(q, k, v, scale):
    """One sequence of one position for each row of q, k, v [N, D]."""
    N, D = q.shape
    table = torch.arange(N, dtype=torch.int32, device=DEV)[:, None]
    out, lse, st = P.paged_attention(q.view(N, 1, 1, D), k.view(N, 1, 1, D), v.view(N, 1, 1, D), table, torch.ones(N, dtype=torch.int32, device=DEV), scale=scale)
    assert int(st.abs().max()) == 0
    return out.view(N, D), lse.view(N)


@pytest.mark.parametrize("D", [4, 64, 80, 128, 256])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_product_whose_factors_have_long_rests(D, sign):
    """Factors of 1 + 2^-10 - 2^-21: eleven bits and a rest of nearly a unit of the eleventh.  Rests of the same sign on both sides would lose 2^-20 of the product.  Here the first factor
    is 1 + 2^-10 and a rest of -2^-21, the second 1 and 2^-10 - 2^-21, all exact: the product is off by two sums of float32 (cut: 2^-23 each), log2(e) times it, the sum with the
    maximum, ln 2 times that and the two constants by 2^-24 each."""
    x = 1 + 2.0 ** -10 - 2.0 ** -21
    q, k = torch.zeros((32, D), device=DEV), torch.zeros((32, D), device=DEV)
    for i in range(32):
        q[i, (5 * i) % D], k[i, (5 * i) % D] = x * 2.0 ** (i % 5), sign * x * 2.0 ** -(i % 3)
    _, lse = _single(q, k, torch.ones((32, D), device=DEV), 64.0)
    want = 64 * (q.double() * k.double()).sum(1)
    assert bool(((lse.double() - want).abs() <= 5 * 2.0 ** -23 * want.abs()).all()), float(((lse.double() - want) / want).abs().max())


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_a_value_that_is_seen_alone(D):
    """w v / w: rests 2^-11 and 2^-10 long (2^-21 dropped), their cuts (2^-23, 2^-22), two sums (2^-23 each), a reciprocal and a product (2^-24 each)."""
    g = torch.Generator(device=DEV).manual_seed(D)
    q, k, v = (torch.randn((500, D), generator=g, device=DEV) for _ in range(3))
    out, _ = _single(q, k, v, 1.0)
    tol = 2.0 ** -21 + 2.0 ** -22 + 2.0 ** -23 + 2 * 2.0 ** -23 + 2 * 2.0 ** -24
    assert bool(((out.double() - v.double()).abs() <= tol * v.double().abs()).all())


@pytest.mark.parametrize("D", [64, 80, 256])
def test_the_largest_numbers(D):
    """Keys and values of the largest magnitude where only some of the queries look: the others do not notice."""
    big = torch.finfo(F32).max
    g = torch.Generator(device=DEV).manual_seed(D)
    n, Q = 90, 5
    q = torch.randn((1, Q, 2, D), generator=g, device=DEV)
    k, v = (torch.randn((n, 1, 1, D), generator=g, device=DEV) for _ in range(2))
    table, length = torch.arange(n, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV)
    want = P.paged_attention(q, k, v, table, length)
    for x in (big, -big):
        kk, vv = k.clone(), v.clone()
        kk[n - 1] = vv[n - 1] = x
        got = P.paged_attention(q, kk, vv, table, length)
        assert torch.equal(got[0][:, :Q - 1], want[0][:, :Q - 1]) and torch.equal(got[1][:, :Q - 1], want[1][:, :Q - 1])
