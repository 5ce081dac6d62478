"""Rows of equal or capped logits, thousands of them: more elements at the highest value than a block's list holds, in few groups of pieces.  Every row has the lowest tokens at that value, to the bit."""
import math

import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [1, 40, 128])
@pytest.mark.parametrize("N,V", [(4000, 513), (4000, 600), (4000, 1000), (4000, 2048), (4000, 4099), (4000, 8192), (2000, 8200), (900, 20000), (3, 100000), (1, 151936)])
def test_equal_logits(N, V, k, dtype):
    x = torch.full((N, V), 1.5, dtype=dtype, device=DEV)
    first = None
    for _ in range(4):
        out = P.top_logits(x, k)
        assert bool((out["token"] == torch.arange(k, device=DEV, dtype=torch.int32)).all()) and bool((out["logit"] == 1.5).all()) and not out["row_status"].any()
        assert bool(((out["lse"].double() - 1.5 - math.log(V)).abs() <= 1e-5).all()) and bool((out["lse"] == out["lse"][0]).all())
        first = first or out
        assert all(torch.equal(out[n], first[n]) for n in out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [1, 7, 128])
@pytest.mark.parametrize("N,V", [(3000, 1500), (3000, 6001), (2000, 16384), (4, 151936)])
def test_capped_logits(N, V, k, dtype):
    """Random rows cut off at a value that a few to nearly all of their elements reach."""
    g = torch.Generator(device=DEV).manual_seed(V)
    cap = torch.linspace(-3.0, 3.0, N, device=DEV)[torch.randperm(N, generator=g, device=DEV)]
    x = torch.minimum(torch.randn((N, V), generator=g, device=DEV), cap[:, None]).to(dtype)
    best, token = torch.sort(x, dim=1, descending=True, stable=True)
    for _ in range(4):
        out = P.top_logits(x, k)
        assert torch.equal(out["token"], token[:, :k].to(torch.int32)) and torch.equal(out["logit"], best[:, :k].float())
        want = torch.logsumexp(x.double(), 1)
        assert bool(((out["lse"].double() - want).abs() <= 1e-5 + 2.0 ** -24 * want.abs()).all())
