"""Rows that follow one another in a block with lists in different warps' segments: all of a row's list in one stretch, the next row's in another, in any order."""
import pytest
import torch

from distill_reference import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("N,V,parts,dtype", [(9000, 1100, 4, BF16), (9000, 2048, 8, BF16), (6000, 5000, 16, F32), (3000, 20001, 8, BF16), (1800, 45000, 16, BF16), (900, 70000, 32, BF16), (900, 60000, 32, F32)])
def test_lists_in_other_segments(N, V, parts, dtype, reverse):
    g = torch.Generator(device=DEV).manual_seed(V)
    k, width = 128, V // parts
    s = (2.0 * torch.randn((N, V), generator=g, device=DEV)).to(dtype)
    part = torch.randint(0, parts, (N, 1), generator=g, device=DEV)
    token = part * width + torch.rand((N, width), generator=g, device=DEV).topk(k, 1).indices      # as many as fit into a stretch, in any order
    logit = s.float().gather(1, token) + torch.randn((N, k), generator=g, device=DEV)
    lse = torch.logsumexp(s.float(), 1) + 0.5
    check(s, token.to(torch.int32), logit, lse, reverse, repeats=8)
    low = torch.arange(k, device=DEV, dtype=torch.int32).repeat(N, 1)                               # the lowest tokens of every other row, the highest of the others
    token = torch.where(torch.arange(N, device=DEV)[:, None] % 2 == 0, low, V - 1 - low)
    token = torch.where(torch.rand((N, 1), generator=g, device=DEV) < 0.2, token.flip(1), token).to(torch.int32)
    check(s, token, logit, lse, reverse, repeats=8)
