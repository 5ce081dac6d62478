"""Short rows, several to a block, with lists longer than the row's steps of 32 pieces: some of the warps that bring in the next row's list have no step of the row themselves."""
import pytest
import torch

from distill_reference import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [64, 128])
@pytest.mark.parametrize("V", [100, 250, 500, 700])
@pytest.mark.parametrize("N", [500, 5000])
def test_lists_of_later_rows(N, V, k, dtype):
    g = torch.Generator(device=DEV).manual_seed(N + V + k)
    s = (2.0 * torch.randn((N, V), generator=g, device=DEV)).to(dtype)
    n = min(k, V - 10)
    token = torch.full((N, k), -1, dtype=torch.int32, device=DEV)
    token[:, k - n:] = torch.rand((N, V), generator=g, device=DEV).topk(n, 1).indices.to(torch.int32)      # (every row another list; the entries that are not there first)
    token = torch.where(torch.rand((N, k), generator=g, device=DEV) < 0.1, -1, token)
    logit = s.float().gather(1, token.clamp(min=0).long()) + torch.randn((N, k), generator=g, device=DEV)
    lse = torch.logsumexp(s.float(), 1) + 0.5
    for teacher_lse, reverse in ((lse, False), (lse, True), (None, False)):
        check(s, token, logit, teacher_lse, reverse, repeats=4)
