"""Waits of the cross entropy's products that run out: the call ends, its rows are flagged and its gradients are NaN, and the next call is right."""
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TIMEOUT = 32


@pytest.mark.parametrize("limit", [1, 50, 400, 3000, 20000])
def test_expired_waits(limit):
    g = torch.Generator(device=DEV).manual_seed(1)
    N, d, V = 600, 520, 9000
    h = torch.randn((N, d), generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn((V, d), generator=g, device=DEV) / d ** 0.5).to(torch.bfloat16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    mask = (torch.rand(N, generator=g, device=DEV) < 0.8).to(torch.uint8)
    want = P.linear_ce(h, w, target, mask=mask)
    gradients = P.linear_ce_bwd(h, w, target, want["lse"], mask=mask)
    torch.cuda.synchronize()
    P.check()
    before = P.set_wait_limit(limit)
    try:
        for _ in range(4):
            out = P.linear_ce(h, w, target, mask=mask)
            torch.cuda.synchronize()
            late = out["row_status"][mask != 0] == TIMEOUT
            assert (out["row_status"][mask == 0] == 4).all() and late.all() == late.any()
            if late.any():
                assert not out["loss"].any() and out["lse"][mask != 0].isnan().all() and P.check() == int(mask.sum())
            else:
                assert all(torch.equal(out[k], want[k]) for k in want)
            got = P.linear_ce_bwd(h, w, target, want["lse"], mask=mask)
            torch.cuda.synchronize()
            if got[0].isnan().any():
                assert all(x.isnan().all() for x in got)
            else:
                assert all(torch.equal(a, b) for a, b in zip(got, gradients))
    finally:
        P.set_wait_limit(before)
    out = P.linear_ce(h, w, target, mask=mask)
    got = P.linear_ce_bwd(h, w, target, out["lse"], mask=mask)
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], want[k]) for k in want) and all(torch.equal(a, b) for a, b in zip(got, gradients))
    assert P.check() == 0
