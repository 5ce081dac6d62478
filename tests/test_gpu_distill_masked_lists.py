"""The reverse divergence where a listed token is masked, in the student's row by a large negative number or in the teacher's list by one: p log(p / w) of p = 0 is 0, in the loss and in the gradient.
Against 64 bits, in differences to a row's largest logit, with the tolerances of test_gpu_distill_top.py (2e-5 of the terms, half a step of the type)."""
import math

import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEAST_REST = 2.0 ** -20


@pytest.mark.parametrize("kernel", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [1.0, 0.7, 1e-10])
@pytest.mark.parametrize("N,V,k", [(8, 27, 20), (1000, 700, 40), (40, 40000, 64)])
def test_probabilities_of_zero(N, V, k, tau, dtype, kernel):
    g = torch.Generator(device=DEV).manual_seed(V)
    tau = float(torch.tensor(tau, dtype=torch.float32))
    s = (2.0 * torch.randn((N, V), generator=g, device=DEV) * tau).to(dtype)
    token = torch.rand((N, V), generator=g, device=DEV).topk(k, 1).indices
    logit = 2.0 * torch.randn((N, k), generator=g, device=DEV) * tau
    for j, mask in enumerate((float(torch.finfo(dtype).min), -1e30, -1e9, -2e4)):
        s.scatter_(1, token[:, 2 * j:2 * j + 2], mask)
    lse = torch.logsumexp(logit.double() / tau, 1).float() + 0.5
    logit[:, 0], logit[:, 8:10] = -float(torch.finfo(torch.float32).max), -1e30      # (not -inf: entries that are there, with a weight of 0; the first for a token that the student has masked as well)
    s.scatter_(1, token[:, 8:9], float(torch.finfo(dtype).min))
    s.scatter_(1, token[:, 9:10], -1e30)
    prev = P.set_kernel(kernel)
    try:
        out, grad = P.distill_top(s, token.to(torch.int32), logit, lse, reverse=True, temperature=tau, grad_scale=0.37 * tau)
    finally:
        P.set_kernel(prev)
    d = (s.double() - s.double().amax(1, keepdim=True)) / tau
    lp = d - torch.logsumexp(d, 1, keepdim=True)
    p = lp.exp()
    lw = logit.double() / tau - lse.double()[:, None]
    listed = torch.zeros((N, V), dtype=torch.bool, device=DEV).scatter_(1, token, True)
    ratio = torch.zeros_like(p).scatter_(1, token, lp.gather(1, token) - lw)
    size = torch.zeros_like(p).scatter_(1, token, lp.gather(1, token).abs() + lw.abs())
    R = (1 - lw.exp().sum(1, keepdim=True)).clamp(min=LEAST_REST)
    lS = torch.logsumexp(torch.where(listed, -math.inf, lp), 1, keepdim=True)
    ratio, size = torch.where(listed, ratio, lS - R.log()), torch.where(listed, size, lS.abs() + R.log().abs())
    loss = torch.where(p > 0, p * ratio, 0.0).sum(1, keepdim=True)
    mag = 1 + torch.where(p > 0, p * (1 + size), 0.0).sum(1, keepdim=True)
    assert not out["row_status"].any()
    assert bool(((out["loss"].double() - loss[:, 0]).abs() <= 2e-5 * mag[:, 0]).all())
    want, bound = torch.where(p > 0, p * (ratio - loss), 0.0) * 0.37, torch.where(p > 0, p * (1 + size + mag), 0.0) * 0.37
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
    assert bool(((grad.double() - want).abs() <= 2e-5 * bound + half * want.abs() + 1e-35).all())
