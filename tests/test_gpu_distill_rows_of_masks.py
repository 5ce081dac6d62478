"""Rows masked throughout by a large negative number, and lists of such logits: what counts are differences, so a row of one value is uniform, at any temperature.  Both kernels, against 64 bits in differences
to the row's largest logit, with the tolerances of test_gpu_distill_top.py (2e-5 of the terms, half a step of the type)."""
import math

import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEAST_REST = 2.0 ** -20


@pytest.mark.parametrize("kernel", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [1.0, 1.3, 50.0, 1e-3])
@pytest.mark.parametrize("V,k", [(2, 2), (27, 20), (700, 40), (40000, 64)])
@pytest.mark.parametrize("rest,reverse", [(False, False), (True, False), (True, True)])
def test_rows_of_one_mask(V, k, tau, dtype, rest, reverse, kernel):
    g = torch.Generator(device=DEV).manual_seed(V)
    tau = float(torch.tensor(tau, dtype=torch.float32))
    low = float(torch.finfo(dtype).min)
    s = torch.stack([torch.full((V,), x, device=DEV) for x in (low, -1e30, -1e9, 3e38, 1e30, 0.0, low, low, -1e30)])
    s[6, V - 1], s[7, 0] = -1e30, -math.inf if V > 2 else low      # one far above the others; one that is not there
    s[8] *= 1 + torch.rand(V, generator=g, device=DEV)             # differences of 1e30
    s = s.to(dtype)
    N = s.shape[0]
    token = torch.rand((N, V), generator=g, device=DEV)
    token[:, 0] = -1.0 if V > 2 else 0.5                           # (not listed)
    token = token.topk(k, 1).indices
    logit = torch.randn((N, k), generator=g, device=DEV) * tau
    lse = torch.logsumexp(logit.double() / tau, 1).float() + 0.5 if rest else None
    if not rest:
        logit[0], logit[1], logit[2] = -float(torch.finfo(torch.float32).max), -1e30, 1e30
    prev = P.set_kernel(kernel)
    try:
        out, grad = P.distill_top(s, token.to(torch.int32), logit, lse, reverse=reverse, temperature=tau, grad_scale=0.37 * tau)
    finally:
        P.set_kernel(prev)
    d = (s.double() - s.double().amax(1, keepdim=True)) / tau
    lp = d - torch.logsumexp(d, 1, keepdim=True)
    p = lp.exp()
    t = logit.double()
    if rest:
        lw = t / tau - lse.double()[:, None]
    else:
        t = (t - t.amax(1, keepdim=True)) / tau
        lw = t - torch.logsumexp(t, 1, keepdim=True)
    listed = torch.zeros((N, V), dtype=torch.bool, device=DEV).scatter_(1, token, True)
    lw = torch.zeros_like(p).scatter_(1, token, lw)
    w = torch.where(listed, lw.exp(), 0.0)
    W = w.sum(1, keepdim=True)
    lS = torch.logsumexp(torch.where(listed, -math.inf, lp), 1, keepdim=True)
    there = (lS > -1000 * math.log(2)) & rest
    R = torch.where(there, (1 - W).clamp(min=LEAST_REST), 0.0)
    lS, lR = torch.where(there, lS, 0.0), torch.where(there, R.clamp(min=1e-300).log(), 0.0)
    if reverse:
        ratio, size = torch.where(listed, lp - lw, lS - lR), torch.where(listed, lp.abs() + lw.abs(), lS.abs() + lR.abs())
        loss = torch.where(p > 0, p * ratio, 0.0).sum(1, keepdim=True)
        loss_mag = 1 + torch.where(p > 0, p * (1 + size), 0.0).sum(1, keepdim=True)
        want, mag = torch.where(p > 0, p * (ratio - loss), 0.0), torch.where(p > 0, p * (1 + size + loss_mag), 0.0)
    else:
        loss = torch.where(listed, w * (lw - lp), 0.0).sum(1, keepdim=True) + R * (lR - lS)
        loss_mag = 1 + torch.where(listed, w * (1 + lw.abs() + lp.abs()), 0.0).sum(1, keepdim=True) + R * (1 + lR.abs() + lS.abs())
        q = torch.where(there & ~listed, (lp - lS).exp() * R, 0.0)
        want, mag = torch.where(listed, p * (W + R) - w, p * (W + R) - q), p * (W + R) + w + q
    assert not out["row_status"].any()
    far = loss.abs()[:, 0] > 3.4e38                                # (the largest that float32 holds is 3.4028e38)
    assert bool((far | ((out["loss"].double() - loss[:, 0]).abs() <= 2e-5 * loss_mag[:, 0])).all())
    assert bool((out["loss"][far] >= 3.39e38).all())              # (infinite, or just below)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
    assert bool(((grad.double() - 0.37 * want).abs() <= 0.37 * (2e-5 * mag + half * want.abs()) + 1e-35).all())
