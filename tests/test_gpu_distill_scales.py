"""Gradients whose factor, grad_scale / temperature, is near or beyond what float32 holds: masked entries have gradient 0, others what the float64 oracle has, as far as the type holds it.  Tolerances of
test_gpu_distill_top.py: 2e-5 of the terms, all below 40 times the gradient's factor here, and half a step."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(6, 50), (5, 40000), (1000, 3001)])
@pytest.mark.parametrize("grad_scale,tau", [(1e10, 1e-30), (1e5, 1e-30), (3e38, 0.25), (3e38, 4.0), (1e37, 1.0)])
@pytest.mark.parametrize("rest,reverse", [(False, False), (True, False), (True, True)])
def test_factors_beyond_float32(N, V, grad_scale, tau, rest, reverse, dtype):
    g = torch.Generator(device=DEV).manual_seed(V)
    k = 5
    tau = float(np.float32(tau))
    s = (torch.randn((N, V), generator=g, device=DEV) * tau).to(dtype)
    token = torch.rand((N, V - 10), generator=g, device=DEV).topk(k, 1).indices.to(torch.int32)
    s[:, V - 7] = -float("inf")
    s[1, V - 9:] = -float("inf")
    logit = torch.randn((N, k), generator=g, device=DEV) * tau
    lse = torch.full((N,), 5.0, device=DEV) if rest else None
    out, grad = P.distill_top(s, token, logit, lse, reverse=reverse, temperature=tau, grad_scale=grad_scale)
    assert P.last_kernel() == 4 and not out["row_status"].any()
    rows = list(range(min(N, 6)))
    ref = O.distill_top(*(x[rows].double().cpu().numpy() if x is not token else x[rows].cpu().numpy() for x in (s, token, logit)), None if lse is None else lse[rows].double().cpu().numpy(), reverse,
                        tau, None, float(np.float32(grad_scale)))
    assert np.all(np.abs(out["loss"][rows].double().cpu().numpy() - ref["loss"]) <= 2e-5 * 40)
    assert not grad[:, V - 7].any() and not grad[1, V - 9:].any() and not grad.isnan().any()
    got, want = grad[rows].double().cpu().numpy(), ref["grad"]
    factor, most = float(np.float32(grad_scale)) / tau, float(torch.finfo(dtype).max)
    p = np.exp(s[rows].double().cpu().numpy() / tau - ref["lse"][:, None])
    at = token[rows].long().cpu().numpy()
    np.put_along_axis(p, at, 1.0, 1)
    bound = 2e-5 * 40 * factor * p + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * np.abs(want)
    sure = np.abs(want) + bound < most
    assert np.all(np.abs(got - want)[sure] <= bound[sure])
    beyond = np.abs(want) - bound > most
    assert np.all(np.isinf(got[beyond]) & (np.sign(got[beyond]) == np.sign(want[beyond])))
