"""Distillation at large temperatures, where the lowest finite value over the temperature is no large number: what lies beside a row in memory must not count.  Against the float64 oracle, by the tolerances of
test_gpu_distill_top.py; the gradient's factor, grad_scale / temperature, is 0.37."""
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V,tau", [(9, 9, 3e38), (3, 2, 2e38), (700, 1003, 3e38), (9, 9, 1e37), (700, 1003, 1e37), (40, 30001, 2.0 ** 125), (20, 100003, 1e36), (5, 17, 2.0 ** 100), (5, 500, 1e5)])
@pytest.mark.parametrize("reverse", [False, True])
def test_what_lies_beside_a_row(N, V, tau, dtype, reverse):
    g = torch.Generator(device=DEV).manual_seed(V)
    k = min(8, V - 1)
    wide = torch.zeros((N, V + 5), dtype=dtype, device=DEV)
    wide.copy_(torch.randn((N, V + 5), generator=g, device=DEV) * min(tau, 1e37))
    s = wide[:, 3:3 + V]
    token = torch.rand((N, V), generator=g, device=DEV).topk(k, 1).indices.to(torch.int32)
    logit = torch.randn((N, k), generator=g, device=DEV) * min(tau, 1e37)
    tau = float(torch.tensor(tau, dtype=torch.float32))
    lse = torch.full((N,), float(torch.tensor(float(V)).log()) + 3.0, device=DEV)
    out, grad = P.distill_top(s, token, logit, lse, reverse=reverse, temperature=tau, grad_scale=0.37 * min(tau, 1e37))
    assert P.last_kernel() == 4
    rows = list(range(0, N, max(1, N // 8)))
    ref = O.distill_top(s[rows].double().cpu().numpy(), token[rows].cpu().numpy(), logit[rows].double().cpu().numpy(), lse[rows].double().cpu().numpy(), reverse, tau, None, 0.37 * min(tau, 1e37))
    t64 = lambda x: torch.from_numpy(x).to(DEV)
    assert not out["row_status"].any()
    assert bool(((out["lse"][rows].double() - t64(ref["lse"])).abs() <= 1e-5 + 2.0 ** -24 * t64(ref["lse"]).abs()).all())
    # (log-ratios are below 20 here, the terms' magnitudes below 50 for the loss and below 50 times the largest of pi, w, R / S pi for the gradient)
    assert bool(((out["loss"][rows].double() - t64(ref["loss"])).abs() <= 2e-5 * 50).all())
    want = t64(ref["grad"])
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
    assert bool(((grad[rows].double() - want).abs() <= 2e-5 * 50 * want.abs().amax(1, keepdim=True) + half * want.abs()).all())
