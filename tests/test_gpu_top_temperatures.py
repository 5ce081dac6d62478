"""The log-sum-exp of top_logits over the range of temperatures, of rows whose logits over the temperature are large and negative throughout, among them ones masked by the lowest value.  Against 64 bits, in
differences to the largest logit; tolerance as in test_gpu_top_logits.py, 1e-5 and half a step of the result."""
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [1e-30, 1e-10, 1e-3, 1.0, 50.0, 1e6, 1e20, 1e30, 3e38])
@pytest.mark.parametrize("N,V", [(1, 2), (3, 700), (400, 5000), (4, 151936)])
def test_log_sum_exp(N, V, tau, dtype):
    g = torch.Generator(device=DEV).manual_seed(V)
    tau = float(torch.tensor(tau, dtype=torch.float32))
    for base in (0.0, -1e2, -1e5, -1e7, -9e7, -1.1e8, -2e8, -1e9, -1e12, 1e9):
        if not 1e-30 <= abs(base or 1.0) * tau <= 1e37:
            continue
        x = ((torch.randn((N, V), generator=g, device=DEV) + base).double() * tau).clamp(-3e38, 3e38).to(dtype)
        if N > 1:
            x[1] = float(torch.finfo(dtype).min)
        out = P.top_logits(x, 3, temperature=tau)
        top = x.double().amax(1)
        want = top / tau + torch.logsumexp((x.double() - top[:, None]) / tau, 1)
        fits = want.abs() < 3.4e38
        assert not out["row_status"].any()
        assert bool(((out["lse"].double() - want).abs() <= 1e-5 + 2.0 ** -24 * want.abs())[fits].all()), base
        assert bool((out["lse"][~fits] <= -3.39e38).all())      # (the largest that float32 holds is 3.4028e38: just inside it, or infinite)
        best, token = torch.sort(x, dim=1, descending=True, stable=True)
        assert torch.equal(out["token"][:, :min(3, V)], token[:, :3].to(torch.int32)) and torch.equal(out["logit"][:, :min(3, V)], best[:, :3].float())
