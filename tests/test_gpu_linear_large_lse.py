"""Gradients of rows with a large log-sum-exp, at temperatures at which the factor of the products, log2(e) / temperature, is about half a step of a float32 off.

Two tokens, of logits b + 5 and b - 5 over the temperature, their products exact: G is -p and p of the less likely one, p about 1e-3, and the sum of both 0.  A share r of both probabilities, 1 together, is r in that
sum: r is half a float32 step of the log-sum-exp and half a step of it in base 2, and what float32 exponentials give, 1e-6.  Roundings of G to bf16 are 2^-8 of p, and of what is off, each; that of the sum 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _temperatures(d, n):
    """Those of the float32 numbers from 1 on whose factor is off most, both ways."""
    tau = np.float32(1) + np.arange(200000, dtype=np.float32) * np.float32(2.0 ** -18)
    c = (1.0 + (d + 15) // 16 * 2.0 ** -26) / np.log(2.0) / tau.astype(np.float64)
    off = c.astype(np.float32).astype(np.float64) / c - 1.0
    order = np.argsort(off)
    return [float(x) for x in tau[np.concatenate([order[:n], order[-n:]])]]


@pytest.mark.parametrize("tau", _temperatures(64, 3))
def test_the_factor_s_rounding_cancels(tau):
    N, d = 600, 64
    h, w = torch.zeros((N, d), dtype=BF16, device=DEV), torch.zeros((2, d), dtype=BF16, device=DEV)
    w[:, 0] = 1.0
    w[0, 1], w[1, 1] = 1.0, -1.0
    h[:, 0] = torch.linspace(760.0, 1400.0, N, device=DEV).to(BF16)
    h[:, 1] = 5.0
    target = torch.zeros(N, dtype=torch.int32, device=DEV)
    out = P.linear_ce(h, w, target, temperature=tau)
    dh, _ = P.linear_ce_bwd(h, w, target, out["lse"], temperature=tau, grad_scale=tau, dweight=None)
    rare = 1.0 / (1.0 + np.exp(10.0 / tau))
    lse = out["lse"].cpu().numpy()
    share = (np.spacing(lse) + np.spacing((lse / np.log(2.0)).astype(np.float32)) * np.log(2.0)) / 2 + 1e-6
    bound = (share + 2 * 2.0 ** -8 * (rare + share)) * (1 + 2.0 ** -8)
    err = dh[:, 0].double().abs().cpu().numpy()
    assert np.all(err <= bound), (err / bound).max()
