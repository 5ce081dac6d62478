"""How near the cross entropy from hidden states comes on the whole, beside the worst case of test_gpu_linear_ce.py.

Losses.  A logit of d features is a float32 sum that takes d / 16 additions, each of which the tensor cores cut towards 0: by up to 2^-23 of what the sum is by then, evenly spread.  The average of that is made up for by a
factor of the logits, 1 + d 2^-30; what is left is a sum of d / 16 deviations below 2^-24 of the sum as it grows: as a norm over many rows sqrt(d / 16) 2^-24 of the logits, and a third more for what the average of a row's own logits
leaves: 1e-6 at 2560 features, 1.8e-6 at 8192.  Without the factor, or with twice as much, d 2^-30 of the logits would be left: 2.4e-6 and 7.6e-6.
Gradients.  G and the result are each rounded to bf16: a rounding is off by at most 2^-8 of an element, evenly spread, which is 2^-8 / sqrt(3) of it as a norm; two of them, independent, sqrt(2) times that: 3.2e-3.
Sums that need no rounding (here of one feature a row) come out larger by the factor: off by d 2^-30 of the largest logit, and by what float32 exponentials give, 1e-5 and half a step of the result."""
import math

import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _inputs(N, d, V, seed, lean):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device=DEV)).to(BF16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn((N, d), generator=g, device=DEV) + lean * torch.rand((N, 1), generator=g, device=DEV) * w[target.long()].float()).to(BF16)
    return h, w, target


@pytest.mark.parametrize("lean", [0.0, 4.0])
@pytest.mark.parametrize("d", [256, 1024, 2560, 8192])
def test_losses(d, lean):
    N, V = 1024, 16000
    h, w, target = _inputs(N, d, V, d, lean)
    z = h.double() @ w.double().t()
    want = torch.logsumexp(z, 1) - z.gather(1, target.long()[:, None])[:, 0]
    got = P.linear_ce(h, w, target)["loss"].double()
    assert float((got - want).norm() / want.norm()) <= max(4 / 3 * math.sqrt(d / 16) * 2.0 ** -24, 3e-7)


@pytest.mark.parametrize("N,d,V", [(512, 2560, 16000), (1431, 1096, 8003), (64, 1024, 32000)])
def test_gradients(N, d, V):
    h, w, target = _inputs(N, d, V, N, 4.0)
    out = P.linear_ce(h, w, target)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"], grad_scale=1.0 / N)
    G = torch.softmax(h.double() @ w.double().t(), 1)
    G[torch.arange(N, device=DEV), target.long()] -= 1.0
    G /= N
    for got, want in ((dh, G @ w.double()), (dw, G.t() @ h.double())):
        assert float((got.double() - want).norm() / want.norm()) <= math.sqrt(2 / 3) * 2.0 ** -8


@pytest.mark.parametrize("d", [64, 2560, 8192, 65536])
def test_sums_that_need_no_rounding(d):
    N, V = 200, 1000
    g = torch.Generator(device=DEV).manual_seed(d)
    w = torch.randn((V, d), generator=g, device=DEV).to(BF16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    h = torch.zeros((N, d), dtype=BF16, device=DEV)
    at = torch.randint(0, d, (N,), generator=g, device=DEV)
    h[torch.arange(N, device=DEV), at] = (6.0 * torch.rand(N, generator=g, device=DEV)).to(BF16)
    z = h[torch.arange(N, device=DEV), at].double()[:, None] * w[:, at].double().t()
    lse = torch.logsumexp(z, 1)
    z_tok = z.gather(1, target.long()[:, None])[:, 0]
    out = P.linear_ce(h, w, target)
    lack = d * 2.0 ** -30 * z.abs().amax(1)
    assert bool(((out["lse"].double() - lse).abs() <= lack + 1e-5 + 2.0 ** -24 * lse.abs()).all())
    assert bool(((out["loss"].double() - (lse - z_tok)).abs() <= 2 * lack + 1e-5 + 2.0 ** -24 * (lse - z_tok).abs()).all())
