"""Gradients of the hidden states whose sums over the vocabulary are cut into parts, with a last piece of the vocabulary that has fewer blocks of 64 entries than there are parts: such
parts have nothing to add.  Against float64 products on the GPU, by the tolerances of test_gpu_linear_ce.py: a logit off by d 2^-23 of its terms' magnitudes, a probability by twice that share, G rounded to
bf16 (2^-8 of an element), sums of K terms off by K 2^-23 of the terms' magnitudes, the sum rounded to bf16."""
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


# (9217 to 9472 rows of up to 256 features: pieces of 55 tiles of 256 entries, two parts; 2971 tiles are 54 pieces and one tile, here of one, two, three and four blocks)
@pytest.mark.parametrize("N,d,V,masked", [(9300, 64, 760321, 0), (9217, 200, 760384, 0), (9400, 64, 760385, 300), (9472, 128, 760512, 0), (9250, 8, 760576, 0)])
def test_parts_without_a_block(N, d, V, masked):
    g = torch.Generator(device=DEV).manual_seed(N + d)
    w = (2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device=DEV)).to(BF16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn((N, d), generator=g, device=DEV) + 2.0 * torch.rand((N, 1), generator=g, device=DEV) * w[target.long()].float()).to(BF16)
    mask = (torch.randperm(N, generator=g, device=DEV) >= masked).to(torch.uint8)
    out = P.linear_ce(h, w, target, mask=mask)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"], mask=mask)
    only, _ = P.linear_ce_bwd(h, w, target, out["lse"], mask=mask, dweight=None)
    assert torch.equal(only, dh)              # dH without dW's tiles beside it
    w64 = w.double()
    rows = torch.arange(0, N, 41, device=DEV)
    hr, yr = h[rows].double(), target[rows].long()
    z = hr @ w64.t()
    z_err = (d + 4) * 2.0 ** -23 * float((hr.abs() @ w64.abs().t()).max()) + 4e-6
    G = torch.softmax(z, 1)
    at = torch.arange(rows.numel(), device=DEV)
    p_tok = G[at, yr]
    G[at, yr] -= 1.0
    G *= mask[rows, None]
    want, a = G @ w64, G.abs()
    a[at, yr] += p_tok * 2 * z_err / 2.0 ** -8              # (pi - 1 is off by a share of pi)
    bound = (2.0 ** -8 + V * 2.0 ** -23 + 2 * z_err) * (a @ w64.abs()) + 2.0 ** -8 * want.abs() + 1e-30
    err = (dh[rows].double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    assert not dh[mask == 0].any()
    # the last entries of the vocabulary, from all rows
    last = torch.arange(V - 70, V, device=DEV)
    lse = torch.cat([torch.logsumexp(h[i:i + 256].double() @ w64.t(), 1) for i in range(0, N, 256)])
    h64 = h.double()
    G = torch.exp(h64 @ w64[last].t() - lse[:, None]) - (target.long()[:, None] == last).double()
    G *= mask[:, None]
    want, mag = G.t() @ h64, G.abs().t() @ h64.abs()
    assert bool(((dw[last].double() - want).abs() <= (2.0 ** -8 + N * 2.0 ** -23 + 4 * z_err) * mag + 2.0 ** -8 * want.abs() + 1e-30).all())
    assert P.check() == 0
