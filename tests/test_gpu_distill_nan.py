"""Values that are not finite where a row has next to nothing: among masked entries, far below the row's best, as all of a stretch.  A NaN flags its row wherever it stands, on the streaming kernel as on the
float64 one: loss, log-sum-exp and gradient are 0."""
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


def _rows(N, V, k, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = (2.0 * torch.randn((N, V), generator=g, device=DEV)).to(dtype)
    token = torch.rand((N, V // 4), generator=g, device=DEV).topk(k, 1).indices.to(torch.int32)      # in the first quarter
    logit = 2.0 * torch.randn((N, k), generator=g, device=DEV)
    return s, token, logit


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("V,N,dtype", [(2000, 1000, BF16), (16384, 400, BF16), (40000, 30, BF16), (40000, 400, F32), (151936, 300, BF16), (151936, 152, F32)])
def test_a_nan_among_masked_entries(V, N, dtype, reverse):
    k = 24
    s, token, logit = _rows(N, V, k, dtype, V)
    lse = torch.full((N,), 12.0, device=DEV)
    clean, _ = P.distill_top(s, token, logit, lse, reverse=reverse)
    at = 3 * V // 4
    low = float(torch.finfo(dtype).min)
    bad = {}
    for i, (fill, one) in enumerate([(-INF, NAN), (low, NAN), (-1e9, NAN), (-1e30, -NAN), (-INF, -NAN), (NAN, NAN), (-NAN, -NAN), (-200.0, NAN), (-5000.0, NAN)]):
        for j, where in enumerate((at, (at + V) // 2, V - 1)):
            row = 29 - (3 * i + j) if N < 100 else (31 * (3 * i + j)) % N
            s[row, at:] = fill
            s[row, where] = one
            bad[row] = True
    if N >= 100:
        s[N - 1, at:] = -INF                  # masks alone: as good as any
        s[N - 2, at:] = low
    P.check()
    for kernel in (0, 1):
        prev = P.set_kernel(kernel)
        try:
            out, grad = P.distill_top(s, token, logit, lse, reverse=reverse)
            alone, _ = P.distill_top(s, token, logit, lse, reverse=reverse, dlogits=None)
        finally:
            P.set_kernel(prev)
        want = torch.zeros(N, dtype=torch.int32)
        want[list(bad)] = 8
        assert out["row_status"].cpu().equal(want) and alone["row_status"].cpu().equal(want), kernel
        rows = torch.tensor(list(bad), device=DEV)
        for o in (out, alone):
            assert not o["loss"][rows].any() and not o["lse"][rows].any()
        assert not grad[rows].any() and torch.isfinite(grad).all()
        same = torch.ones(N, dtype=torch.bool, device=DEV)
        same[rows] = False
        if N >= 100:
            same[N - 2:] = False
        if kernel == 0:
            assert torch.equal(out["loss"][same], clean["loss"][same])
        assert P.check() == 2 * len(bad)
