"""No rows at all: either gradient alone is answered, as both are."""
import pytest
import torch

import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_one_gradient_of_no_rows():
    h, w = torch.zeros((0, 64), dtype=torch.bfloat16, device=DEV), torch.ones((300, 64), dtype=torch.bfloat16, device=DEV)
    target = torch.zeros(0, dtype=torch.int32, device=DEV)
    lse = P.linear_ce(h, w, target)["lse"]
    dh, dw = P.linear_ce_bwd(h, w, target, lse, dweight=None)
    assert dh.shape == (0, 64) and dw is None
    dh, dw = P.linear_ce_bwd(h, w, target, lse, dhidden=None, dweight=torch.full_like(w, 3.0))
    assert dh is None and not dw.any()
    dh, dw = P.linear_ce_bwd(h, w, target, lse)
    assert dh.shape == (0, 64) and not dw.any()
