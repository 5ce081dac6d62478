"""A gradient's factor, grad_scale / temperature, that no float32 holds is refused, on the host: times sums of 0 (masked rows, tokens that no row is near) it would be NaN."""
import ctypes as C

import pytest

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


@pytest.mark.parametrize("grad_scale,temperature", [(1e10, 1e-30), (-1e10, 1e-30), (3e38, 0.5), (1.0, 1e-39), (float("inf"), 1e30), (float("nan"), 1.0)])
def test_refused(grad_scale, temperature):
    i = binding.SakiLinearIn()
    i.hidden = i.weight = i.target = ONE
    i.N, i.d, i.V, i.ld_h, i.ld_w, i.temperature = 10, 64, 1000, 64, 64, temperature
    lib = binding.load_library()
    assert lib.saki_linear_ce_bwd(C.byref(i), ONE, ONE, 64, ONE, 64, grad_scale, ONE, 1 << 40, None) == 1
    assert "grad_scale" in P.last_error()


def test_large_ones_that_float32_holds():
    """... are not: the next check answers."""
    i = binding.SakiLinearIn()
    i.hidden = i.weight = i.target = ONE
    i.N, i.d, i.V, i.ld_h, i.ld_w, i.temperature = 10, 64, 1000, 64, 64, 1e-8
    assert binding.load_library().saki_linear_ce_bwd(C.byref(i), ONE, ONE, 64, ONE, 64, 1e30, ONE, 100, None) == 1
    assert "scratch" in P.last_error()
