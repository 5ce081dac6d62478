"""Arguments that saki_linear_ce_fwd and saki_linear_ce_bwd refuse, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


def _in(**other):
    i = binding.SakiLinearIn()
    i.hidden = i.weight = i.target = ONE
    i.N, i.d, i.V, i.ld_h, i.ld_w, i.temperature = 10, 64, 1000, 64, 64, 1.0
    for k, v in other.items():
        setattr(i, k, v)
    return i


def _fwd(scratch=ONE, scratch_bytes=1 << 40, lse=ONE, **other):
    o = binding.SakiLinearOut()
    o.lse = lse
    return binding.load_library().saki_linear_ce_fwd(C.byref(_in(**other)), C.byref(o), scratch, scratch_bytes, None)


def _bwd(scratch=ONE, scratch_bytes=1 << 40, lse=ONE, dhidden=ONE, ld_dh=64, dweight=ONE, ld_dw=64, grad_scale=1.0, **other):
    return binding.load_library().saki_linear_ce_bwd(C.byref(_in(**other)), lse, dhidden, ld_dh, dweight, ld_dw, grad_scale, scratch, scratch_bytes, None)


BAD = [dict(N=-1), dict(N=(1 << 22) + 1), dict(d=0), dict(d=(1 << 16) + 8), dict(V=1), dict(V=(1 << 22) + 1), dict(temperature=0.0), dict(temperature=-1.0),
       dict(temperature=float("nan")), dict(temperature=float("inf")), dict(ld_h=63), dict(ld_w=56), dict(hidden=None), dict(weight=None), dict(target=None),
       dict(corrected=ONE), dict(lse=None), dict(scratch=None), dict(scratch_bytes=100)]


@pytest.mark.parametrize("other", BAD)
def test_refused(other):
    assert _fwd(**other) == 1 and P.last_error()
    assert _bwd(**other) == 1 and P.last_error()


@pytest.mark.parametrize("other", [dict(ld_dh=63), dict(ld_dw=0), dict(grad_scale=float("nan")), dict(grad_scale=float("inf")), dict(dhidden=None, dweight=None)])
def test_refused_backward(other):
    assert _bwd(**other) == 1 and P.last_error()


@pytest.mark.parametrize("other", [dict(weight=ONE + 8), dict(ld_w=68), dict(d=60), dict(hidden=ONE + 1), dict(scratch=ONE + 128)])
def test_alignment(other):
    assert _fwd(**other) == 2 and P.last_error()
    assert _bwd(**other) == 2 and P.last_error()


def test_alignment_of_the_gradients():
    for other in (dict(dhidden=ONE + 2), dict(dweight=ONE + 8), dict(ld_dh=68), dict(ld_dw=65)):
        assert _bwd(**other) == 2 and P.last_error()


def test_empty_calls_and_scratch():
    lib = binding.load_library()
    assert _fwd(N=0, hidden=None, target=None, lse=None, scratch=None, scratch_bytes=0) == 0
    assert _bwd(N=0, hidden=None, target=None, lse=None, scratch=None, scratch_bytes=0, dweight=None) == 0
    assert lib.saki_linear_ce_fwd(None, None, ONE, 1, None) == 1 and lib.saki_linear_ce_bwd(None, ONE, ONE, 64, ONE, 64, 1.0, ONE, 1, None) == 1
    assert lib.saki_linear_ce_scratch_bytes(10, 64, 1, 0) == 0 and lib.saki_linear_ce_scratch_bytes(0, 64, 1000, 1) > 0
    for n, d, v in ((1, 8, 2), (8192, 2560, 151936), (1 << 20, 64, 1 << 22), (300, 1 << 16, 5000)):
        for backward in (0, 1):
            need = lib.saki_linear_ce_scratch_bytes(n, d, v, backward)
            assert need > 2 * n * d and _fwd(N=n, d=d, V=v, ld_h=d, ld_w=d, scratch_bytes=lib.saki_linear_ce_scratch_bytes(n, d, v, 0) - 1) == 1


def test_tensors_are_checked():
    h, w, t = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for args in ((h, w[:, :56], t), (h.float(), w, t), (h, w, t[:3]), (h, w, t.long()), (h.t(), w, t), (h, w, t)):
        with pytest.raises(ValueError):      # the last: not on a GPU
            P.linear_ce(*args)
