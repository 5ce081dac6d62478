"""Arguments that saki_top_logits refuses, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


def _call(scratch=ONE, scratch_bytes=1 << 40, out=None, **other):
    i, o = binding.SakiTopIn(), binding.SakiTopOut()
    i.logits = o.token = o.logit = ONE
    i.N, i.V, i.dtype, i.ld, i.k, i.temperature = 10, 1000, 1, 1000, 16, 1.0
    for k, v in other.items():
        setattr(i, k, v)
    for k, v in (out or {}).items():
        setattr(o, k, v)
    return binding.load_library().saki_top_logits(C.byref(i), C.byref(o), scratch, scratch_bytes, None)


@pytest.mark.parametrize("other", [dict(N=-1), dict(N=(1 << 24) + 1), dict(V=1), dict(V=(1 << 22) + 1), dict(dtype=2), dict(k=0), dict(k=129), dict(ld=-1), dict(temperature=0.0),
                                   dict(temperature=float("nan")), dict(temperature=float("inf")), dict(logits=None), dict(scratch=None), dict(scratch_bytes=100),
                                   dict(out=dict(token=None)), dict(out=dict(logit=None))])
def test_refused(other):
    assert _call(**other) == 1 and P.last_error()


def test_alignment_and_empty_calls():
    assert _call(scratch=ONE + 16) == 2 and _call(logits=ONE + 1) == 2 and _call(dtype=0, logits=ONE + 2) == 2
    assert _call(N=0, logits=None, scratch=None, scratch_bytes=0, out=dict(token=None, logit=None)) == 0
    lib = binding.load_library()
    assert lib.saki_top_logits(None, None, ONE, 1, None) == 1
    assert lib.saki_top_scratch_bytes(8, 151936, 64) > 8 * 64 * 8 and lib.saki_top_scratch_bytes(8, 1, 64) == 0 and lib.saki_top_scratch_bytes(0, 100, 1) > 0


def test_tensors_are_checked():
    x = torch.zeros(4, 50)
    for args in ((x.t(), 3), (x, 0), (x, 129), (x[0], 3), (x, 3)):
        with pytest.raises(ValueError):      # the last: not on a GPU
            P.top_logits(*args)
    with pytest.raises(P.SakiError):
        P.top_logits(x.half(), 3)
