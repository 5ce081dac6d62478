"""Arguments that saki_beam_select refuses, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


def _call(out=None, scratch=ONE, scratch_bytes=1 << 30, **other):
    i, o = binding.SakiBeamIn(), binding.SakiBeamOut()
    i.logits = i.score = o.parent = o.token = o.score = ONE
    i.B, i.W, i.V, i.n, i.dtype, i.pad, i.temperature, i.ld_seq, i.ld_beam = 2, 4, 1000, 4, 1, 0, 1.0, 4000, 1000
    for k, v in other.items():
        setattr(i, k, v)
    for k, v in (out or {}).items():
        setattr(o, k, v)
    return binding.load_library().saki_beam_select(C.byref(i), C.byref(o), scratch, scratch_bytes, None)


@pytest.mark.parametrize("other", [dict(W=0), dict(W=65), dict(n=0), dict(n=65), dict(B=-1), dict(B=1 << 19), dict(V=1), dict(V=(1 << 22) + 1),
                                   dict(dtype=2), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                                   dict(pad=-1), dict(pad=1000), dict(ld_beam=999), dict(ld_seq=-1), dict(logits=None), dict(score=None),
                                   dict(out=dict(parent=None)), dict(out=dict(token=None)), dict(out=dict(score=None)), dict(scratch=None),
                                   dict(scratch_bytes=100)])
def test_refused(other):
    assert _call(**other) == 1 and P.last_error()


def test_alignment_and_empty_calls():
    assert _call(scratch=ONE + 16) == 2
    assert _call(B=0, logits=None, score=None, scratch=None, scratch_bytes=0) == 0
    lib = binding.load_library()
    assert lib.saki_beam_select(None, None, ONE, 1, None) == 1
    assert lib.saki_beam_scratch_bytes(1, 4, 151936, 4) > 0 and lib.saki_beam_scratch_bytes(1, 4, 1, 4) == 0
