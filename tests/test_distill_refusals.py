"""Arguments that saki_distill_top refuses, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


def _call(scratch=ONE, scratch_bytes=1 << 40, dlogits=ONE, ld_g=1000, grad_scale=1.0, out=None, **other):
    i, o = binding.SakiDistillIn(), binding.SakiDistillOut()
    i.student_logits = i.token = i.logit = i.teacher_lse = o.loss = ONE
    i.N, i.V, i.dtype, i.ld_s, i.ld_k, i.k, i.temperature = 10, 1000, 1, 1000, 16, 16, 1.0
    for k, v in other.items():
        setattr(i, k, v)
    for k, v in (out or {}).items():
        setattr(o, k, v)
    return binding.load_library().saki_distill_top(C.byref(i), C.byref(o), dlogits, ld_g, grad_scale, scratch, scratch_bytes, None)


@pytest.mark.parametrize("other", [dict(N=-1), dict(N=1 << 31), dict(V=1), dict(V=(1 << 22) + 1), dict(dtype=2), dict(k=0), dict(k=129, ld_k=129), dict(ld_k=15), dict(ld_s=999),
                                   dict(ld_g=999), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(grad_scale=float("inf")),
                                   dict(reverse=1, teacher_lse=None), dict(student_logits=None), dict(token=None), dict(logit=None), dict(scratch=None), dict(scratch_bytes=100),
                                   dict(out=dict(loss=None), dlogits=None)])
def test_refused(other):
    assert _call(**other) == 1 and P.last_error()


def test_alignment_and_empty_calls():
    assert _call(scratch=ONE + 16) == 2 and _call(student_logits=ONE + 1) == 2 and _call(dtype=0, dlogits=ONE + 2) == 2
    assert _call(N=0, student_logits=None, token=None, logit=None, scratch=None, scratch_bytes=0) == 0
    lib = binding.load_library()
    assert lib.saki_distill_top(None, None, ONE, 1000, 1.0, ONE, 1, None) == 1
    assert lib.saki_distill_scratch_bytes(4096, 64) > 4096 * 64 * 12 and lib.saki_distill_scratch_bytes(4096, 129) == 0 and lib.saki_distill_scratch_bytes(0, 1) > 0


def test_tensors_are_checked():
    s, token, logit = torch.zeros(4, 50), torch.zeros(4, 8, dtype=torch.int32), torch.zeros(4, 8)
    for args in ((s, token.long(), logit), (s, token[:3], logit), (s, token, logit[:, :7]), (s, token, logit.double()), (s.t(), token, logit), (s, token[:, ::2], logit[:, ::2]),
                 (s, token, torch.zeros(4, 9)[:, :8]), (s, token, logit)):
        with pytest.raises(ValueError):      # the last: not on a GPU
            P.distill_top(*args)
    with pytest.raises(P.SakiError):
        P.distill_top(s.half(), token, logit)
