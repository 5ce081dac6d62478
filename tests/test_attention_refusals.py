"""Arguments that saki_paged_attention refuses, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer, never followed


def _call(out=ONE, scratch=ONE, scratch_bytes=1 << 40, **other):
    i, o = binding.SakiAttnIn(), binding.SakiAttnOut()
    i.q = i.k_pages = i.v_pages = i.page_table = i.length = ONE
    i.B, i.Q, i.Hq, i.H, i.D, i.page_size, i.max_pages, i.n_pages, i.dtype, i.ld_table, i.scale = 2, 1, 8, 2, 64, 16, 4, 32, 1, 4, 0.125
    i.kp_page = i.vp_page = 16 * 2 * 64
    i.kp_pos = i.vp_pos = 2 * 64
    i.kp_head = i.vp_head = 64
    o.out = out
    for k, v in other.items():
        setattr(i, k, v)
    return binding.load_library().saki_paged_attention(C.byref(i), C.byref(o), scratch, scratch_bytes, None)


@pytest.mark.parametrize("other", [dict(dtype=2), dict(B=-1), dict(B=(1 << 20) + 1), dict(Q=0), dict(Q=33), dict(H=0), dict(Hq=7), dict(Hq=130), dict(D=0),
                                   dict(D=260), dict(D=12), dict(D=2, dtype=0), dict(page_size=0), dict(max_pages=0), dict(n_pages=0), dict(ld_table=3),
                                   dict(max_pages=1 << 20, ld_table=1 << 20, page_size=1 << 11), dict(window=-1), dict(sinks=-1),
                                   dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k_pages=None), dict(v_pages=None),
                                   dict(page_table=None), dict(length=None), dict(out=None), dict(scratch=None), dict(scratch_bytes=1000)])
def test_refused(other):
    assert _call(**other) == 1 and P.last_error()


@pytest.mark.parametrize("other", [dict(k_pages=ONE + 8), dict(v_pages=ONE + 2), dict(kp_pos=129), dict(vp_head=68), dict(kp_page=1), dict(scratch=ONE + 64)])
def test_alignment(other):
    assert _call(**other) == 2 and "16 bytes" in P.last_error()


def test_empty_calls_and_scratch():
    assert _call(B=0, q=None, scratch=None, scratch_bytes=0) == 0
    lib = binding.load_library()
    assert lib.saki_paged_attention(None, None, ONE, 1, None) == 1
    assert lib.saki_paged_attention_scratch_bytes(None) == 0


def test_struct_layouts_match_the_header():
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("saki_attn_in", "saki_attn_out", "saki_beam_in", "saki_beam_out")
    src = '#include <stdio.h>\n#include "saki.h"\nint main(){printf("%s\\n",%s);return 0;}\n' % (
        " ".join(["%zu"] * len(names)), ",".join("sizeof(%s)" % n for n in names))
    with tempfile.TemporaryDirectory() as td:
        c = os.path.join(td, "a.c")
        open(c, "w").write(src)
        exe = os.path.join(td, "a.out")
        subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), c, "-o", exe])
        sizes = [int(v) for v in subprocess.check_output([exe]).split()]
    assert sizes == [C.sizeof(t) for t in (binding.SakiAttnIn, binding.SakiAttnOut, binding.SakiBeamIn, binding.SakiBeamOut)]
