"""Arguments that the calls around a paged key-value cache refuse, on the host: no GPU is needed, nothing is launched."""
import ctypes as C

import pytest
import torch

import paper_2609_36601_b200 as P
from paper_2609_36601_b200 import binding

ONE = 1 << 20                    # stands in for a pointer: 16-byte aligned, never followed


def _cache(**other):
    c = binding.SakiCache()
    c.page_table = c.length = c.ref_count = c.scratch = ONE
    c.B, c.max_pages, c.n_pages, c.page_size, c.ld_table, c.scratch_bytes = 4, 8, 64, 16, 8, 1 << 20
    for k, v in other.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("other", [dict(B=-1), dict(B=(1 << 20) + 1), dict(max_pages=0), dict(page_size=0), dict(n_pages=0), dict(ld_table=7),
                                   dict(n_pages=(1 << 30) + 1), dict(max_pages=1 << 16, page_size=1 << 15, ld_table=1 << 16), dict(page_table=None),
                                   dict(length=None), dict(ref_count=None)])
def test_every_call_refuses_a_cache_that_is_none(other):
    lib = binding.load_library()
    c = C.byref(_cache(**other))
    kv = binding.SakiCacheKv()
    kv.k = kv.v = kv.k_pages = kv.v_pages = ONE
    kv.Q, kv.H, kv.D, kv.dtype = 1, 1, 8, 1
    assert lib.saki_cache_reserve(c, None, 1, ONE, ONE, None, None) == 1 and P.last_error()
    assert lib.saki_cache_truncate(c, ONE, 0, -1, None, None) == 1
    assert lib.saki_cache_fork(c, ONE, 4, None, None) == 1
    assert lib.saki_cache_compact(c, ONE, ONE, None, None, None) == 1
    assert lib.saki_cache_write(c, C.byref(kv), None) == 1


def test_arguments_of_single_calls():
    lib = binding.load_library()
    ok = C.byref(_cache())
    assert lib.saki_cache_reserve(None, None, 1, ONE, ONE, None, None) == 1
    assert lib.saki_cache_reserve(ok, None, -1, ONE, ONE, None, None) == 1 and "negative" in P.last_error()
    assert lib.saki_cache_reserve(ok, None, 1, None, ONE, None, None) == 1
    assert lib.saki_cache_truncate(ok, None, 0, -1, None, None) == 1
    assert lib.saki_cache_fork(ok, ONE, 0, None, None) == 1
    assert lib.saki_cache_fork(ok, None, 4, None, None) == 1
    assert lib.saki_cache_compact(ok, None, ONE, None, None, None) == 1
    need = lib.saki_cache_scratch_bytes(4, 8, 64)
    assert need >= 4 * (3 * 64 + 4) and lib.saki_cache_scratch_bytes(-1, 8, 64) == 0
    for small in (_cache(scratch_bytes=need - 1), _cache(scratch=None)):
        assert lib.saki_cache_reserve(C.byref(small), None, 1, ONE, ONE, None, None) == 1 and "scratch" in P.last_error()
        assert lib.saki_cache_fork(C.byref(small), ONE, 4, None, None) == 1
        assert lib.saki_cache_compact(C.byref(small), ONE, ONE, None, None, None) == 1
    assert lib.saki_cache_reserve(C.byref(_cache(scratch=ONE + 8)), None, 1, ONE, ONE, None, None) == 2
    empty = C.byref(_cache(B=0, page_table=None, length=None, ref_count=None))
    assert lib.saki_cache_reserve(empty, None, 1, None, None, None, None) == 0          # no sequences: nothing to do
    assert lib.saki_cache_truncate(empty, None, 0, -1, None, None) == 0
    assert lib.saki_cache_fork(empty, None, 4, None, None) == 0


def test_arguments_of_write_and_copy():
    lib = binding.load_library()
    ok = C.byref(_cache())
    for other in (dict(dtype=5), dict(Q=-1), dict(H=0), dict(D=0), dict(Q=1 << 30), dict(H=1 << 13, D=1 << 12), dict(k=None), dict(v_pages=None)):
        kv = binding.SakiCacheKv()
        kv.k = kv.v = kv.k_pages = kv.v_pages = ONE
        kv.Q, kv.H, kv.D, kv.dtype = 1, 1, 8, 1
        for k, v in other.items():
            setattr(kv, k, v)
        assert lib.saki_cache_write(ok, C.byref(kv), None) == 1, other
    assert lib.saki_cache_write(ok, None, None) == 1
    pool, stride, size = (C.c_void_p * 1)(ONE), (C.c_int64 * 1)(64), (C.c_int64 * 1)(64)
    copy = lib.saki_cache_copy_pages
    assert copy(pool, stride, size, 1, None, ONE, 3, 8, None) == 1
    assert copy(pool, stride, size, -1, ONE, ONE, 3, 8, None) == 1
    assert copy(pool, stride, size, 1, ONE, ONE, 3, 0, None) == 1
    assert copy(pool, (C.c_int64 * 1)(32), size, 1, ONE, ONE, 3, 8, None) == 1
    assert copy((C.c_void_p * 1)(None), stride, size, 1, ONE, ONE, 3, 8, None) == 1
    assert copy(pool, stride, size, 1, ONE, ONE, 0, 8, None) == 0
    assert copy(None, None, None, 0, ONE, ONE, 3, 8, None) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    with pytest.raises(ValueError):
        P.PageCache(torch.zeros(10, dtype=torch.int32), 1, 2, 8, 4)              # 11 elements
    with pytest.raises(ValueError):
        P.PageCache(torch.zeros(11), 1, 2, 8, 4)
    cache = P.PageCache.empty(1, 2, 8, 4, "cpu")
    assert cache.page_table.tolist() == [[-1, -1]] and cache.length.tolist() == [0] and cache.ref_count.tolist() == [0] * 8
    with pytest.raises(ValueError, match="GPU"):
        P.cache_reserve(cache, 1)


def test_struct_layouts_match_the_header():
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("saki_cache", "saki_cache_kv")
    src = '#include <stdio.h>\n#include "saki.h"\nint main(){printf("%s\\n",%s);return 0;}\n' % (
        " ".join(["%zu"] * len(names)), ",".join("sizeof(%s)" % n for n in names))
    with tempfile.TemporaryDirectory() as td:
        c = os.path.join(td, "a.c")
        open(c, "w").write(src)
        exe = os.path.join(td, "a.out")
        subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), c, "-o", exe])
        sizes = [int(v) for v in subprocess.check_output([exe]).split()]
    assert sizes == [C.sizeof(binding.SakiCache), C.sizeof(binding.SakiCacheKv)]
