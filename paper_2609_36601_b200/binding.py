"""Thin binding of the C-ABI library: argument marshalling only, by ctypes, and for the entry points of a decoding or
training step by the compiled module `_saki_torch` (the same work, without the interpreter's share of it).

Every function takes torch tensors (device memory and streams are torch's),
passes raw pointers, sizes and strides to the library, and returns torch
tensors.  There is no CPU fallback: if the library is missing or cannot be
loaded the first call raises."""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsaki.so")
_lib = None
_fast = None          # the module _saki_torch, bound to the library
_BOUND = ("saki_route_fwd", "saki_route_fwd_bwd", "saki_route_fwd_bwd_noalloc", "saki_route_bwd_from_meta", "saki_select_tm",
          "saki_spec_verify", "saki_sample_proposal", "saki_vshard_stage", "saki_cache_scratch_bytes", "saki_cache_reserve", "saki_cache_truncate",
          "saki_cache_fork", "saki_cache_compact", "saki_cache_copy_pages", "saki_cache_write", "saki_paged_attention_scratch_bytes", "saki_paged_attention",
          "saki_beam_scratch_bytes", "saki_beam_select", "saki_linear_ce_scratch_bytes", "saki_linear_ce_fwd", "saki_linear_ce_bwd", "saki_distill_scratch_bytes", "saki_distill_top", "saki_top_scratch_bytes", "saki_top_logits",
          "saki_last_error")

SAKI_F32, SAKI_BF16 = 0, 1
ROW_SATURATED, ROW_EPS_ZERO, ROW_MASKED, ROW_NONFINITE, ROW_BAD_ID, ROW_TIMEOUT, ROW_NOT_COMPUTED = 1, 2, 4, 8, 16, 32, 64
ROW_BAD_PAGE, ROW_BAD_LENGTH, ROW_NO_PAGES = 128, 256, 512

_FLOAT_FIELDS = ("lambda", "kl", "tv", "accept_prob", "logp_x", "logq_x", "logT_x", "logp_y", "logq_y", "logT_y", "loss")
EXPORTS = ("saki_route_fwd", "saki_route_fwd_bwd", "saki_route_fwd_bwd_noalloc", "saki_route_host",
           "saki_route_bwd_from_meta", "saki_select_tm", "saki_spec_verify",
           "saki_vshard_partial", "saki_vshard_stage", "saki_vshard_combine", "saki_vshard_combine_host",
           "saki_lmhead_scratch_bytes", "saki_lmhead_lse",
           "saki_cache_scratch_bytes", "saki_cache_reserve", "saki_cache_truncate", "saki_cache_fork", "saki_cache_compact",
           "saki_cache_copy_pages", "saki_cache_write", "saki_paged_attention_scratch_bytes", "saki_paged_attention", "saki_beam_scratch_bytes", "saki_beam_select",
           "saki_linear_ce_scratch_bytes", "saki_linear_ce_fwd", "saki_linear_ce_bwd", "saki_distill_scratch_bytes", "saki_distill_top", "saki_top_scratch_bytes", "saki_top_logits",
           "saki_sample_proposal", "saki_check", "saki_set_kernel", "saki_last_kernel", "saki_last_layout", "saki_last_rowsm_layout", "saki_redo_count",
           "saki_set_spec_early_out", "saki_spec_positions_routed", "saki_solve_evaluations", "saki_set_wait_limit", "saki_set_phase_clock", "saki_phase_cycles",
           "saki_launch_count",
           "saki_last_error", "saki_version")


class SakiError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"saki error {code}: {text}")
        self.code = code


class SakiIn(C.Structure):
    _fields_ = [("student_logits", C.c_void_p), ("teacher_logits", C.c_void_p),
                ("ld_s", C.c_int64), ("ld_t", C.c_int64), ("N", C.c_int64),
                ("V", C.c_int32), ("dtype", C.c_int32),
                ("proposal", C.c_void_p), ("mask", C.c_void_p),
                ("eps", C.c_float), ("temperature", C.c_float),
                ("seed", C.c_uint64), ("row_offset", C.c_uint64)]


class SakiOut(C.Structure):
    _fields_ = [("corrected", C.c_void_p), ("token", C.c_void_p), ("teacher_top1", C.c_void_p)] + \
               [(f, C.c_void_p) for f in _FLOAT_FIELDS] + [("row_status", C.c_void_p)]


class SakiMetaIn(C.Structure):
    _fields_ = [("student_logits", C.c_void_p), ("ld_s", C.c_int64), ("N", C.c_int64),
                ("V", C.c_int32), ("dtype", C.c_int32),
                ("corrected", C.c_void_p), ("proposal", C.c_void_p), ("teacher_top1", C.c_void_p),
                ("advantage", C.c_void_p), ("mask", C.c_void_p), ("rollout_status", C.c_void_p),
                ("temperature", C.c_float)]


class SakiMetaOut(C.Structure):
    _fields_ = [("loss", C.c_void_p), ("logp_tok", C.c_void_p), ("row_status", C.c_void_p)]


class SakiSelectIn(C.Structure):
    _fields_ = [("N", C.c_int64), ("B", C.c_int64), ("seq_start", C.c_void_p), ("corrected", C.c_void_p),
                ("tv", C.c_void_p), ("mask", C.c_void_p), ("rollout_status", C.c_void_p), ("mode", C.c_int32),
                ("seed", C.c_uint64), ("row_offset", C.c_uint64)]


class SakiVshardIn(C.Structure):
    _fields_ = [("student_logits", C.c_void_p), ("teacher_logits", C.c_void_p),
                ("ld_s", C.c_int64), ("ld_t", C.c_int64), ("N", C.c_int64),
                ("V", C.c_int32), ("V_local", C.c_int32), ("v0", C.c_int32), ("dtype", C.c_int32),
                ("proposal", C.c_void_p), ("mask", C.c_void_p),
                ("eps", C.c_float), ("temperature", C.c_float),
                ("seed", C.c_uint64), ("row_offset", C.c_uint64),
                ("rank", C.c_int32), ("world", C.c_int32)]


VSHARD_PARTIALS, VSHARD_STATE = 16, 32


class SakiLmheadIn(C.Structure):
    _fields_ = [("hidden", C.c_void_p), ("ld_h", C.c_int64), ("weight", C.c_void_p), ("ld_w", C.c_int64),
                ("N", C.c_int64), ("d", C.c_int32), ("V", C.c_int32), ("temperature", C.c_float)]


class SakiSpecIn(C.Structure):
    _fields_ = [("student_logits", C.c_void_p), ("teacher_logits", C.c_void_p),
                ("ss_seq", C.c_int64), ("ss_pos", C.c_int64), ("ts_seq", C.c_int64), ("ts_pos", C.c_int64),
                ("B", C.c_int64), ("K", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int32),
                ("draft", C.c_void_p), ("draft_ld", C.c_int64),
                ("eps", C.c_float), ("temperature", C.c_float),
                ("seed", C.c_uint64), ("seq_offset", C.c_uint64)]


class SakiSpecOut(C.Structure):
    _fields_ = [("n_accept", C.c_void_p), ("next_token", C.c_void_p), ("next_is_correction", C.c_void_p),
                ("per_pos", SakiOut)]


class SakiCache(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("ld_table", C.c_int64), ("length", C.c_void_p), ("ref_count", C.c_void_p),
                ("scratch", C.c_void_p), ("scratch_bytes", C.c_int64), ("B", C.c_int64),
                ("max_pages", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("row_status", C.c_void_p)]


class SakiCacheKv(C.Structure):
    _fields_ = [("k", C.c_void_p), ("k_seq", C.c_int64), ("k_pos", C.c_int64), ("k_head", C.c_int64),
                ("v", C.c_void_p), ("v_seq", C.c_int64), ("v_pos", C.c_int64), ("v_head", C.c_int64),
                ("k_pages", C.c_void_p), ("kp_page", C.c_int64), ("kp_pos", C.c_int64), ("kp_head", C.c_int64),
                ("v_pages", C.c_void_p), ("vp_page", C.c_int64), ("vp_pos", C.c_int64), ("vp_head", C.c_int64),
                ("Q", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("n_new", C.c_void_p), ("row_status", C.c_void_p)]


class SakiAttnIn(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_seq", C.c_int64), ("q_pos", C.c_int64), ("q_head", C.c_int64),
                ("k_pages", C.c_void_p), ("kp_page", C.c_int64), ("kp_pos", C.c_int64), ("kp_head", C.c_int64),
                ("v_pages", C.c_void_p), ("vp_page", C.c_int64), ("vp_pos", C.c_int64), ("vp_head", C.c_int64),
                ("page_table", C.c_void_p), ("ld_table", C.c_int64), ("length", C.c_void_p), ("n_query", C.c_void_p), ("B", C.c_int64),
                ("Q", C.c_int32), ("Hq", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("page_size", C.c_int32),
                ("max_pages", C.c_int32), ("n_pages", C.c_int32), ("dtype", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32),
                ("scale", C.c_float), ("row_status", C.c_void_p)]


class SakiAttnOut(C.Structure):
    _fields_ = [("out", C.c_void_p), ("o_seq", C.c_int64), ("o_pos", C.c_int64), ("o_head", C.c_int64), ("lse", C.c_void_p),
                ("row_status", C.c_void_p)]


class SakiBeamIn(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("ld_seq", C.c_int64), ("ld_beam", C.c_int64), ("score", C.c_void_p), ("finished", C.c_void_p),
                ("B", C.c_int64), ("W", C.c_int32), ("V", C.c_int32), ("n", C.c_int32), ("dtype", C.c_int32), ("pad", C.c_int32),
                ("temperature", C.c_float)]


class SakiBeamOut(C.Structure):
    _fields_ = [("parent", C.c_void_p), ("token", C.c_void_p), ("score", C.c_void_p), ("row_status", C.c_void_p)]


class SakiLinearIn(C.Structure):
    _fields_ = [("hidden", C.c_void_p), ("ld_h", C.c_int64), ("weight", C.c_void_p), ("ld_w", C.c_int64), ("N", C.c_int64), ("d", C.c_int32), ("V", C.c_int32),
                ("target", C.c_void_p), ("advantage", C.c_void_p), ("corrected", C.c_void_p), ("teacher_top1", C.c_void_p), ("mask", C.c_void_p),
                ("rollout_status", C.c_void_p), ("temperature", C.c_float)]


class SakiLinearOut(C.Structure):
    _fields_ = [("loss", C.c_void_p), ("logp_tok", C.c_void_p), ("lse", C.c_void_p), ("row_status", C.c_void_p)]


class SakiDistillIn(C.Structure):
    _fields_ = [("student_logits", C.c_void_p), ("ld_s", C.c_int64), ("N", C.c_int64), ("V", C.c_int32), ("dtype", C.c_int32), ("token", C.c_void_p),
                ("logit", C.c_void_p), ("ld_k", C.c_int64), ("k", C.c_int32), ("reverse", C.c_int32), ("teacher_lse", C.c_void_p), ("mask", C.c_void_p),
                ("temperature", C.c_float)]


class SakiDistillOut(C.Structure):
    _fields_ = [("loss", C.c_void_p), ("lse", C.c_void_p), ("row_status", C.c_void_p)]


class SakiTopIn(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("ld", C.c_int64), ("N", C.c_int64), ("V", C.c_int32), ("dtype", C.c_int32), ("k", C.c_int32), ("temperature", C.c_float)]


class SakiTopOut(C.Structure):
    _fields_ = [("token", C.c_void_p), ("logit", C.c_void_p), ("lse", C.c_void_p), ("row_status", C.c_void_p)]


def load_library(path: str | None = None):
    """Loads libsaki.so (built in-tree by `python -m paper_2609_36601_b200.build`)."""
    global _lib, _fast
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise SakiError(-1, f"{p} not found: build it with `python -m paper_2609_36601_b200.build`; "
                            "there is no CPU fallback")
    lib = C.CDLL(p)
    lib.saki_route_fwd.argtypes = [C.POINTER(SakiIn), C.POINTER(SakiOut), C.c_void_p]
    lib.saki_route_fwd_bwd.argtypes = [C.POINTER(SakiIn), C.POINTER(SakiOut), C.c_void_p, C.c_int64, C.c_float, C.c_void_p]
    lib.saki_route_fwd_bwd_noalloc.argtypes = lib.saki_route_fwd_bwd.argtypes
    lib.saki_route_fwd_bwd_noalloc.restype = C.c_int
    lib.saki_route_host.argtypes = [C.POINTER(SakiIn), C.POINTER(SakiOut), C.c_void_p, C.c_int64, C.c_float]
    lib.saki_route_bwd_from_meta.argtypes = [C.POINTER(SakiMetaIn), C.POINTER(SakiMetaOut), C.c_void_p, C.c_int64,
                                             C.c_float, C.c_void_p]
    lib.saki_route_bwd_from_meta.restype = C.c_int
    lib.saki_select_tm.argtypes = [C.POINTER(SakiSelectIn), C.c_void_p, C.c_void_p, C.c_void_p]
    lib.saki_select_tm.restype = C.c_int
    lib.saki_spec_verify.argtypes = [C.POINTER(SakiSpecIn), C.POINTER(SakiSpecOut), C.c_void_p]
    lib.saki_sample_proposal.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_float,
                                         C.c_uint64, C.c_uint64, C.c_void_p, C.c_void_p]
    lib.saki_check.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
    lib.saki_set_kernel.argtypes = [C.c_int]
    lib.saki_redo_count.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
    lib.saki_set_spec_early_out.argtypes = [C.c_int]
    lib.saki_set_spec_early_out.restype = C.c_int
    lib.saki_spec_positions_routed.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
    lib.saki_spec_positions_routed.restype = C.c_int
    lib.saki_solve_evaluations.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
    lib.saki_solve_evaluations.restype = C.c_int
    lib.saki_vshard_partial.argtypes = [C.POINTER(SakiVshardIn), C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                        C.c_float, C.c_void_p]
    lib.saki_vshard_partial.restype = C.c_int
    lib.saki_vshard_combine.argtypes = [C.POINTER(SakiVshardIn), C.c_int, C.c_void_p, C.c_void_p, C.POINTER(SakiOut),
                                        C.c_void_p, C.c_void_p]
    lib.saki_vshard_combine.restype = C.c_int
    lib.saki_vshard_combine_host.argtypes = [C.POINTER(SakiVshardIn), C.c_int, C.c_void_p, C.c_void_p, C.POINTER(SakiOut),
                                             C.POINTER(C.c_int32)]
    lib.saki_vshard_combine_host.restype = C.c_int
    lib.saki_lmhead_scratch_bytes.argtypes = [C.c_int64, C.c_int32]
    lib.saki_lmhead_scratch_bytes.restype = C.c_int64
    lib.saki_lmhead_lse.argtypes = [C.POINTER(SakiLmheadIn), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_int64, C.c_void_p]
    lib.saki_lmhead_lse.restype = C.c_int
    lib.saki_cache_scratch_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32]
    lib.saki_cache_scratch_bytes.restype = C.c_int64
    for f, args in (("reserve", [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
                    ("truncate", [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
                    ("fork", [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
                    ("compact", [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
                    ("write", [C.POINTER(SakiCacheKv), C.c_void_p])):
        getattr(lib, "saki_cache_" + f).argtypes = [C.POINTER(SakiCache), *args]
        getattr(lib, "saki_cache_" + f).restype = C.c_int
    lib.saki_cache_copy_pages.argtypes = [C.POINTER(C.c_void_p), C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_int32, C.c_void_p,
                                          C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
    lib.saki_cache_copy_pages.restype = C.c_int
    lib.saki_paged_attention_scratch_bytes.argtypes = [C.POINTER(SakiAttnIn)]
    lib.saki_paged_attention_scratch_bytes.restype = C.c_int64
    lib.saki_paged_attention.argtypes = [C.POINTER(SakiAttnIn), C.POINTER(SakiAttnOut), C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_paged_attention.restype = C.c_int
    lib.saki_beam_scratch_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
    lib.saki_beam_scratch_bytes.restype = C.c_int64
    lib.saki_beam_select.argtypes = [C.POINTER(SakiBeamIn), C.POINTER(SakiBeamOut), C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_beam_select.restype = C.c_int
    lib.saki_linear_ce_scratch_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int]
    lib.saki_linear_ce_scratch_bytes.restype = C.c_int64
    lib.saki_linear_ce_fwd.argtypes = [C.POINTER(SakiLinearIn), C.POINTER(SakiLinearOut), C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_linear_ce_fwd.restype = C.c_int
    lib.saki_linear_ce_bwd.argtypes = [C.POINTER(SakiLinearIn), C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_linear_ce_bwd.restype = C.c_int
    lib.saki_distill_scratch_bytes.argtypes = [C.c_int64, C.c_int32]
    lib.saki_distill_scratch_bytes.restype = C.c_int64
    lib.saki_distill_top.argtypes = [C.POINTER(SakiDistillIn), C.POINTER(SakiDistillOut), C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_distill_top.restype = C.c_int
    lib.saki_top_scratch_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32]
    lib.saki_top_scratch_bytes.restype = C.c_int64
    lib.saki_top_logits.argtypes = [C.POINTER(SakiTopIn), C.POINTER(SakiTopOut), C.c_void_p, C.c_int64, C.c_void_p]
    lib.saki_top_logits.restype = C.c_int
    lib.saki_set_wait_limit.argtypes = [C.c_int64]
    lib.saki_set_wait_limit.restype = C.c_int64
    lib.saki_set_phase_clock.argtypes = [C.c_int]
    lib.saki_set_phase_clock.restype = C.c_int
    lib.saki_phase_cycles.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
    lib.saki_phase_cycles.restype = C.c_int
    lib.saki_last_layout.argtypes = [C.POINTER(C.c_int32)] * 3
    lib.saki_last_layout.restype = None
    lib.saki_last_rowsm_layout.argtypes = [C.POINTER(C.c_int32)] * 2
    lib.saki_last_rowsm_layout.restype = None
    lib.saki_launch_count.restype = C.c_uint64
    lib.saki_last_error.restype = C.c_char_p
    for f in ("saki_route_fwd", "saki_route_fwd_bwd", "saki_route_host", "saki_spec_verify",
              "saki_sample_proposal", "saki_check", "saki_set_kernel", "saki_last_kernel", "saki_redo_count",
              "saki_version"):
        getattr(lib, f).restype = C.c_int
    from . import build
    if os.path.exists(build.TORCH_LIB) and not build.host_matches():
        raise SakiError(-1, f"{build.TORCH_LIB} was built for another torch or Python: build it with "
                            "`python -m paper_2609_36601_b200.build`")
    try:
        from . import _saki_torch
    except ImportError as e:
        raise SakiError(-1, f"_saki_torch: {e}: build it with `python -m paper_2609_36601_b200.build`") from e
    _saki_torch.bind(SakiError, *(C.cast(getattr(lib, f), C.c_void_p).value for f in _BOUND))
    _lib, _fast = lib, _saki_torch
    return lib


def _tensors():
    """The module _saki_torch, bound to the loaded library."""
    if _fast is None:
        load_library()
    return _fast


def _raise(lib, rc):
    if rc != 0:
        raise SakiError(rc, lib.saki_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SAKI_F32
    if t.dtype == torch.bfloat16:
        return SAKI_BF16
    raise SakiError(1, f"unsupported logits dtype {t.dtype}")


def _stream_ptr(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return int(stream.cuda_stream)


def _handle(stream):
    """For _saki_torch: None (torch's current stream) or the stream's handle."""
    return None if stream is None else int(stream.cuda_stream)


def alloc_outputs(n: int, device):
    """Preallocated per-position output tensors for the calls that take `out=`."""
    return _tensors().alloc_outputs(n, device)


def _alloc_pinned(n: int):
    kw = dict(device="cpu", pin_memory=True)
    out = {"corrected": torch.empty(n, dtype=torch.uint8, **kw)}
    out.update((f, torch.empty(n, dtype=torch.int32, **kw)) for f in ("token", "teacher_top1", "row_status"))
    out.update((f, torch.empty(n, dtype=torch.float32, **kw)) for f in _FLOAT_FIELDS)
    return out


def _out_struct(out: dict) -> SakiOut:
    so = SakiOut()
    for name, _ in SakiOut._fields_:
        t = out.get(name)
        setattr(so, name, t.data_ptr() if t is not None else None)
    return so


def _check_rows(s, t):
    if s.dim() != 2 or t.shape != s.shape or t.dtype != s.dtype or s.stride(1) != 1 or t.stride(1) != 1:
        raise SakiError(1, "student/teacher logits must be [N,V] of the same dtype with unit stride along V")


def _in_struct(s, t, proposal, mask, eps, temperature, seed, row_offset) -> SakiIn:
    si = SakiIn()
    si.student_logits, si.teacher_logits = s.data_ptr(), t.data_ptr()
    si.ld_s, si.ld_t = (s.stride(0) if s.shape[0] > 1 else s.shape[1]), (t.stride(0) if t.shape[0] > 1 else t.shape[1])
    si.N, si.V, si.dtype = s.shape[0], s.shape[1], _dtype_code(s)
    si.proposal = proposal.data_ptr()
    si.mask = mask.data_ptr() if mask is not None else None
    si.eps, si.temperature, si.seed, si.row_offset = eps, temperature, seed, row_offset
    return si


def route_fwd(s, t, proposal, eps, temperature=1.0, seed=0, row_offset=0, mask=None, out=None, stream=None):
    """saki_route_fwd on device tensors; returns the dict of per-position output tensors."""
    return (_fast or _tensors()).route(0, s, t, proposal, eps, temperature, seed, row_offset, mask, 1.0, out, None, _handle(stream))


def route_fwd_bwd(s, t, proposal, eps, temperature=1.0, seed=0, row_offset=0, mask=None, grad_scale=1.0,
                  out=None, dlogits=None, stream=None):
    """saki_route_fwd_bwd on device tensors; returns (outputs dict, dlogits)."""
    return (_fast or _tensors()).route(1, s, t, proposal, eps, temperature, seed, row_offset, mask, grad_scale, out, dlogits,
                                       _handle(stream))


def route_bwd_from_meta(s, corrected, proposal, teacher_top1, advantage, temperature=1.0, mask=None,
                        rollout_status=None, grad_scale=1.0, dlogits=None, stream=None):
    """saki_route_bwd_from_meta on device tensors: loss and gradient of the routed objective for the
    current student logits `s`, from the rollout's metadata.  Returns (outputs dict, dlogits)."""
    return (_fast or _tensors()).meta(s, corrected, proposal, teacher_top1, advantage, temperature, mask, rollout_status, grad_scale,
                                      dlogits, _handle(stream))


SELECT_RANDOM, SELECT_TV_WEIGHTED = 0, 1


def select_tm(seq_start, corrected, tv, mode, seed=0, row_offset=0, mask=None, rollout_status=None, stream=None):
    """saki_select_tm on device tensors: the placement controls (Random-TM, TV-Weighted-TM).  `seq_start`
    is the int64 [B+1] tensor of trajectory boundaries.  Returns (selected uint8 [N], m int32 [B])."""
    return (_fast or _tensors()).select(seq_start, corrected, tv, mode, seed, row_offset, mask, rollout_status, _handle(stream))


def route_fwd_bwd_noalloc(s, t, proposal, eps, out, dlogits, temperature=1.0, seed=0, row_offset=0, mask=None,
                          grad_scale=1.0, stream=None):
    """saki_route_fwd_bwd_noalloc: the variant for callers that cannot allocate device memory.  The caller
    passes every buffer (`out`: dict of preallocated output tensors, `dlogits`); the library's own scratch
    is a fixed device array, so nothing is allocated on the way (at most 1,048,576 rows per call)."""
    return (_fast or _tensors()).route(2, s, t, proposal, eps, temperature, seed, row_offset, mask, grad_scale, out, dlogits,
                                       _handle(stream))


def vshard_in(s_loc, t_loc, v0, V, proposal, eps, temperature=1.0, seed=0, row_offset=0, mask=None, rank=0, world=1,
              dtype=None, n_rows=None) -> SakiVshardIn:
    """The argument record of the vocabulary-sharded calls: this rank's columns [v0, v0 + V_local) of both logit
    tensors.  `s_loc` / `t_loc` may be None for the host-side combine (which reads no logits); then `dtype`
    ("bf16" / "f32") and `n_rows` say what the slices hold."""
    si = SakiVshardIn()
    if s_loc is not None:
        si.student_logits, si.teacher_logits = s_loc.data_ptr(), t_loc.data_ptr()
        si.ld_s = s_loc.stride(0) if s_loc.shape[0] > 1 else max(1, s_loc.shape[1])
        si.ld_t = t_loc.stride(0) if t_loc.shape[0] > 1 else max(1, t_loc.shape[1])
        si.N, si.V_local, si.dtype = s_loc.shape[0], s_loc.shape[1], _dtype_code(s_loc)
    else:
        si.N, si.V_local, si.dtype = n_rows, 0, (SAKI_BF16 if dtype == "bf16" else SAKI_F32)
    si.V, si.v0 = V, v0
    si.proposal = proposal.data_ptr()
    si.mask = mask.data_ptr() if mask is not None else None
    si.eps, si.temperature, si.seed, si.row_offset = eps, temperature, seed, row_offset
    si.rank, si.world = rank, world
    return si


def vshard_partial(si: SakiVshardIn, stage: int, state, partial, dlogits=None, grad_scale=1.0, stream=None):
    """saki_vshard_partial: this rank's partial vectors of one stage (device tensors, float64)."""
    lib = load_library()
    ld_g = 0
    if dlogits is not None:
        ld_g = dlogits.stride(0) if dlogits.shape[0] > 1 else max(1, dlogits.shape[1])
    _raise(lib, lib.saki_vshard_partial(C.byref(si), stage, state.data_ptr() if state is not None else None,
                                        partial.data_ptr(), dlogits.data_ptr() if dlogits is not None else None, ld_g,
                                        grad_scale, _stream_ptr(stream)))


def vshard_combine(si: SakiVshardIn, stage: int, gathered, state, out=None, n_solving=None, stream=None):
    """saki_vshard_combine: folds the gathered partials [world, N, 16] into the per-row state (device tensors)."""
    lib = load_library()
    so = _out_struct(out) if out is not None else None
    _raise(lib, lib.saki_vshard_combine(C.byref(si), stage, gathered.data_ptr(), state.data_ptr(),
                                        C.byref(so) if so is not None else None,
                                        n_solving.data_ptr() if n_solving is not None else None, _stream_ptr(stream)))


def vshard_combine_host(si: SakiVshardIn, stage: int, gathered, state, out=None) -> int:
    """saki_vshard_combine_host: the same combine on host tensors; returns the number of rows still solving."""
    lib = load_library()
    so = _out_struct(out) if out is not None else None
    n = C.c_int32(0)
    _raise(lib, lib.saki_vshard_combine_host(C.byref(si), stage, gathered.data_ptr(), state.data_ptr(),
                                             C.byref(so) if so is not None else None, C.byref(n)))
    return int(n.value)


def lmhead_lse(hidden, weight, temperature=1.0, logits=None, scratch=None, stream=None):
    """saki_lmhead_lse: logits = hidden @ weight.T (bf16 in, fp32 accumulation, bf16 out) with each row's maximum and
    log-sum-exp (of the stored bf16 values / temperature) from the GEMM's epilogue.  hidden [N, d], weight [V, d] on
    the GPU.  Returns (logits, row_max, lse)."""
    lib = load_library()
    if hidden.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16 or hidden.shape[1] != weight.shape[1]:
        raise ValueError("hidden [N, d] and weight [V, d] must be bf16 with the same d")
    if hidden.stride(1) != 1 or weight.stride(1) != 1:
        raise ValueError("hidden and weight need unit stride along d")
    N, d = hidden.shape
    V = weight.shape[0]
    dev = hidden.device
    logits = logits if logits is not None else torch.empty((N, V), dtype=torch.bfloat16, device=dev)
    need = int(lib.saki_lmhead_scratch_bytes(N, V))
    if scratch is None or scratch.numel() * scratch.element_size() < need:
        scratch = torch.empty(need, dtype=torch.uint8, device=dev)
    row_max = torch.empty(N, dtype=torch.float32, device=dev)
    lse = torch.empty(N, dtype=torch.float32, device=dev)
    li = SakiLmheadIn()
    li.hidden, li.ld_h = hidden.data_ptr(), (hidden.stride(0) if N > 1 else d)
    li.weight, li.ld_w = weight.data_ptr(), (weight.stride(0) if V > 1 else d)
    li.N, li.d, li.V, li.temperature = N, d, V, temperature
    ld_l = logits.stride(0) if N > 1 else V
    _raise(lib, lib.saki_lmhead_lse(C.byref(li), logits.data_ptr(), ld_l, row_max.data_ptr(), lse.data_ptr(),
                                    scratch.data_ptr(), scratch.numel() * scratch.element_size(), _stream_ptr(stream)))
    return logits, row_max, lse


def linear_ce(hidden, weight, target, advantage=None, corrected=None, teacher_top1=None, mask=None, rollout_status=None, temperature=1.0, stream=None):
    """saki_linear_ce_fwd: the loss -coef log softmax(hidden @ weight.T / temperature)[tok] of every row, without its logits in memory.
    hidden [N, d], weight [V, d] bf16, target int32 [N].  (coef, tok) is (1, target), with `advantage` (float32) (advantage, target), and where
    `corrected` (uint8, with `teacher_top1` int32) is set (1, teacher_top1): pass the metadata of a routing call, its proposals as targets.  Rows with mask 0 or
    an unusable rollout_status contribute nothing and cost nothing.  Returns a dict of loss, logp_tok, lse (float32 [N]) and row_status (int32 [N])."""
    loss, logp, lse, status = (_fast or _tensors()).linear(hidden, weight, target, advantage, corrected, teacher_top1, mask, rollout_status, temperature, _handle(stream))
    return {"loss": loss, "logp_tok": logp, "lse": lse, "row_status": status}


def linear_ce_bwd(hidden, weight, target, lse, advantage=None, corrected=None, teacher_top1=None, mask=None, rollout_status=None, temperature=1.0,
                  grad_scale=1.0, dhidden=True, dweight=True, stream=None):
    """saki_linear_ce_bwd: the gradients of grad_scale times the sum of linear_ce's losses with respect to `hidden` and `weight`, bf16.  `lse` is what
    linear_ce returned, the other arguments are those of that call.  dhidden, dweight: a tensor to write to, True (a new one) or None (not wanted).
    Returns (dhidden, dweight)."""
    return (_fast or _tensors()).linear_bwd(hidden, weight, target, advantage, corrected, teacher_top1, mask, rollout_status, temperature, lse, grad_scale,
                                            dhidden, dweight, _handle(stream))


def top_logits(logits, k, temperature=1.0, stream=None):
    """saki_top_logits: the k largest logits of every row of `logits` [N, V], largest first, of equal ones the lowest token first.  Returns a dict of token (int32
    [N, k]; -1: no more that are not masked by -inf), logit (float32 [N, k], -inf there), lse (float32 [N], log sum exp(logits / temperature)) and row_status (int32 [N]):
    of a teacher's rows, what distill_top takes.  No gradient."""
    token, logit, lse, status = (_fast or _tensors()).top(logits, k, temperature, _handle(stream))
    return {"token": token, "logit": logit, "lse": lse, "row_status": status}


def distill_top(s, token, logit, teacher_lse=None, reverse=False, temperature=1.0, mask=None, grad_scale=1.0, dlogits=True, stream=None):
    """saki_distill_top: divergence between a teacher of which a list of top logits is known (top_logits' token int32 and logit float32 [N, k], token -1: no
    entry) and the student's rows s [N, V], with its gradient.  With `teacher_lse` (float32 [N]) the tokens outside the list are one event, without it the list
    is all there is.  reverse: KL(student || teacher) instead of KL(teacher || student); needs teacher_lse.  dlogits: a tensor to write to, True (a new
    one) or None (the loss alone).  Returns (dict of loss, lse of the student's rows, row_status; dlogits)."""
    loss, lse, status, g = (_fast or _tensors()).distill(s, token, logit, teacher_lse, reverse, temperature, mask, grad_scale, dlogits, _handle(stream))
    return {"loss": loss, "lse": lse, "row_status": status}, g


def route_host(s, t, proposal, eps, temperature=1.0, seed=0, row_offset=0, mask=None, grad_scale=1.0,
               backward=True, out=None, dlogits=None):
    """saki_route_host: every tensor lives in HOST memory (pinned for full copy speed); the library
    stages the rows through the GPU and returns when the host outputs are complete."""
    lib = load_library()
    _check_rows(s, t)
    if s.is_cuda:
        raise SakiError(1, "route_host takes host tensors")
    out = out if out is not None else _alloc_pinned(s.shape[0])
    if backward and dlogits is None:
        dlogits = torch.empty(s.shape, dtype=s.dtype, pin_memory=True)
    ld_g = (dlogits.stride(0) if dlogits.shape[0] > 1 else dlogits.shape[1]) if backward else 0
    si, so = _in_struct(s, t, proposal, mask, eps, temperature, seed, row_offset), _out_struct(out)
    _raise(lib, lib.saki_route_host(C.byref(si), C.byref(so), dlogits.data_ptr() if backward else None, ld_g,
                                    grad_scale))
    return out, dlogits


def spec_verify(s, t, draft, eps, temperature=1.0, seed=0, seq_offset=0, stream=None):
    """saki_spec_verify on device tensors s, t: [B,K+1,V], draft: [B,K] int32.  (`per_pos["loss"]` is not written: block
    verification has no loss.)"""
    return (_fast or _tensors()).spec(s, t, draft, eps, temperature, seed, seq_offset, _handle(stream))


def sample_proposal(s, temperature=1.0, seed=0, row_offset=0, stream=None):
    """saki_sample_proposal: x_i ~ softmax(s_i / temperature) by Philox-keyed Gumbel-max."""
    return (_fast or _tensors()).propose(s, temperature, seed, row_offset, _handle(stream))


def beam_select(logits, score, n, temperature=1.0, finished=None, pad=0, stream=None):
    """saki_beam_select: the n best continuations of every group of beams.  logits [B, W, V], score float32 [B, W] (sums of
    log-probabilities so far), finished uint8 [B, W] or None: such a beam goes on with the token `pad` and its own score.  Returns
    a dict of parent, token (int32 [B, n]), score (float32 [B, n]) and row_status (int32 [B, W]).  No gradient."""
    parent, token, best, status = (_fast or _tensors()).beams(logits, score, n, temperature, finished, pad, _handle(stream))
    return {"parent": parent, "token": token, "score": best, "row_status": status}


class PageCache:
    """Page tables, lengths and counts of holders of a paged key-value cache (saki_cache), in one int32 tensor `meta` on the GPU:
    `page_table` [B, max_pages], `length` [B] and `ref_count` [n_pages] are views of it.  `PageCache.empty` makes one without
    positions.  The pools that hold keys and values, [n_pages, page_size, H, D] each, are the caller's, a pair per layer."""
    __slots__ = ("meta", "B", "max_pages", "n_pages", "page_size")

    def __init__(self, meta, B, max_pages, n_pages, page_size):
        if meta.dtype != torch.int32 or not meta.is_contiguous() or meta.numel() != B * max_pages + B + n_pages:
            raise ValueError("a cache's tables must be a contiguous int32 tensor of B * max_pages + B + n_pages elements")
        self.meta, self.B, self.max_pages, self.n_pages, self.page_size = meta, B, max_pages, n_pages, page_size

    @classmethod
    def empty(cls, B, max_pages, n_pages, page_size, device):
        meta = torch.zeros(B * max_pages + B + n_pages, dtype=torch.int32, device=device)
        meta[:B * max_pages] = -1
        return cls(meta, B, max_pages, n_pages, page_size)

    @property
    def page_table(self):
        return self.meta.as_strided((self.B, self.max_pages), (self.max_pages, 1))

    @property
    def length(self):
        return self.meta.as_strided((self.B,), (1,), self.meta.storage_offset() + self.B * self.max_pages)

    @property
    def ref_count(self):
        return self.meta.as_strided((self.n_pages,), (1,), self.meta.storage_offset() + self.B * (self.max_pages + 1))

    def clone(self):
        """Another cache with the same tables, on the same pools."""
        return PageCache(self.meta.clone(), self.B, self.max_pages, self.n_pages, self.page_size)

    def _args(self):
        return self.meta, self.B, self.max_pages, self.n_pages, self.page_size


def cache_reserve(cache, n_new, stream=None):
    """saki_cache_reserve: n_new (an int, or an int32 tensor [B]) more positions for every sequence of a PageCache.  Returns
    (copy_src, copy_dst, row_status), int32 [B]: pass the lists to copy_pages before anything is written (where the cache was forked),
    the status to cache_write."""
    return (_fast or _tensors()).cache_reserve(*cache._args(), n_new, _handle(stream))


def cache_write(cache, k, v, k_pages, v_pages, row_status=None, n_new=None, stream=None):
    """saki_cache_write: k, v [B, Q, H, D] become the last Q (n_new[b]) positions of the sequences in one layer's pools
    [n_pages, page_size, H, D].  Sequences that row_status (of cache_reserve) flags are passed over."""
    (_fast or _tensors()).cache_write(*cache._args(), k, v, k_pages, v_pages, row_status, n_new, _handle(stream))


def cache_truncate(cache, keep, of=None, keep_add=0, stream=None, row_status=None):
    """saki_cache_truncate: sequence b keeps the first keep[b] + keep_add (int32 [B]) of its last `of` positions, or of all of
    them (None).  cache_truncate(cache, verdict["n_accept"], of=K + 1, keep_add=1, row_status=status) commits a verified block: sequences that
    row_status (of cache_reserve) flags did not get those positions and are passed over.  Returns row_status."""
    return (_fast or _tensors()).cache_truncate(*cache._args(), keep, keep_add, -1 if of is None else of, row_status, _handle(stream))


def cache_fork(cache, parent, group=None, stream=None):
    """saki_cache_fork: every sequence takes the pages of its parent (int32, B elements), counted within groups of `group`
    sequences (None: all of them).  Returns row_status."""
    return (_fast or _tensors()).cache_fork(*cache._args(), parent, max(1, cache.B) if group is None else group, _handle(stream))


def cache_compact(cache, stream=None, return_status=False):
    """saki_cache_compact: the used pages move to the lowest ids.  Returns (copy_src, copy_dst, n_moves), with return_status row_status
    (int32 [B]) behind them: pass the lists to copy_pages before the cache is used again."""
    found = (_fast or _tensors()).cache_compact(*cache._args(), _handle(stream))
    return found if return_status else found[:3]


def copy_pages(pools, copy_src, copy_dst, stream=None):
    """saki_cache_copy_pages: page copy_src[i] to page copy_dst[i] (int32; -1: none) in every pool of the sequence `pools`,
    tensors [n_pages, ...] of any strides.  (64 runs of memory go into a launch: a page is one, unless heads or positions are outermost or its rows lie apart.)"""
    (_fast or _tensors()).copy_pages(pools, copy_src, copy_dst, _handle(stream))


def paged_attention(q, k_pages, v_pages, page_table, length, scale=None, window=0, sinks=0, n_query=None, out=None, stream=None, row_status=None):
    """saki_paged_attention: attention of the last Q (n_query[b], int32) positions of every sequence over a paged cache.  q [B, Q, Hq, D],
    pools [n_pages, page_size, H, D] of its type, page_table int32 [B, max_pages], length int32 [B] (a PageCache's), scale 1 / sqrt(D)
    where None; window > 0: only the last `window` positions and the first `sinks` are seen.  Sequences that row_status (of cache_reserve) flags
    have not got their new positions: out 0, lse -inf.  No gradient: what it returns is apart from the graph of its inputs.  Returns (out like q, lse float32
    [B, Q, Hq], row_status int32 [B])."""
    return (_fast or _tensors()).attention(q, k_pages, v_pages, page_table, length, scale, window, sinks, n_query, out, row_status, _handle(stream))


def check(stream=None) -> int:
    """saki_check: synchronises the stream and returns the number of rows flagged since the last check."""
    lib = load_library()
    n = C.c_uint64(0)
    rc = lib.saki_check(_stream_ptr(stream), C.byref(n))
    if rc not in (0, 4):
        _raise(lib, rc)
    return int(n.value)


def set_kernel(which: int) -> int:
    """saki_set_kernel: 0 automatic, 1 general (float64), 2 cluster, 3 row-per-SM; returns the previous choice."""
    return load_library().saki_set_kernel(which)


def last_kernel() -> int:
    """The kernel that served the calling thread's last routing call: 1 general (float64), 2 cluster, 3 row-per-SM,
    4 the streaming kernel of route_bwd_from_meta."""
    return load_library().saki_last_kernel()


def last_layout():
    """(blocks per row, blocks per SM, rows resident at once) of the calling thread's last call that the general kernel served."""
    n = (C.c_int32 * 3)()
    load_library().saki_last_layout(*(C.cast(C.byref(n, 4 * k), C.POINTER(C.c_int32)) for k in range(3)))
    return tuple(n)


def last_rowsm_layout():
    """(blocks per row, blocks per SM) of the calling thread's last routing call if the row-per-SM kernel served it, else zeros."""
    n = (C.c_int32 * 2)()
    load_library().saki_last_rowsm_layout(*(C.cast(C.byref(n, 4 * k), C.POINTER(C.c_int32)) for k in range(2)))
    return tuple(n)


def redo_count(stream=None) -> int:
    """Rows of the last routing call that the float32 kernel handed to the float64 kernel (synchronises)."""
    lib = load_library()
    n = C.c_uint64(0)
    _raise(lib, lib.saki_redo_count(_stream_ptr(stream), C.byref(n)))
    return int(n.value)


def solve_evaluations(stream=None) -> int:
    """Evaluation passes of the row-per-SM kernel in the last routing call, over all rows (synchronises)."""
    lib = load_library()
    n = C.c_uint64(0)
    _raise(lib, lib.saki_solve_evaluations(_stream_ptr(stream), C.byref(n)))
    return int(n.value)


PHASES = ("row_top", "copy_wait", "lse", "lse_reduce", "lse_gather", "lse_scalar", "solve_top", "solve",
          "solve_combine", "solve_scalar", "final_top", "final", "row_end", "tail", "spare", "rows")


def set_wait_limit(cycles: int) -> int:
    """SM cycles a block of the row-per-SM kernel waits for a row's bulk copy, and one of either that or the general kernel for
    its next row, before it flags rows TIMEOUT (0: the default of about two seconds); returns the previous setting."""
    return int(load_library().saki_set_wait_limit(int(cycles)))


def set_phase_clock(on: bool) -> bool:
    """Phase clock of the row-per-SM kernel for the calls that follow (default off); returns the previous setting."""
    return bool(load_library().saki_set_phase_clock(1 if on else 0))


def phase_cycles(stream=None) -> dict:
    """SM cycles per phase of the row-per-SM kernel's row loop in the last routing call, summed over thread
    blocks, and the number of rows behind them (synchronises)."""
    lib = load_library()
    buf = (C.c_uint64 * len(PHASES))()
    _raise(lib, lib.saki_phase_cycles(_stream_ptr(stream), buf))
    return {k: int(v) for k, v in zip(PHASES, buf)}


def set_spec_early_out(on: bool) -> bool:
    """Early out of block verification on the row-per-SM kernel (default on); returns the previous setting."""
    return bool(load_library().saki_set_spec_early_out(1 if on else 0))


def spec_positions_routed(stream=None) -> int:
    """Positions the last spec_verify actually routed under early out (synchronises); 0 without early out."""
    lib = load_library()
    n = C.c_uint64(0)
    _raise(lib, lib.saki_spec_positions_routed(_stream_ptr(stream), C.byref(n)))
    return int(n.value)


def launch_count() -> int:
    return int(load_library().saki_launch_count())


def last_error() -> str:
    return load_library().saki_last_error().decode()


def version() -> int:
    return load_library().saki_version()
