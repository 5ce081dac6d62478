// The tensor side of the Python binding: argument checks, output tensors, argument records and the call into the C ABI
// for the entry points whose kernels take no longer than that work takes in Python (a forward call on eight rows: 34 us of
// host time through ctypes and fifteen torch.empty calls, against 25 us on the GPU).  No arithmetic: binding.py holds the
// signatures and documentation, libsaki.so the library, whose functions are handed over by address (bind).
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/cuda/CUDAEvent.h>
#include <ATen/ops/empty_native.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <algorithm>
#include <cmath>
#include <string>
#include <utility>
#include <vector>
#include "../../include/saki.h"

namespace {

struct Lib {
  decltype(&saki_route_fwd) route_fwd;
  decltype(&saki_route_fwd_bwd) route_fwd_bwd;
  decltype(&saki_route_fwd_bwd_noalloc) route_fwd_bwd_noalloc;
  decltype(&saki_route_bwd_from_meta) route_bwd_from_meta;
  decltype(&saki_select_tm) select_tm;
  decltype(&saki_spec_verify) spec_verify;
  decltype(&saki_sample_proposal) sample_proposal;
  decltype(&saki_vshard_stage) vshard_stage;
  decltype(&saki_cache_scratch_bytes) cache_scratch_bytes;
  decltype(&saki_cache_reserve) cache_reserve;
  decltype(&saki_cache_truncate) cache_truncate;
  decltype(&saki_cache_fork) cache_fork;
  decltype(&saki_cache_compact) cache_compact;
  decltype(&saki_cache_copy_pages) cache_copy_pages;
  decltype(&saki_cache_write) cache_write;
  decltype(&saki_paged_attention_scratch_bytes) paged_attention_scratch_bytes;
  decltype(&saki_paged_attention) paged_attention;
  decltype(&saki_beam_scratch_bytes) beam_scratch_bytes;
  decltype(&saki_beam_select) beam_select;
  decltype(&saki_last_error) last_error;
};
Lib lib = {};
PyObject* saki_error = nullptr;     // the exception class

constexpr int N_FIELDS = 15;
// saki_out's members, in order
const char* const FIELD[N_FIELDS] = {"corrected", "token", "teacher_top1", "lambda", "kl", "tv", "accept_prob", "logp_x", "logq_x",
                                     "logT_x", "logp_y", "logq_y", "logT_y", "loss", "row_status"};
// ... and in the order in which the output dict lists them
const int DICT_ORDER[N_FIELDS] = {0, 1, 2, 14, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13};
PyObject* field_key[N_FIELDS];
PyObject *key_loss, *key_logp_tok, *key_row_status, *key_n_accept, *key_next_token, *key_next_is_correction, *key_per_pos;

struct Raised {};     // a Python exception is set
[[noreturn]] void raise_saki(int code, const char* text) {
  PyObject* e = PyObject_CallFunction(saki_error, "is", code, text);
  if (e) { PyErr_SetObject(saki_error, e); Py_DECREF(e); }
  throw Raised();
}
[[noreturn]] void raise_value(const std::string& text) {
  PyErr_SetString(PyExc_ValueError, text.c_str());
  throw Raised();
}
void check_rc(int rc) { if (rc != 0) raise_saki(rc, lib.last_error()); }

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
    throw Raised();
  }
  return THPVariable_Unpack(o);
}
void* ptr_or_null(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}
uint64_t word(PyObject* o) {       // as a 64-bit field takes an int: the low bits
  const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (uint64_t)-1 && PyErr_Occurred()) throw Raised();
  return v;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
void* stream_of(PyObject* o) {     // None: torch's current stream; else the handle
  if (o == Py_None) return (void*)c10::cuda::getCurrentCUDAStream().stream();
  return (void*)word(o);
}
int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return SAKI_F32;
  if (t.scalar_type() == at::kBFloat16) return SAKI_BF16;
  raise_saki(1, (std::string("unsupported logits dtype ") + c10::toString(t.scalar_type())).c_str());
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, at::Device dev) {
  // on a GPU the function that the dispatcher would end up in: a call on eight rows, fifteen fields, is about as long as its
  // kernels (17.6 us) with it, 18.1 us, and takes 21.5 us through the dispatcher
  if (dev.is_cuda()) return at::native::empty_cuda(sizes, type, std::nullopt, dev, std::nullopt, std::nullopt);
  return at::empty(sizes, at::TensorOptions().dtype(type).device(dev));
}
at::ScalarType field_type(int k) { return k == 0 ? at::kByte : (k <= 2 || k == 14) ? at::kInt : at::kFloat; }

struct Owned {            // a reference of our own
  PyObject* p;
  explicit Owned(PyObject* o) : p(o) { if (!p) throw Raised(); }
  ~Owned() { Py_XDECREF(p); }
  Owned(const Owned&) = delete;
  PyObject* release() { PyObject* o = p; p = nullptr; return o; }
};
void put(PyObject* dict, PyObject* key, const at::Tensor& t) {
  Owned v(THPVariable_Wrap(t));
  if (PyDict_SetItem(dict, key, v.p) < 0) throw Raised();
}

// The per-position outputs as a dict of tensors, and their record (so may be NULL).  A tensor of its own per field, in the
// dict's order: pieces of one allocation would tie a field that a caller keeps to the fourteen others, could not be saved
// (torch.save refuses one storage under several types), and grow into one another where one is resized.
PyObject* alloc_outputs(int64_t n, at::Device dev, saki_out* so) {
  Owned d(PyDict_New());
  void** const m = (void**)so;
  for (int k : DICT_ORDER) {
    const at::Tensor f = empty({n}, field_type(k), dev);
    put(d.p, field_key[k], f);
    if (so) m[k] = f.data_ptr();
  }
  return d.release();
}
static_assert(sizeof(saki_out) == N_FIELDS * sizeof(void*), "saki_out is fifteen pointers in FIELD's order");

void out_record(PyObject* out, saki_out* so) {
  void** const m = (void**)so;
  for (int k = 0; k < N_FIELDS; ++k) {
    m[k] = nullptr;
    if (PyDict_Check(out)) {
      PyObject* const v = PyDict_GetItemWithError(out, field_key[k]);
      if (!v && PyErr_Occurred()) throw Raised();
      if (v) m[k] = ptr_or_null(v);
    } else {
      Owned v(PyObject_CallMethod(out, "get", "O", field_key[k]));
      m[k] = ptr_or_null(v.p);
    }
  }
}

struct Unlocked {      // without the interpreter lock while it lives, however its scope is left
  PyThreadState* const save = PyEval_SaveThread();
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(save); }
};
template <typename F> auto unlocked(F&& call) {      // a call that may take long or wait
  const Unlocked u;
  return call();
}
template <typename F> PyObject* guarded(F&& body) {  // what torch raises becomes the Python exception that torch makes of it
  HANDLE_TH_ERRORS
  try { return body(); }
  catch (const Raised&) { return nullptr; }
  END_HANDLE_TH_ERRORS
}
void n_args(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) { PyErr_Format(PyExc_TypeError, "%zd arguments, got %zd", want, got); throw Raised(); }
}

// bind(SakiError, address of each function of Lib in order)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    constexpr Py_ssize_t N_LIB = sizeof(Lib) / sizeof(void*);
    n_args(n, 1 + N_LIB);
    Py_INCREF(a[0]);
    Py_XSETREF(saki_error, a[0]);
    void** const f = (void**)&lib;
    for (Py_ssize_t k = 0; k < N_LIB; ++k) f[k] = (void*)word(a[1 + k]);
    Py_RETURN_NONE;
  });
}

// alloc_outputs(n, device)
PyObject* py_alloc_outputs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 2);
    if (PyLong_Check(a[1])) return alloc_outputs(integer(a[0]), at::Device(at::kCUDA, (c10::DeviceIndex)integer(a[1])), nullptr);
    Owned text(PyObject_Str(a[1]));
    return alloc_outputs(integer(a[0]), at::Device(PyUnicode_AsUTF8(text.p)), nullptr);
  });
}

// route(mode, s, t, proposal, eps, temperature, seed, row_offset, mask, grad_scale, out, dlogits, stream)
// mode 0: saki_route_fwd -> out; 1: saki_route_fwd_bwd, 2: saki_route_fwd_bwd_noalloc -> (out, dlogits)
PyObject* py_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 13);
    const int64_t mode = integer(a[0]);
    const at::Tensor &s = tensor(a[1]), &t = tensor(a[2]);
    if (s.dim() != 2 || !t.sizes().equals(s.sizes()) || t.scalar_type() != s.scalar_type() || s.stride(1) != 1 || t.stride(1) != 1)
      raise_saki(1, "student/teacher logits must be [N,V] of the same dtype with unit stride along V");
    saki_in si = {};
    si.student_logits = s.data_ptr(); si.teacher_logits = t.data_ptr();
    si.ld_s = row_stride(s); si.ld_t = row_stride(t);
    si.N = s.size(0); si.V = (int32_t)s.size(1); si.dtype = dtype_code(s);
    si.proposal = (const int32_t*)tensor(a[3]).data_ptr();
    si.eps = (float)number(a[4]); si.temperature = (float)number(a[5]);
    si.seed = word(a[6]); si.row_offset = word(a[7]);
    si.mask = (const uint8_t*)ptr_or_null(a[8]);
    saki_out so;
    PyObject* out_obj = a[10];
    if (out_obj == Py_None) out_obj = alloc_outputs(si.N, s.device(), &so);
    else { Py_INCREF(out_obj); out_record(out_obj, &so); }
    Owned out(out_obj);
    void* const st = stream_of(a[12]);
    if (mode == 0) {
      check_rc(unlocked([&] { return lib.route_fwd(&si, &so, st); }));
      return out.release();
    }
    const float gs = (float)number(a[9]);
    at::Tensor g = a[11] == Py_None ? at::empty_like(s) : tensor(a[11]);
    const int64_t ld_g = row_stride(g);
    void* const gp = g.data_ptr();
    check_rc(unlocked([&] { return (mode == 1 ? lib.route_fwd_bwd : lib.route_fwd_bwd_noalloc)(&si, &so, gp, ld_g, gs, st); }));
    Owned go(a[11] == Py_None ? THPVariable_Wrap(g) : Py_NewRef(a[11]));
    return PyTuple_Pack(2, out.p, go.p);
  });
}

const void* vector(PyObject* o, at::ScalarType type, int64_t n, at::Device dev, const char* name) {
  const at::Tensor& v = tensor(o);
  if (v.scalar_type() != type || v.dim() != 1 || v.size(0) != n || v.device() != dev || !v.is_contiguous())
    raise_value(std::string(name) + " must be a contiguous " +
                (type == at::kByte ? "torch.uint8" : type == at::kInt ? "torch.int32" : "torch.float32") +
                " tensor of length N on the logits' device");
  return v.data_ptr();
}

// meta(s, corrected, proposal, teacher_top1, advantage, temperature, mask, rollout_status, grad_scale, dlogits, stream)
PyObject* py_meta(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 11);
    const at::Tensor& s = tensor(a[0]);
    if (s.dim() != 2 || s.stride(1) != 1) raise_value("logits must be [N,V] with unit stride along V");
    const int64_t N = s.size(0);
    const at::Device dev = s.device();
    at::Tensor g = a[9] == Py_None ? at::empty_like(s) : tensor(a[9]);
    saki_meta_in mi = {};
    mi.student_logits = s.data_ptr(); mi.ld_s = row_stride(s); mi.N = N; mi.V = (int32_t)s.size(1);
    mi.corrected = (const uint8_t*)vector(a[1], at::kByte, N, dev, "corrected");
    mi.proposal = (const int32_t*)vector(a[2], at::kInt, N, dev, "proposal");
    mi.teacher_top1 = (const int32_t*)vector(a[3], at::kInt, N, dev, "teacher_top1");
    mi.advantage = (const float*)vector(a[4], at::kFloat, N, dev, "advantage");
    mi.dtype = dtype_code(s);
    if (a[6] != Py_None) mi.mask = (const uint8_t*)vector(a[6], at::kByte, N, dev, "mask");
    if (a[7] != Py_None) mi.rollout_status = (const uint32_t*)vector(a[7], at::kInt, N, dev, "rollout_status");
    mi.temperature = (float)number(a[5]);
    const float gs = (float)number(a[8]);
    const at::Tensor loss = empty({N}, at::kFloat, dev), logp = empty({N}, at::kFloat, dev), status = empty({N}, at::kInt, dev);
    saki_meta_out mo = {(float*)loss.data_ptr(), (float*)logp.data_ptr(), (uint32_t*)status.data_ptr()};
    void* const st = stream_of(a[10]);
    void* const gp = g.data_ptr();
    const int64_t ld_g = row_stride(g);
    check_rc(unlocked([&] { return lib.route_bwd_from_meta(&mi, &mo, gp, ld_g, gs, st); }));
    Owned d(PyDict_New());
    put(d.p, key_loss, loss); put(d.p, key_logp_tok, logp); put(d.p, key_row_status, status);
    Owned go(a[9] == Py_None ? THPVariable_Wrap(g) : Py_NewRef(a[9]));
    return PyTuple_Pack(2, d.p, go.p);
  });
}

// select(seq_start, corrected, tv, mode, seed, row_offset, mask, rollout_status, stream)
PyObject* py_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 9);
    const at::Tensor &seq = tensor(a[0]), &corrected = tensor(a[1]);
    const at::Device dev = corrected.device();
    const int64_t N = corrected.size(0), B = seq.size(0) - 1;
    if (seq.scalar_type() != at::kLong || seq.device() != dev || !seq.is_contiguous())
      raise_value("seq_start must be a contiguous int64 tensor on the same device");
    saki_select_in si = {};
    si.N = N; si.B = B; si.seq_start = (const int64_t*)seq.data_ptr();
    si.corrected = (const uint8_t*)vector(a[1], at::kByte, N, dev, "corrected");
    if (a[2] != Py_None) si.tv = (const float*)vector(a[2], at::kFloat, N, dev, "tv");
    si.mode = (int32_t)integer(a[3]); si.seed = word(a[4]); si.row_offset = word(a[5]);
    if (a[6] != Py_None) si.mask = (const uint8_t*)vector(a[6], at::kByte, N, dev, "mask");
    if (a[7] != Py_None) si.rollout_status = (const uint32_t*)vector(a[7], at::kInt, N, dev, "rollout_status");
    const at::Tensor selected = empty({N}, at::kByte, dev), m = empty({std::max<int64_t>(B, 0)}, at::kInt, dev);
    void* const st = stream_of(a[8]);
    uint8_t* const sp = (uint8_t*)selected.data_ptr();
    int32_t* const mp = (int32_t*)m.data_ptr();
    check_rc(unlocked([&] { return lib.select_tm(&si, sp, mp, st); }));
    Owned x(THPVariable_Wrap(selected)), y(THPVariable_Wrap(m));
    return PyTuple_Pack(2, x.p, y.p);
  });
}

// spec(s, t, draft, eps, temperature, seed, seq_offset, stream)
PyObject* py_spec(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 8);
    const at::Tensor &s = tensor(a[0]), &t = tensor(a[1]), &draft = tensor(a[2]);
    if (s.dim() != 3 || !t.sizes().equals(s.sizes()) || t.scalar_type() != s.scalar_type() || s.stride(2) != 1 || t.stride(2) != 1)
      raise_saki(1, "logits must be [B,K+1,V] with unit stride along V");
    const int64_t B = s.size(0), K1 = s.size(1);
    const at::Device dev = s.device();
    saki_spec_out so = {};
    Owned per(alloc_outputs(B * K1, dev, &so.per_pos));
    const at::Tensor n_accept = empty({B}, at::kInt, dev), next_token = empty({B}, at::kInt, dev), is_corr = empty({B}, at::kByte, dev);
    saki_spec_in si = {};
    si.student_logits = s.data_ptr(); si.teacher_logits = t.data_ptr();
    si.ss_seq = s.stride(0); si.ss_pos = s.stride(1); si.ts_seq = t.stride(0); si.ts_pos = t.stride(1);
    si.B = B; si.K = (int32_t)(K1 - 1); si.V = (int32_t)s.size(2); si.dtype = dtype_code(s);
    si.draft = (const int32_t*)draft.data_ptr(); si.draft_ld = B > 1 ? draft.stride(0) : draft.size(1);
    si.eps = (float)number(a[3]); si.temperature = (float)number(a[4]); si.seed = word(a[5]); si.seq_offset = word(a[6]);
    so.n_accept = (int32_t*)n_accept.data_ptr(); so.next_token = (int32_t*)next_token.data_ptr(); so.next_is_correction = (uint8_t*)is_corr.data_ptr();
    void* const st = stream_of(a[7]);
    check_rc(unlocked([&] { return lib.spec_verify(&si, &so, st); }));
    Owned d(PyDict_New());
    put(d.p, key_n_accept, n_accept); put(d.p, key_next_token, next_token); put(d.p, key_next_is_correction, is_corr);
    if (PyDict_SetItem(d.p, key_per_pos, per.p) < 0) throw Raised();
    return d.release();
  });
}

// propose(s, temperature, seed, row_offset, stream)
PyObject* py_propose(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 5);
    const at::Tensor& s = tensor(a[0]);
    const at::Tensor out = empty({s.size(0)}, at::kInt, s.device());
    const float tau = (float)number(a[1]);
    const uint64_t seed = word(a[2]), off = word(a[3]);
    void* const st = stream_of(a[4]);
    const int code = dtype_code(s);
    int32_t* const op = (int32_t*)out.data_ptr();
    check_rc(unlocked([&] { return lib.sample_proposal(s.data_ptr(), row_stride(s), s.size(0), (int32_t)s.size(1), code, tau, seed, off, op, st); }));
    return THPVariable_Wrap(out);
  });
}

// vshard_local(slices, V, proposal, eps, temperature, seed, row_offset, mask, grad_scale, backward, stream, eager_waves,
// max_waves): the stages of all ranks' slices on one device -> (out, gradient slices, waves, state)
PyObject* py_vshard_local(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 13);
    Owned seq(PySequence_Fast(a[0], "slices must be a sequence of (student, teacher, first column)"));
    const int world = (int)PySequence_Fast_GET_SIZE(seq.p);
    if (world < 1) raise_value("no slices");
    const bool backward = PyObject_IsTrue(a[9]) == 1;
    std::vector<saki_vshard_in> in((size_t)world);
    std::vector<void*> part((size_t)world), grad;
    std::vector<int64_t> ld_g;
    Owned gs(PyList_New(world));
    at::Device dev = at::kCPU;
    int64_t N = 0;
    for (int r = 0; r < world; ++r) {
      Owned item(PySequence_Fast(PySequence_Fast_GET_ITEM(seq.p, r), "a slice is (student, teacher, first column)"));
      if (PySequence_Fast_GET_SIZE(item.p) != 3) raise_value("a slice is (student, teacher, first column)");
      const at::Tensor &s = tensor(PySequence_Fast_GET_ITEM(item.p, 0)), &t = tensor(PySequence_Fast_GET_ITEM(item.p, 1));
      if (r == 0) { dev = s.device(); N = s.size(0); }
      saki_vshard_in& si = in[(size_t)r];
      si = saki_vshard_in{};
      si.student_logits = s.data_ptr(); si.teacher_logits = t.data_ptr();
      si.ld_s = s.size(0) > 1 ? s.stride(0) : std::max<int64_t>(1, s.size(1));
      si.ld_t = t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(1, t.size(1));
      si.N = s.size(0); si.V_local = (int32_t)s.size(1); si.dtype = dtype_code(s);
      si.V = (int32_t)integer(a[1]); si.v0 = (int32_t)integer(PySequence_Fast_GET_ITEM(item.p, 2));
      si.proposal = (const int32_t*)tensor(a[2]).data_ptr();
      si.eps = (float)number(a[3]); si.temperature = (float)number(a[4]); si.seed = word(a[5]); si.row_offset = word(a[6]);
      si.mask = (const uint8_t*)ptr_or_null(a[7]);
      si.rank = r; si.world = world;
      if (backward) {
        const at::Tensor g = at::empty_like(s);
        grad.push_back(g.data_ptr());
        ld_g.push_back(g.size(0) > 1 ? g.stride(0) : std::max<int64_t>(1, g.size(1)));
        PyList_SET_ITEM(gs.p, r, THPVariable_Wrap(g));
      } else PyList_SET_ITEM(gs.p, r, Py_NewRef(Py_None));
    }
    // the slices' device is the current one from here on: without a stream from the caller, the stages, the zeroing and the reading
    // of the counters take one and the same stream of it
    c10::cuda::OptionalCUDAGuard on_device;
    if (dev.is_cuda()) on_device.set_device(dev);
    const float scale = (float)number(a[8]);
    void* const st = stream_of(a[10]);
    const int eager = (int)integer(a[11]), max_waves = (int)integer(a[12]);
    saki_out so;
    Owned out(alloc_outputs(N, dev, &so));
    // the caller's stream is torch's current one from here on: the counters are zeroed and read in the order of the stages,
    // and what is freed at the end of the call goes back to the allocator on the stream that used it
    c10::cuda::OptionalCUDAStreamGuard on_stream;
    if (a[10] != Py_None && dev.is_cuda()) on_stream.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)st, dev.index()));
    const at::Tensor state = empty({N, SAKI_VSHARD_STATE}, at::kDouble, dev), gathered = empty({world, N, SAKI_VSHARD_PARTIALS}, at::kDouble, dev);
    const at::Tensor counts = at::zeros({eager + 1, 2}, at::TensorOptions().dtype(at::kInt).device(dev));
    double* const sp = (double*)state.data_ptr();
    double* const gp = (double*)gathered.data_ptr();
    uint32_t* const np = (uint32_t*)counts.data_ptr();
    for (int r = 0; r < world; ++r) part[(size_t)r] = gp + (int64_t)r * N * SAKI_VSHARD_PARTIALS;   // where the all-gather would put it
    auto stage = [&](int k, uint32_t* count, int flags) {
      check_rc(unlocked([&] {
        return lib.vshard_stage(in.data(), world, k, sp, (double* const*)part.data(), gp, k == 2 && backward ? (void* const*)grad.data() : nullptr,
                                ld_g.data(), scale, k == 3 ? &so : nullptr, count, flags, st);
      }));
    };
    // the rows still solving after stage 0 and after each wave, and those marked for float64 (page-locked: the device is idle
    // until the host has looked at them)
    const at::Tensor h = at::empty({eager + 1, 2}, at::TensorOptions().dtype(at::kInt).pinned_memory(dev.is_cuda()));
    at::cuda::CUDAEvent copied;
    auto read = [&] {
      return unlocked([&] {
        h.copy_(counts, true);
        if (dev.is_cuda()) { copied.record(c10::cuda::getCurrentCUDAStream(dev.index())); copied.synchronize(); }
        return (const int32_t*)h.data_ptr();
      });
    };
    int waves = 0;
    if (N > 0) {
      constexpr int NONE = SAKI_VSHARD_NONE_MARKED;
      stage(0, np, NONE);                                    // a wave's combine is the first that can mark a row
      for (int k = 0; k < eager; ++k) stage(1, np + 2 * (1 + k), k == 0 ? NONE : 0);
      const int32_t* c = read();
      while (waves < eager && c[2 * waves] > 0) ++waves;
      int32_t sum = c[2 * eager], left = sum, marked = 0;
      for (int k = 0; k < eager; ++k) marked += c[2 * k + 1];
      while (left > 0 && waves < max_waves) {
        stage(1, np + 2 * eager, 0);                         // (adds to the last pair)
        ++waves;
        c = read();
        left = c[2 * eager] - sum;
        sum = c[2 * eager];
      }
      marked += c[2 * eager + 1];
      stage(2, nullptr, marked ? 0 : NONE);
      stage(3, nullptr, marked ? 0 : NONE);
    }
    Owned w(PyLong_FromLong(waves)), sv(THPVariable_Wrap(state));
    return PyTuple_Pack(4, out.p, gs.p, w.p, sv.p);
  });
}

// ---- the pages of a key-value cache ----

// The tensors' device and the caller's stream are the current ones while it lives: outputs and scratch come from the pool of the
// stream that uses them.
struct OnStream {
  c10::cuda::OptionalCUDAGuard device;
  c10::cuda::OptionalCUDAStreamGuard stream;
  void* handle;
  OnStream(at::Device dev, PyObject* given) {
    if (!dev.is_cuda()) raise_value("tensors must be on a GPU");
    device.set_device(dev);
    if (given != Py_None) stream.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)word(given), dev.index()));
    handle = (void*)c10::cuda::getCurrentCUDAStream(dev.index()).stream();
  }
};
const char* type_name(at::ScalarType t) { return t == at::kInt ? "int32" : t == at::kByte ? "uint8" : t == at::kFloat ? "float32" : "other"; }
// a contiguous tensor of n elements, any shape
const at::Tensor& packed(PyObject* o, at::ScalarType type, int64_t n, at::Device dev, const char* name) {
  const at::Tensor& v = tensor(o);
  if (v.scalar_type() != type || v.numel() != n || v.device() != dev || !v.is_contiguous())
    raise_value(std::string(name) + " must be a contiguous " + type_name(type) + " tensor of " + std::to_string(n) + " elements on the same device");
  return v;
}
int64_t step_of(const at::Tensor& t, int64_t d) { return t.size(d) > 1 ? t.stride(d) : 0; }      // (of a dimension of one: never used)

struct Cache {
  saki_cache c = {};
  at::Device dev = at::kCPU;
  at::Tensor scratch;
};
constexpr int CACHE_ARGS = 5;      // meta, B, max_pages, n_pages, page_size
Cache cache_of(PyObject* const* a) {
  Cache k;
  const at::Tensor& m = tensor(a[0]);
  saki_cache& c = k.c;
  c.B = integer(a[1]);
  const int64_t max_pages = integer(a[2]), n_pages = integer(a[3]), page = integer(a[4]);
  if (c.B < 0 || max_pages < 1 || n_pages < 1 || page < 1 || max_pages > INT32_MAX || n_pages > INT32_MAX || page > INT32_MAX || c.B > INT32_MAX)
    raise_value("a cache has B >= 0 sequences, and at least one page per sequence, page and position");
  c.max_pages = (int32_t)max_pages; c.n_pages = (int32_t)n_pages; c.page_size = (int32_t)page; c.ld_table = max_pages;
  if (m.scalar_type() != at::kInt || !m.is_contiguous() || m.numel() != c.B * max_pages + c.B + n_pages)
    raise_value("a cache's tables must be a contiguous int32 tensor of B * max_pages + B + n_pages elements");
  k.dev = m.device();
  c.page_table = (int32_t*)m.data_ptr();
  c.length = c.page_table + c.B * max_pages;
  c.ref_count = c.length + c.B;
  return k;
}
void with_scratch(Cache& k) {      // (of the current stream, like the outputs)
  k.c.scratch_bytes = lib.cache_scratch_bytes(k.c.B, k.c.max_pages, k.c.n_pages);
  k.scratch = empty({k.c.scratch_bytes}, at::kByte, k.dev);
  k.c.scratch = k.scratch.data_ptr();
}

// cache_reserve(cache..., n_new, stream) -> (copy_src, copy_dst, row_status)
PyObject* py_cache_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, CACHE_ARGS + 2);
    Cache k = cache_of(a);
    const OnStream on(k.dev, a[6]);
    with_scratch(k);
    const int32_t* each = nullptr;
    int64_t all = 0;
    if (THPVariable_Check(a[5])) each = (const int32_t*)packed(a[5], at::kInt, k.c.B, k.dev, "n_new").data_ptr();
    else if ((all = integer(a[5])) > INT32_MAX || all < INT32_MIN) raise_value("n_new out of range");
    const at::Tensor src = empty({k.c.B}, at::kInt, k.dev), dst = empty({k.c.B}, at::kInt, k.dev), st = empty({k.c.B}, at::kInt, k.dev);
    check_rc(unlocked([&] { return lib.cache_reserve(&k.c, each, (int32_t)all, (int32_t*)src.data_ptr(), (int32_t*)dst.data_ptr(), (uint32_t*)st.data_ptr(), on.handle); }));
    Owned x(THPVariable_Wrap(src)), y(THPVariable_Wrap(dst)), z(THPVariable_Wrap(st));
    return PyTuple_Pack(3, x.p, y.p, z.p);
  });
}

// cache_truncate(cache..., keep, keep_add, of, row_status, stream) -> row_status
PyObject* py_cache_truncate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, CACHE_ARGS + 5);
    Cache k = cache_of(a);
    const OnStream on(k.dev, a[9]);
    if (a[8] != Py_None) k.c.row_status = (const uint32_t*)packed(a[8], at::kInt, k.c.B, k.dev, "row_status").data_ptr();
    const int32_t* const keep = (const int32_t*)packed(a[5], at::kInt, k.c.B, k.dev, "keep").data_ptr();
    const int64_t add = integer(a[6]), of = integer(a[7]);
    if (add > INT32_MAX || add < INT32_MIN || of > INT32_MAX || of < INT32_MIN) raise_value("keep_add or of out of range");
    const at::Tensor st = empty({k.c.B}, at::kInt, k.dev);
    check_rc(unlocked([&] { return lib.cache_truncate(&k.c, keep, (int32_t)add, (int32_t)of, (uint32_t*)st.data_ptr(), on.handle); }));
    return THPVariable_Wrap(st);
  });
}

// cache_fork(cache..., parent, group, stream) -> row_status
PyObject* py_cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, CACHE_ARGS + 3);
    Cache k = cache_of(a);
    const OnStream on(k.dev, a[7]);
    with_scratch(k);
    const int32_t* const parent = (const int32_t*)packed(a[5], at::kInt, k.c.B, k.dev, "parent").data_ptr();
    const int64_t group = integer(a[6]);
    const at::Tensor st = empty({k.c.B}, at::kInt, k.dev);
    check_rc(unlocked([&] { return lib.cache_fork(&k.c, parent, group, (uint32_t*)st.data_ptr(), on.handle); }));
    return THPVariable_Wrap(st);
  });
}

// cache_compact(cache..., stream) -> (copy_src, copy_dst, n_moves, row_status)
PyObject* py_cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, CACHE_ARGS + 1);
    Cache k = cache_of(a);
    const OnStream on(k.dev, a[5]);
    with_scratch(k);
    const int64_t half = k.c.n_pages / 2;
    const at::Tensor src = empty({half}, at::kInt, k.dev), dst = empty({half}, at::kInt, k.dev), moves = empty({}, at::kInt, k.dev), st = empty({k.c.B}, at::kInt, k.dev);
    check_rc(unlocked([&] { return lib.cache_compact(&k.c, (int32_t*)src.data_ptr(), (int32_t*)dst.data_ptr(), (int32_t*)moves.data_ptr(), (uint32_t*)st.data_ptr(), on.handle); }));
    Owned x(THPVariable_Wrap(src)), y(THPVariable_Wrap(dst)), z(THPVariable_Wrap(moves)), w(THPVariable_Wrap(st));
    return PyTuple_Pack(4, x.p, y.p, z.p, w.p);
  });
}

// The runs of memory that a page of the pool is made of: where each starts within the page, in elements, and the elements of one.  (In most layouts there is one; heads or
// positions outermost, or rows with something between them, make several.)
int64_t page_runs(const at::Tensor& t, std::vector<int64_t>& starts) {
  std::vector<std::pair<int64_t, int64_t>> dims;
  for (int64_t d = 1; d < t.dim(); ++d)
    if (t.size(d) != 1) dims.emplace_back(t.stride(d), t.size(d));
  std::sort(dims.begin(), dims.end());
  int64_t run = 1;
  size_t k = 0;
  for (; k < dims.size() && dims[k].first == run; ++k) run *= dims[k].second;
  starts.assign(1, 0);
  int64_t upto = run;              // elements that the page spans so far
  for (; k < dims.size(); ++k) {
    const int64_t stride = dims[k].first, n = dims[k].second, have = (int64_t)starts.size();
    if (stride < upto) raise_value("the elements of a pool's page must not overlap");
    for (int64_t i = 1; i < n; ++i)
      for (int64_t r = 0; r < have; ++r) starts.push_back(starts[(size_t)r] + i * stride);
    upto += (n - 1) * stride;
  }
  return run;
}
// copy_pages(pools, copy_src, copy_dst, stream)
PyObject* py_copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 4);
    Owned seq(PySequence_Fast(a[0], "pools must be a sequence of tensors"));
    const int m = (int)PySequence_Fast_GET_SIZE(seq.p);
    if (m == 0) Py_RETURN_NONE;
    const at::Tensor &src = tensor(a[1]);
    const at::Device dev = src.device();
    const OnStream on(dev, a[3]);
    packed(a[1], at::kInt, src.numel(), dev, "copy_src");
    const at::Tensor& dst = packed(a[2], at::kInt, src.numel(), dev, "copy_dst");
    std::vector<void*> pool;         // a run of the pages of a pool each
    std::vector<int64_t> step, bytes, starts;
    int64_t pages = 0;
    for (int i = 0; i < m; ++i) {
      const at::Tensor& t = tensor(PySequence_Fast_GET_ITEM(seq.p, i));
      if (t.device() != dev || t.dim() < 2 || t.numel() == 0) raise_value("a pool must be a tensor [n_pages, ...] on the lists' device");
      if (i == 0) pages = t.size(0);
      if (t.size(0) != pages || pages > INT32_MAX) raise_value("the pools of a call have the same number of pages");
      const int64_t size = (int64_t)t.element_size(), run = page_runs(t, starts) * size;
      for (int64_t at : starts) {
        pool.push_back((char*)t.data_ptr() + at * size);
        bytes.push_back(run);
        step.push_back(pages > 1 ? t.stride(0) * size : run);
      }
    }
    if (pool.size() > (size_t)INT32_MAX) raise_value("too many pools");
    check_rc(unlocked([&] {
      return lib.cache_copy_pages(pool.data(), step.data(), bytes.data(), (int32_t)pool.size(), (const int32_t*)src.data_ptr(), (const int32_t*)dst.data_ptr(), src.numel(), (int32_t)pages, on.handle);
    }));
    Py_RETURN_NONE;
  });
}

int kv_dtype(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return SAKI_F32;
  if (t.scalar_type() == at::kBFloat16) return SAKI_BF16;
  raise_value(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
}
void check_pool(const at::Tensor& t, const at::Tensor& like, at::Device dev, int64_t n_pages, int64_t page, int64_t H, int64_t D, const char* name) {
  if (t.dim() != 4 || t.device() != dev || t.scalar_type() != like.scalar_type() || t.size(1) != page || t.size(2) != H || t.size(3) != D ||
      (n_pages >= 0 && t.size(0) != n_pages) || (D > 1 && t.stride(3) != 1))
    raise_value(std::string(name) + " must be a tensor [n_pages, page_size, H, D] of the other tensors' type and device, with unit stride along D");
}
// cache_write(cache..., k, v, k_pages, v_pages, row_status, n_new, stream)
PyObject* py_cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, CACHE_ARGS + 7);
    Cache c = cache_of(a);
    const OnStream on(c.dev, a[11]);
    const at::Tensor &k = tensor(a[5]), &v = tensor(a[6]), &kp = tensor(a[7]), &vp = tensor(a[8]);
    if (k.dim() != 4 || !v.sizes().equals(k.sizes()) || v.scalar_type() != k.scalar_type() || k.size(0) != c.c.B || k.device() != c.dev || v.device() != c.dev ||
        (k.size(3) > 1 && (k.stride(3) != 1 || v.stride(3) != 1)))
      raise_value("k and v must be [B, Q, H, D] of one type on the cache's device, with unit stride along D");
    const int64_t H = k.size(2), D = k.size(3);
    check_pool(kp, k, c.dev, c.c.n_pages, c.c.page_size, H, D, "k_pages");
    check_pool(vp, k, c.dev, c.c.n_pages, c.c.page_size, H, D, "v_pages");
    if (k.size(1) > INT32_MAX || H > INT32_MAX || D > INT32_MAX) raise_value("sizes out of range");
    saki_cache_kv w = {};
    w.k = k.data_ptr(); w.k_seq = step_of(k, 0); w.k_pos = step_of(k, 1); w.k_head = step_of(k, 2);
    w.v = v.data_ptr(); w.v_seq = step_of(v, 0); w.v_pos = step_of(v, 1); w.v_head = step_of(v, 2);
    w.k_pages = kp.data_ptr(); w.kp_page = step_of(kp, 0); w.kp_pos = step_of(kp, 1); w.kp_head = step_of(kp, 2);
    w.v_pages = vp.data_ptr(); w.vp_page = step_of(vp, 0); w.vp_pos = step_of(vp, 1); w.vp_head = step_of(vp, 2);
    w.Q = (int32_t)k.size(1); w.H = (int32_t)H; w.D = (int32_t)D; w.dtype = kv_dtype(k);
    if (a[9] != Py_None) w.row_status = (const uint32_t*)packed(a[9], at::kInt, c.c.B, c.dev, "row_status").data_ptr();
    if (a[10] != Py_None) w.n_new = (const int32_t*)packed(a[10], at::kInt, c.c.B, c.dev, "n_new").data_ptr();
    check_rc(unlocked([&] { return lib.cache_write(&c.c, &w, on.handle); }));
    Py_RETURN_NONE;
  });
}

// attention(q, k_pages, v_pages, page_table, length, scale, window, sinks, n_query, out, row_status, stream) -> (out, lse, row_status)
PyObject* py_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 12);
    const at::Tensor &q = tensor(a[0]), &kp = tensor(a[1]), &vp = tensor(a[2]), &table = tensor(a[3]);
    if (q.dim() != 4 || kp.dim() != 4 || (q.size(3) > 1 && q.stride(3) != 1)) raise_value("q must be [B, Q, Hq, D] with unit stride along D, the pools [n_pages, page_size, H, D]");
    const at::Device dev = q.device();
    const int64_t B = q.size(0), Q = q.size(1), Hq = q.size(2), D = q.size(3), pages = kp.size(0), page = kp.size(1), H = kp.size(2);
    check_pool(kp, q, dev, -1, page, H, D, "k_pages");
    check_pool(vp, q, dev, pages, page, H, D, "v_pages");
    if (table.dim() != 2 || table.size(0) != B || table.scalar_type() != at::kInt || table.device() != dev || (table.size(1) > 1 && table.stride(1) != 1))
      raise_value("page_table must be an int32 tensor [B, max_pages] on the same device, with unit stride along the pages");
    for (int64_t s : {Q, Hq, D, pages, page, H, table.size(1)})
      if (s > INT32_MAX) raise_value("sizes out of range");
    saki_attn_in in = {};
    in.dtype = kv_dtype(q);
    const OnStream on(dev, a[11]);
    in.q = q.data_ptr(); in.q_seq = step_of(q, 0); in.q_pos = step_of(q, 1); in.q_head = step_of(q, 2);
    in.k_pages = kp.data_ptr(); in.kp_page = step_of(kp, 0); in.kp_pos = step_of(kp, 1); in.kp_head = step_of(kp, 2);
    in.v_pages = vp.data_ptr(); in.vp_page = step_of(vp, 0); in.vp_pos = step_of(vp, 1); in.vp_head = step_of(vp, 2);
    in.page_table = (const int32_t*)table.data_ptr(); in.ld_table = B > 1 ? table.stride(0) : table.size(1);
    in.length = (const int32_t*)packed(a[4], at::kInt, B, dev, "length").data_ptr();
    if (a[8] != Py_None) in.n_query = (const int32_t*)packed(a[8], at::kInt, B, dev, "n_query").data_ptr();
    if (a[10] != Py_None) in.row_status = (const uint32_t*)packed(a[10], at::kInt, B, dev, "row_status").data_ptr();
    in.B = B; in.Q = (int32_t)Q; in.Hq = (int32_t)Hq; in.H = (int32_t)H; in.D = (int32_t)D;
    in.page_size = (int32_t)page; in.max_pages = (int32_t)table.size(1); in.n_pages = (int32_t)pages;
    const int64_t window = integer(a[6]), sinks = integer(a[7]);
    if (window < 0 || sinks < 0) raise_value("window and sinks must be >= 0");
    in.window = (int32_t)std::min<int64_t>(window, INT32_MAX); in.sinks = (int32_t)std::min<int64_t>(sinks, INT32_MAX);
    in.scale = a[5] == Py_None ? (float)(1.0 / std::sqrt((double)std::max<int64_t>(D, 1))) : (float)number(a[5]);
    const at::Tensor out = a[9] == Py_None ? empty({B, Q, Hq, D}, q.scalar_type(), dev) : tensor(a[9]);
    if (!out.sizes().equals(q.sizes()) || out.scalar_type() != q.scalar_type() || out.device() != dev || (D > 1 && out.stride(3) != 1))
      raise_value("out must be like q, with unit stride along D");
    const at::Tensor lse = empty({B, Q, Hq}, at::kFloat, dev), st = empty({B}, at::kInt, dev);
    saki_attn_out o = {out.data_ptr(), step_of(out, 0), step_of(out, 1), step_of(out, 2), (float*)lse.data_ptr(), (uint32_t*)st.data_ptr()};
    const int64_t bytes = lib.paged_attention_scratch_bytes(&in);
    if (bytes == 0) raise_saki(SAKI_ERR_INVALID_ARG, lib.last_error());
    const at::Tensor scratch = empty({bytes}, at::kByte, dev);
    check_rc(unlocked([&] { return lib.paged_attention(&in, &o, scratch.data_ptr(), bytes, on.handle); }));
    Owned x(THPVariable_Wrap(out)), y(THPVariable_Wrap(lse)), z(THPVariable_Wrap(st));
    return PyTuple_Pack(3, x.p, y.p, z.p);
  });
}

// beams(logits, score, n, temperature, finished, pad, stream) -> (parent, token, score, row_status)
PyObject* py_beams(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    n_args(n, 7);
    const at::Tensor& z = tensor(a[0]);
    if (z.dim() != 3 || (z.size(2) > 1 && z.stride(2) != 1)) raise_value("logits must be [B, W, V] with unit stride along V");
    const at::Device dev = z.device();
    const int64_t B = z.size(0), W = z.size(1), V = z.size(2), m = integer(a[2]), pad = integer(a[5]);
    if (W > INT32_MAX || V > INT32_MAX || m < 1 || m > 64 || pad < 0 || pad >= V) raise_value("n must be in [1,64] and pad in [0,V)");
    saki_beam_in in = {};
    in.dtype = dtype_code(z);
    const OnStream on(dev, a[6]);
    in.logits = z.data_ptr(); in.ld_seq = step_of(z, 0); in.ld_beam = W > 1 ? z.stride(1) : V;
    in.score = (const float*)packed(a[1], at::kFloat, B * W, dev, "score").data_ptr();
    if (a[4] != Py_None) in.finished = (const uint8_t*)packed(a[4], at::kByte, B * W, dev, "finished").data_ptr();
    in.B = B; in.W = (int32_t)W; in.V = (int32_t)V; in.n = (int32_t)m; in.pad = (int32_t)pad; in.temperature = (float)number(a[3]);
    const at::Tensor parent = empty({B, m}, at::kInt, dev), token = empty({B, m}, at::kInt, dev), score = empty({B, m}, at::kFloat, dev), st = empty({B, W}, at::kInt, dev);
    const int64_t bytes = lib.beam_scratch_bytes(B, in.W, in.V, in.n);
    const at::Tensor scratch = empty({bytes}, at::kByte, dev);
    saki_beam_out out = {(int32_t*)parent.data_ptr(), (int32_t*)token.data_ptr(), (float*)score.data_ptr(), (uint32_t*)st.data_ptr()};
    check_rc(unlocked([&] { return lib.beam_select(&in, &out, scratch.data_ptr(), bytes, on.handle); }));
    Owned x(THPVariable_Wrap(parent)), y(THPVariable_Wrap(token)), w(THPVariable_Wrap(score)), v(THPVariable_Wrap(st));
    return PyTuple_Pack(4, x.p, y.p, w.p, v.p);
  });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, nullptr},
    {"alloc_outputs", (PyCFunction)(void (*)(void))py_alloc_outputs, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void (*)(void))py_route, METH_FASTCALL, nullptr},
    {"meta", (PyCFunction)(void (*)(void))py_meta, METH_FASTCALL, nullptr},
    {"select", (PyCFunction)(void (*)(void))py_select, METH_FASTCALL, nullptr},
    {"spec", (PyCFunction)(void (*)(void))py_spec, METH_FASTCALL, nullptr},
    {"propose", (PyCFunction)(void (*)(void))py_propose, METH_FASTCALL, nullptr},
    {"cache_reserve", (PyCFunction)(void (*)(void))py_cache_reserve, METH_FASTCALL, nullptr},
    {"cache_truncate", (PyCFunction)(void (*)(void))py_cache_truncate, METH_FASTCALL, nullptr},
    {"cache_fork", (PyCFunction)(void (*)(void))py_cache_fork, METH_FASTCALL, nullptr},
    {"cache_compact", (PyCFunction)(void (*)(void))py_cache_compact, METH_FASTCALL, nullptr},
    {"copy_pages", (PyCFunction)(void (*)(void))py_copy_pages, METH_FASTCALL, nullptr},
    {"cache_write", (PyCFunction)(void (*)(void))py_cache_write, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)(void))py_attention, METH_FASTCALL, nullptr},
    {"beams", (PyCFunction)(void (*)(void))py_beams, METH_FASTCALL, nullptr},
    {"vshard_local", (PyCFunction)(void (*)(void))py_vshard_local, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_saki_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// the torch and the interpreter that this file was compiled against, to be found in the binary
extern "C" __attribute__((used, visibility("default"))) const char saki_built_for[] = SAKI_BUILT_FOR;

PyMODINIT_FUNC PyInit__saki_torch(void) {
  for (int k = 0; k < N_FIELDS; ++k) field_key[k] = PyUnicode_InternFromString(FIELD[k]);
  key_loss = PyUnicode_InternFromString("loss"); key_logp_tok = PyUnicode_InternFromString("logp_tok");
  key_row_status = PyUnicode_InternFromString("row_status"); key_n_accept = PyUnicode_InternFromString("n_accept");
  key_next_token = PyUnicode_InternFromString("next_token"); key_next_is_correction = PyUnicode_InternFromString("next_is_correction");
  key_per_pos = PyUnicode_InternFromString("per_pos");
  return PyModule_Create(&module);
}
