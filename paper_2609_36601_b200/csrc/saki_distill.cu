// Distillation of a student's rows from a teacher's top logits: loss and gradient (see include/saki.h for the definition).  With pi = softmax(z / tau), K the
// listed tokens, w_j their teacher's probabilities, W their sum, R the rest of the teacher's mass (0: the list is all there is), S the student's mass outside K:
//   forward   L = sum_K w (log w - log pi) + R (log R - log S)      dL/dz_v = (W + R) pi_v - w_v in K, (W + R - R / S) pi_v outside
//   reverse   L = sum_K pi (log pi - log w) + S (log S - log R)     dL/dz_v = pi_v (log pi_v - log w_v - L) in K, pi_v (log S - log R - L) outside
// so outside K the gradient is one number a row times pi.  S is summed over the elements outside K: 1 - sum_K pi would cancel where the student
// agrees with its teacher, which is what it is trained to.
//
// Three kernels:
//   distill_lists_kernel    a warp a row: looks through the lists (ranges, a token twice), w and log w from float64 exponentials (R = 1 - W cancels)
//   distill_stream_kernel   persistent CTAs, a row each: a row is read from HBM once and its gradient written once.  Every lane owns 16-byte slots of shared
//                           memory that it fills with cp.async; the leading steps of a warp's segment stay there for both passes, the rest goes through a
//                           ring (its second touch comes from L2); while a row's gradient is written the slots take the next row.  A warp knows from a word of bits
//                           at which of its steps there are listed tokens, and looks for them only there.
//   distill_general_kernel  float64, any layout, a block a row: for what the other cannot serve, and the rows that it cannot resolve (row list).  Its exponentials cost 13 ms for 1000 float32 rows of
//                           262144, the first length that it serves alone, where the other takes 0.51 for 262000
// What bounds it: 4096 bf16 rows of 151936 with lists of 64, 540 us where the bytes take 380 (70 %; lists of 1: 495, of 128: 580; without the gradient 285, bytes 190): instructions (63 % of the issue slots are filled, 62 % of the
// special-function pipe) and the two block barriers of a row, at which warps wait a fifth of their time.  float32 rows of 151936 run at 81 % of the copy rate.
#include "saki_device.cuh"
#include <algorithm>
#include <cfloat>
#include <mutex>
#include <type_traits>

namespace saki {

namespace {

constexpr int KMAX = 128;
constexpr double LEAST_REST = 0x1p-20;
constexpr double LEAST_LOG_S = -1000 * LN2;      // a student's mass outside K below 2^-1000 is none: all there is masked, by -inf or by the type's lowest value

// what a row's list comes to
struct alignas(16) ListRow {
  double W, R, H, log_R;      // W: sum of w as rounded to float32, R of the exact ones, H: sum of w log w; R 0: there is no rest
  int n;                      // tokens that are there
  uint32_t status;            // MASKED, BAD_ID, NONFINITE: the row contributes nothing
};

struct DistillParams {
  saki_distill_in in;
  saki_distill_out out;
  void* dlogits;
  int64_t ld_g;
  float grad_scale;
  ListRow* rows;              // [N]
  int* id;                    // [N][k] the tokens that are there, -1 elsewhere
  float2* w;                  // [N][k] (w, log w)
  unsigned long long* flagged;
  int32_t* redo_list;         // [N] rows that the streaming kernel hands to the float64 kernel
  unsigned int* redo_count;
  int32_t from_list;
};

__device__ __forceinline__ void write_result(const DistillParams& P, int64_t row, float loss, float lse, uint32_t status) {
  if (P.out.loss) P.out.loss[row] = loss;
  if (P.out.lse) P.out.lse[row] = lse;
  if (P.out.row_status) P.out.row_status[row] = status;
  if (status & (SAKI_ROW_NONFINITE | SAKI_ROW_BAD_ID)) atomicAdd(P.flagged, 1ull);
}
__device__ __forceinline__ float warp_least(float x) {      // of numbers, over the warp
  float r;
  asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float warp_most(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ double warp_max(double a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a = fmax(a, __shfl_xor_sync(0xffffffffu, a, o));
  return a;
}

// ---------------------------------------------------------------- lists
__global__ void __launch_bounds__(256) distill_lists_kernel(const DistillParams P) {
  __shared__ alignas(16) int ids[8][KMAX];
  launch_dependents();
  wait_for_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = P.in.k;
  const int64_t row = (int64_t)blockIdx.x * 8 + warp;
  if (blockIdx.x == 0 && threadIdx.x == 0) *P.redo_count = 0;
  if (row >= P.in.N) return;
  const double rtau = 1.0 / (double)P.in.temperature;
  uint32_t status = 0;
  int id[KMAX / 32];
  double t[KMAX / 32];                 // logits, not divided by the temperature: differences first, which float64 holds however large they are
  bool bad_id = false, bad = false;
  if (P.in.mask && P.in.mask[row] == 0) status = SAKI_ROW_MASKED;
  int n = 0;
#pragma unroll
  for (int r = 0; r < KMAX / 32; ++r) {
    const int j = r * 32 + lane;
    id[r] = -1; t[r] = -CUDART_INF;
    if (j < k && !status) {
      const int v = P.in.token[row * P.in.ld_k + j];
      const float x = P.in.logit[row * P.in.ld_k + j];
      bad_id |= v < -1 || v >= P.in.V;
      if (v >= 0 && v < P.in.V && x != -CUDART_INF_F) {
        id[r] = v; t[r] = (double)x;
        bad |= !(fabsf(x) < CUDART_INF_F);
      }
    }
    ids[warp][j] = id[r];
    n += __popc(__ballot_sync(0xffffffffu, id[r] >= 0));
  }
  __syncwarp();
  int same[KMAX / 32] = {};            // entries with the same token, itself among them
  for (int i = 0; i < k; i += 4) {
    const int4 v = *(const int4*)&ids[warp][i];
#pragma unroll
    for (int r = 0; r < KMAX / 32; ++r)
      if (r * 32 < k) same[r] += (v.x == id[r]) + (v.y == id[r]) + (v.z == id[r]) + (v.w == id[r]);
  }
#pragma unroll
  for (int r = 0; r < KMAX / 32; ++r) bad_id |= id[r] >= 0 && same[r] > 1;
  const bool with_rest = P.in.teacher_lse != nullptr;
  double top = 0, ref = 0;             // log w = (t - top) rtau - ref
  if (with_rest) {
    const float l = P.in.teacher_lse[row];
    ref = (double)l;
    bad |= !(fabsf(l) < CUDART_INF_F);
  } else {
    double m = -CUDART_INF, s = 0;
#pragma unroll
    for (int r = 0; r < KMAX / 32; ++r) m = fmax(m, t[r]);
    m = warp_max(m);
#pragma unroll
    for (int r = 0; r < KMAX / 32; ++r)
      if (r * 32 < k && id[r] >= 0) s += exp((t[r] - m) * rtau);
    s = warp_sum(s);
    if (n) { top = m; ref = log(s); }
  }
  if (!status && __any_sync(0xffffffffu, bad_id)) status = SAKI_ROW_BAD_ID;
  if (!status && __any_sync(0xffffffffu, bad)) status = SAKI_ROW_NONFINITE;
  double W = 0, W32 = 0, H = 0;      // (the loss takes sums of w z from sums of w times the log-sum-exp: the same w in both, or a large common z would not cancel)
#pragma unroll
  for (int r = 0; r < KMAX / 32; ++r) {
    const int j = r * 32 + lane;
    float2 w = make_float2(0.f, 0.f);
    if (r * 32 < k && id[r] >= 0) {
      const double lw = (t[r] - top) * rtau - ref, e = exp(lw);
      w = make_float2((float)e, (float)fmax(lw, -(double)FLT_MAX));      // (finite: a student's probability of 0 times it is 0)
      W += e; W32 += (double)w.x; H += e > 0 ? e * lw : 0;
    }
    if (j < k) {
      P.id[row * k + j] = status ? -1 : id[r];
      P.w[row * k + j] = w;
    }
  }
  W = warp_sum(W); W32 = warp_sum(W32); H = warp_sum(H);
  if (lane == 0) {
    const bool rest = with_rest && n < P.in.V;
    const double R = rest ? fmax(1.0 - W, LEAST_REST) : 0;
    P.rows[row] = ListRow{W32, R, H, rest ? log(R) : 0, n, status};
  }
}

// ---------------------------------------------------------------- general kernel (float64)
constexpr int DG_THREADS = 256;
struct GeneralShared {
  double sum[DG_THREADS / 32];
  int id[KMAX];
  double lw[KMAX];
  float w[KMAX];
  uint32_t bits[128];          // a bit for the low 12 bits of a listed token
};
__device__ __forceinline__ double block_fold(double v, double* sh, bool max) {
  v = max ? warp_max(v) : warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double a = sh[0];
  for (int w = 1; w < DG_THREADS / 32; ++w) a = max ? fmax(a, sh[w]) : a + sh[w];
  return a;
}

template <typename T>
__global__ void __launch_bounds__(DG_THREADS) distill_general_kernel(const DistillParams P) {
  __shared__ GeneralShared sh;
  wait_for_predecessor();
  const int64_t n_items = P.from_list ? (int64_t)*P.redo_count : P.in.N;      // (an empty row list, as a rule)
  const int V = P.in.V, k = P.in.k;
  const double rtau = 1.0 / (double)P.in.temperature;
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int64_t row = P.from_list ? (int64_t)P.redo_list[item] : item;
    const T* s = (const T*)P.in.student_logits + row * P.in.ld_s;
    T* g = P.dlogits ? (T*)P.dlogits + row * P.ld_g : nullptr;
    const ListRow list = P.rows[row];
    uint32_t status = list.status;
    __syncthreads();
    for (int i = threadIdx.x; i < 128; i += DG_THREADS) sh.bits[i] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < k; j += DG_THREADS) {
      const int v = P.id[row * k + j];
      const float2 w = P.w[row * k + j];
      sh.id[j] = v; sh.w[j] = w.x; sh.lw[j] = w.y;
      if (v >= 0) atomicOr(&sh.bits[(v & 4095) >> 5], 1u << (v & 31));
    }
    __syncthreads();
    auto place = [&](int v) {          // of v in the list, -1: not listed
      if (!(sh.bits[(v & 4095) >> 5] >> (v & 31) & 1u)) return -1;
      for (int j = 0; j < k; ++j)
        if (sh.id[j] == v) return j;
      return -1;
    };
    // (largest logits and differences to them before the temperature: log-probabilities of rows of 1e30 or the lowest value, masked throughout, are no differences of their own rounding)
    double in_max = -CUDART_INF, out_max = -CUDART_INF, bad = 0;
    if (!status) {
      for (int v = threadIdx.x; v < V; v += DG_THREADS) {
        const double x = (double)ld_as_float(s, v);
        const bool listed = place(v) >= 0;
        if (!(x < CUDART_INF) || (listed && !(x > -CUDART_INF))) bad = 1;
        if (listed) in_max = fmax(in_max, x);
        else out_max = fmax(out_max, x);
      }
      bad = block_fold(bad, sh.sum, true);
      in_max = block_fold(in_max, sh.sum, true);
      out_max = block_fold(out_max, sh.sum, true);
      if (bad != 0 || !(fmax(in_max, out_max) > -CUDART_INF)) status = SAKI_ROW_NONFINITE;
    }
    if (status) {
      if (g) for (int v = threadIdx.x; v < V; v += DG_THREADS) st_from_float(g, v, 0.f);
      if (threadIdx.x == 0) write_result(P, row, 0.f, 0.f, status);
      continue;
    }
    double in_sum = 0, out_sum = 0;
    for (int v = threadIdx.x; v < V; v += DG_THREADS) {
      const double x = (double)ld_as_float(s, v);
      if (place(v) >= 0) in_sum += exp((x - in_max) * rtau);
      else if (x > -CUDART_INF) out_sum += exp((x - out_max) * rtau);
    }
    in_sum = block_fold(in_sum, sh.sum, false);
    out_sum = block_fold(out_sum, sh.sum, false);
    const double top = fmax(in_max, out_max);
    const double log_sum = log((in_sum > 0 ? in_sum * exp((in_max - top) * rtau) : 0) + (out_sum > 0 ? out_sum * exp((out_max - top) * rtau) : 0)), lse = top * rtau + log_sum;
    auto log_pi = [&](int v) { return ((double)ld_as_float(s, v) - top) * rtau - log_sum; };
    double lS = out_sum > 0 ? (out_max - top) * rtau + log(out_sum) - log_sum : -CUDART_INF;
    const bool rest = list.R > 0 && lS > LEAST_LOG_S;
    if (!rest) lS = 0;
    const double S = rest ? exp(lS) : 0;
    double loss = 0;
    for (int j = threadIdx.x; j < k; j += DG_THREADS) {
      const int v = sh.id[j];
      if (v < 0) continue;
      const double lp = log_pi(v);
      loss += P.in.reverse ? exp(lp) * (lp - sh.lw[j]) : (double)sh.w[j] * (sh.lw[j] - lp);
    }
    loss = block_fold(loss, sh.sum, false);
    if (rest) loss += P.in.reverse ? S * (lS - list.log_R) : list.R * (list.log_R - lS);
    if (threadIdx.x == 0) write_result(P, row, (float)loss, (float)lse, 0u);
    if (!g) continue;
    const double kg = (double)P.grad_scale * rtau, Z = list.W + (rest ? list.R : 0);
    const double outside = P.in.reverse ? (rest ? lS - list.log_R : 0) - loss : Z - (rest ? exp(list.log_R - lS) : 0);
    for (int v = threadIdx.x; v < V; v += DG_THREADS) {
      const double lp = log_pi(v), p = exp(lp);
      const int j = place(v);
      double x = outside * p;
      if (j >= 0) x = P.in.reverse ? p * (lp - sh.lw[j] - loss) : Z * p - (double)sh.w[j];
      st_from_float(g, v, (float)(kg * x));
    }
  }
}

// ---------------------------------------------------------------- streaming kernel
constexpr int KEEP = 12, RING = 4, RESIDENT = KEEP - RING;      // 512-byte steps of a warp in shared memory; of them, where a segment does not fit, the ring's (both even: steps go in pairs)
constexpr int MAX_STEPS = 64;
constexpr float MARGIN = 60.f;                                  // in base 2: how far a lane's elements may lie above its shift

template <typename T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
  static constexpr int E = 8, LOG = 3, STEP_LOG = 8;
  static constexpr uint32_t FILLER = 0xFF80FF80u;               // two of -inf: nothing at any temperature
  static __device__ __forceinline__ float2 pair(const uint4& w, int i) { return unpack_bf16x2(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
  static __device__ __forceinline__ float top(const uint4& w) {
    const float2 a = unpack_bf16x2(max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w)));
    return fmaxf(a.x, a.y);
  }
  // whether an element lies above the limit (a pair of the same bf16, rounded down)
  using Limit = uint32_t;
  static __device__ __forceinline__ Limit limit(float x) { const uint32_t h = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rd(x)); return h << 16 | h; }
  static __device__ __forceinline__ uint32_t pairs(const uint4& w) { return max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w)); }
  static __device__ __forceinline__ bool above(const uint4& w, const uint4& u, Limit l) { return max_bf16x2(max_bf16x2(pairs(w), pairs(u)), l) != l; }
  static __device__ __forceinline__ float get(const uint4& w, int e) {
    const int i = e >> 1;
    const uint32_t r = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    return __uint_as_float(e & 1 ? r & 0xffff0000u : r << 16);
  }
  static __device__ __forceinline__ void put(uint4& w, int e, float x) {
    const int i = e >> 1;
    uint32_t r = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    const uint32_t h = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x));
    r = e & 1 ? (r & 0x0000ffffu) | (h << 16) : (r & 0xffff0000u) | h;
    if (i == 0) w.x = r; else if (i == 1) w.y = r; else if (i == 2) w.z = r; else w.w = r;
  }
};
template <> struct Elem<float> {
  static constexpr int E = 4, LOG = 2, STEP_LOG = 7;
  static constexpr uint32_t FILLER = 0xFF800000u;
  static __device__ __forceinline__ float2 pair(const uint4& w, int i) { return i == 0 ? make_float2(__uint_as_float(w.x), __uint_as_float(w.y)) : make_float2(__uint_as_float(w.z), __uint_as_float(w.w)); }
  static __device__ __forceinline__ float top(const uint4& w) { return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w))); }
  using Limit = float;
  static __device__ __forceinline__ Limit limit(float x) { return x; }
  static __device__ __forceinline__ bool above(const uint4& w, const uint4& u, Limit l) { return fmaxf(top(w), top(u)) > l; }
  static __device__ __forceinline__ float get(const uint4& w, int e) { return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w); }
  static __device__ __forceinline__ void put(uint4& w, int e, float x) {
    const uint32_t r = __float_as_uint(x);
    if (e == 0) w.x = r; else if (e == 1) w.y = r; else if (e == 2) w.z = r; else w.w = r;
  }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint64_t pol) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "l"(pol) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(__cvta_generic_to_global(src)) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(__cvta_generic_to_global(src)) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t at, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void st_stream(void* p, const uint4& v, uint64_t pol) {
  asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(__cvta_generic_to_global(p)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "l"(pol) : "memory");
}
__device__ __forceinline__ uint64_t policy(bool keep) {
  uint64_t p;
  if (keep) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// A row in 16-byte pieces that start on 16-byte boundaries of memory: its first and last piece may hold elements of no row of the call.
template <typename T> struct View {
  const char* base;            // of piece 0; NULL: there is no row
  int head;                    // elements of piece 0 before the row
  int full0, full;             // pieces full0 .. full0 + full - 1 lie within the row
  int n;                       // pieces
};
template <typename T> __device__ __forceinline__ View<T> view_of(const T* row, int V) {
  constexpr int E = Elem<T>::E;
  View<T> v;
  const uintptr_t a = (uintptr_t)row;
  v.base = (const char*)(a & ~(uintptr_t)15);
  v.head = (int)((a & 15) / sizeof(T));
  v.full0 = v.head ? 1 : 0;
  v.full = max((V + v.head) / E - v.full0, 0);      // (a row that ends within its first piece has none)
  v.n = (V + v.head + E - 1) / E;
  return v;
}
// a piece with elements of other rows, or none: the filler there
template <typename T> __device__ __forceinline__ uint4 odd_piece(const char* base, int head, int V, int c) {
  constexpr int E = Elem<T>::E;
  uint4 w = make_uint4(Elem<T>::FILLER, Elem<T>::FILLER, Elem<T>::FILLER, Elem<T>::FILLER);
  const T* p = (const T*)base + (int64_t)c * E;
#pragma unroll
  for (int e = 0; e < E; ++e)      // (all on their way at once)
    if (c * E + e >= head && c * E + e < head + V) Elem<T>::put(w, e, ld_as_float(p, e));
  return w;
}
template <typename T> __device__ __forceinline__ void fill_piece(uint32_t slot, const View<T>& v, int V, int c, uint64_t pol) {
  if ((unsigned)(c - v.full0) < (unsigned)v.full) copy16(slot, v.base + (uint32_t)c * 16u, pol);      // (a row has less than 2^31 bytes)
  else if (v.base) sts128(slot, odd_piece<T>(v.base, v.head, V, c));
}

struct Segment { int c0, steps, res; };      // of a warp: its first piece, steps of 32 pieces, how many of them stay in shared memory

// A lane's pieces of a row, by step; at steps lo to hi - 1 those of all lanes lie within the row.  INNER: at all steps of the warp.
template <typename T, bool INNER> struct Source {
  View<T> v;
  const char* at;              // the lane's first piece
  int V, c0, lo, hi;
  __device__ __forceinline__ Source(const View<T>& view, int V_, int first, int lane) : v(view), at(view.base + (int64_t)(first + lane) * 16), V(V_), c0(first + lane) {
    lo = max((view.full0 - first + 31) >> 5, 0);
    hi = max((view.full0 + view.full - first) >> 5, lo);
  }
  __device__ __forceinline__ bool whole(int step) const { return INNER || (unsigned)(step - lo) < (unsigned)(hi - lo); }
  __device__ __forceinline__ void fill(uint32_t slot, int step, uint64_t pol) const {
    if (whole(step)) copy16(slot, at + (uint32_t)step * 512u, pol);      // (a row has less than 2^31 bytes)
    else fill_piece<T>(slot, v, V, c0 + 32 * step, pol);
  }
};

// Visits the warp's steps in order, two at a time: body(words, words of the next step, step), single(words, step) for one that is left over.  Every visit
// commits one group of copies; all but the last group are there before words are read.  A streamed step, once read, requests the streamed step RING
// further on: of this pass, or past its end the first streamed steps of the pass that follows, over `wrap` (the same row again, or the next one).
// With REFILL a resident step, once read, requests the same step of `wrap`.
template <bool REFILL, typename S, typename Body, typename Single>
__device__ __forceinline__ void visit(const Segment& sg, uint32_t base, const S& cur, const S& wrap, uint64_t pol_cur, uint64_t pol_wrap, uint64_t pol_res, uint32_t& ring_slot,
                                      Body&& body, Single&& single) {
  uint32_t slot = base, ring = ring_slot;
  auto next_slot = [&] {
    const uint32_t at = ring;
    ring += 512;
    if (ring == base + KEEP * 512) ring = base + RESIDENT * 512;
    return at;
  };
  auto refill = [&](uint32_t at, int step) {
    if (step + RING < sg.steps) cur.fill(at, step + RING, pol_cur);
    else wrap.fill(at, step + RING - (sg.steps - sg.res), pol_wrap);
  };
  int k = 0;
#pragma unroll 1
    for (; k + 1 < sg.res; k += 2, slot += 1024) {
      copies_wait<1>();
      const uint4 a = lds128(slot), b = lds128(slot + 512);
      if constexpr (REFILL) { wrap.fill(slot, k, pol_res); wrap.fill(slot + 512, k + 1, pol_res); }
      copies_commit();
      body(a, b, k);
    }
#pragma unroll 1
    for (; k >= sg.res && k + 1 < sg.steps; k += 2) {
      copies_wait<1>();
      const uint32_t s0 = next_slot(), s1 = next_slot();
      const uint4 a = lds128(s0), b = lds128(s1);
      refill(s0, k);
      refill(s1, k + 1);
      copies_commit();
      body(a, b, k);
    }
    if (k < sg.steps) {
      const bool stays = k < sg.res;
      copies_wait<1>();
      const uint32_t at = stays ? slot : next_slot();
      const uint4 a = lds128(at);
      if (!stays) refill(at, k);
      else if constexpr (REFILL) wrap.fill(at, k, pol_res);
      copies_commit();
      single(a, k);
    }
  ring_slot = ring;
}

using One = std::integral_constant<int, 1>;
using Two = std::integral_constant<int, 2>;

template <int MW> struct StreamShared {
  double red[4][MW];           // by warp: the sum outside K, its shift, the sum in K, the sum for the loss
  // by row parity: a warp may be a pass behind the others (what it reads is written again only behind the next barrier but one)
  float bc[2][4];
  double dc[2][4];
  ListRow list[3];             // of three rows in turn: written while a warp may still read the one before last
  int id[3][KMAX];
  float2 w[3][KMAX];
  float x[2][KMAX], g[KMAX];   // listed elements, by row parity (a warp may write the next row's while another still reads this one's), and their gradients: of the warp that has them
  uint32_t mine[MW][KMAX];     // by warp: what lies in its segment, place in elements << 8 | place in the list
};
template <int MW> constexpr int stream_smem = MW * KEEP * 512 + (int)sizeof(StreamShared<MW>);
template <int MW> constexpr int BLOCKS = std::min(32 / MW, 227 * 1024 / (stream_smem<MW> + 1024));      // on an SM

// The listed elements in steps `step` to `step` + STEPS - 1 of a warp (STEPS 1 or 2, step a multiple of it): body(place within the steps, place in the list).
template <int STEPS, int STEP_LOG, typename Body> __device__ __forceinline__ void each_listed(const uint32_t* mine, int n, int step, int lane, Body&& body) {
#pragma unroll 1
  for (int q = 0; q < n; q += 32) {
    const uint32_t entry = q + lane < n ? mine[q + lane] : ~0u;
    unsigned m = __ballot_sync(0xffffffffu, entry >> (7 + STEP_LOG + STEPS) == (uint32_t)step >> (STEPS - 1));
#pragma unroll 1
    while (m) {
      const int src = __ffs(m) - 1;
      m &= m - 1;
      const uint32_t e = __shfl_sync(0xffffffffu, entry, src);
      body((int)(e >> 8) & ((STEPS << STEP_LOG) - 1), (int)(e & 255u));
    }
  }
}

// 1 / x and 2^e for sums of a row, 2^-126 to 2^126: the first to some 1e-14
__device__ __forceinline__ double pow2_near(int e) { return __longlong_as_double((long long)(1023 + e) << 52); }
__device__ __forceinline__ double rcp_near(double x) {
  const int e = (int)(__double_as_longlong(x) >> 52) - 1023;
  return rcp_fast(x * pow2_near(-e)) * pow2_near(-e);
}

template <typename T, int MW, bool BWD>
__global__ void __launch_bounds__(MW * 32, BLOCKS<MW>) distill_stream_kernel(const DistillParams P) {
  using El = Elem<T>;
  constexpr int E = El::E;
  extern __shared__ __align__(128) unsigned char dsm[];
  StreamShared<MW>& sh = *(StreamShared<MW>*)(dsm + MW * KEEP * 512);
  launch_dependents();
  wait_for_predecessor();
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int V = P.in.V, k = P.in.k;
  const int64_t N = P.in.N;
  // whole steps of 32 pieces, dealt out in order: for a row that starts anywhere
  const int steps_all = ((V + 2 * E - 2) / E + 31) / 32, steps_q = steps_all / MW, steps_r = steps_all - steps_q * MW;
  Segment sg;
  sg.steps = steps_q + (warp < steps_r ? 1 : 0);
  sg.c0 = 32 * (warp * steps_q + min(warp, steps_r));
  sg.res = sg.steps <= KEEP ? sg.steps : RESIDENT;
  const uint32_t base = smem_addr(dsm) + (uint32_t)warp * (KEEP * 512) + (uint32_t)lane * 16;
  uint32_t ring_slot = base + RESIDENT * 512;
  const double rtau = 1.0 / (double)P.in.temperature;
  const float c32 = (float)(INV_LN2 * rtau), rc32 = 1.f / c32;
  const double x0_tau = rtau / (double)c32;      // of a shift, in units of the log-sum-exp
  const uint64_t pol_last = policy(true), pol_first = policy(false);
  const bool few_groups = sg.steps <= 4;      // a short segment: its copies are fewer groups back than the waits assume
  const bool reverse = P.in.reverse != 0;
  View<T> none = {};

  auto view = [&](int64_t row) { return row < N ? view_of<T>((const T*)P.in.student_logits + row * P.in.ld_s, V) : none; };
  auto stage_list = [&](int64_t row, int b) {       // a row's list and what it comes to, on their way into shared memory
    if (row >= N) return;
    for (int j = tid; j < k; j += MW * 32) {
      copy4(smem_addr(&sh.id[b][j]), P.id + row * k + j);
      copy8(smem_addr(&sh.w[b][j]), P.w + row * k + j);
    }
    if (tid < (int)sizeof(ListRow) / 8) copy8(smem_addr((char*)&sh.list[b] + tid * 8), (const char*)(P.rows + row) + tid * 8);
  };

  View<T> cur = view(blockIdx.x);
  stage_list(blockIdx.x, 0);
  for (int s = 0; s < sg.res; ++s) { fill_piece<T>(base + s * 512, cur, V, sg.c0 + lane + 32 * s, pol_first); copies_commit(); }
  if (sg.res < sg.steps)
    for (int j = 0; j < RING; ++j) { fill_piece<T>(ring_slot + j * 512, cur, V, sg.c0 + lane + 32 * (sg.res + j), pol_last); copies_commit(); }
  copies_commit();
  copies_wait<0>();
  __syncthreads();

  int b = 0, parity = 0;
  for (int64_t row = blockIdx.x; row < N; row += gridDim.x, parity ^= 1) {
    const int64_t next_row = row + gridDim.x;
    const View<T> nxt = view(next_row);
    const int next_b = b == 2 ? 0 : b + 1;
    if (few_groups) copies_wait<0>();
    stage_list(next_row, next_b);      // (goes with the first step's group, and is there before the row's second barrier)
    const bool live = sh.list[b].status == 0;
    // what of the list lies in this warp's segment, and at which steps
    uint32_t* const mine = sh.mine[warp];
    int n_mine = 0;
    uint32_t here_lo = 0, here_hi = 0;
#pragma unroll 1
    for (int q = 0; q < k; q += 32) {
      const int id = q + lane < k ? sh.id[b][q + lane] : -1;
      const int place = id + cur.head - sg.c0 * E;
      const bool in = id >= 0 && place >= 0 && place < sg.steps * 32 * E;
      const unsigned m = __ballot_sync(0xffffffffu, in);
      if (m == 0) continue;
      if (in) mine[n_mine + __popc(m & ((1u << lane) - 1))] = (uint32_t)place << 8 | (uint32_t)(q + lane);
      n_mine += __popc(m);
      const int step = place >> El::STEP_LOG;
      here_lo |= __reduce_or_sync(0xffffffffu, in && step < 32 ? 1u << step : 0u);
      here_hi |= __reduce_or_sync(0xffffffffu, in && step >= 32 ? 1u << (step - 32) : 0u);
    }
    __syncwarp();
    const uint64_t here = (uint64_t)here_hi << 32 | here_lo;
    // The segment lies within whole pieces of this row and the next: long rows have loops of their own for that (4096 rows of 151936 567 -> 544 us; for short ones it is code that
    // has to be fetched: 16 rows of 32000 11 -> 16 us).
    auto holds = [&](const View<T>& v) { return sg.c0 >= v.full0 && sg.c0 + 32 * sg.steps <= v.full0 + v.full; };
    const bool inner = MW == 32 && nxt.base && holds(cur) && holds(nxt);

    // ------------------------------------------------ pass 1: the sum outside K of 2^(c x + shift).  A lane's shift comes from the warp's first elements, and moves where
    // elements lie MARGIN above it (with the first ones masked, say)
    float shift = 0.f;
    typename El::Limit limit;
    {
      copies_wait<1>();
      float m0 = sg.steps > 0 ? El::top(lds128(base)) : -CUDART_INF_F;
      m0 = fminf(fmaxf(warp_most(m0), -1e8f), 1e30f);      // (masks, of the lowest value or -inf, stay below it; a NaN is passed over: it comes out of the sum)
      shift = -ceilf(c32 * m0);
      limit = El::limit((MARGIN - shift) * rc32);
    }
    float2 S0 = splat(0.f), S1 = splat(0.f);
    uint64_t bits = here;             // of the steps that are left
    {
      const float2 cc = splat(c32);
      const bool ahead = sg.steps == sg.res && nxt.base != nullptr;      // a resident row leaves L2 free: the next one is sent on its way there
      float2 kk = splat(shift);
      auto ahead_of = [&](int step) {
        if (BWD && ahead && (lane & 7) == 0 && sg.c0 + lane + 32 * step < nxt.n) asm volatile("prefetch.global.L2 [%0];" ::"l"(nxt.base + (int64_t)(sg.c0 + lane + 32 * step) * 16));
      };
      auto leave_out = [&](auto steps, uint4& w0, uint4& w1, int step) {      // listed elements
        each_listed<steps.value, El::STEP_LOG>(mine, n_mine, step, lane, [&](int e, int j) {
          if (lane == (e >> El::LOG & 31)) {
            const bool second = e >> El::STEP_LOG;
            sh.x[parity][j] = El::get(second ? w1 : w0, e & (E - 1));
            if (second) El::put(w1, e & (E - 1), -CUDART_INF_F);
            else El::put(w0, e & (E - 1), -CUDART_INF_F);
          }
        });
      };
      auto move = [&](float top) {                    // a new shift; sums so far go along
        const float to = -ceilf(c32 * fminf(top, 1e30f)), f = ex2f(fmaxf(to - kk.x, -200.f));
        S0 = fmul2(S0, splat(f)); S1 = fmul2(S1, splat(f));
        kk = splat(to);
        limit = El::limit((MARGIN - to) * rc32);
      };
      auto add = [&](const uint4& w) {
#pragma unroll
        for (int i = 0; i < E / 2; i += 2) {
          S0 = fadd2(S0, ex2f2(ffma2(El::pair(w, i), cc, kk)));
          S1 = fadd2(S1, ex2f2(ffma2(El::pair(w, i + 1), cc, kk)));
        }
      };
      auto two = [&](uint4 w0, uint4 w1, int step) {
        ahead_of(step); ahead_of(step + 1);
        if (bits & 3ull) leave_out(Two{}, w0, w1, step);
        bits >>= 2;
        if (El::above(w0, w1, limit)) move(fmaxf(El::top(w0), El::top(w1)));
        add(w0); add(w1);
      };
      auto one = [&](uint4 w, int step) {
        ahead_of(step);
        if (bits & 1ull) leave_out(One{}, w, w, step);
        bits >>= 1;
        if (El::above(w, w, limit)) move(El::top(w));
        add(w);
      };
      auto pass = [&](auto in) {
        const Source<T, in.value> c(cur, V, sg.c0, lane), n(nxt, V, sg.c0, lane);
        visit<!BWD>(sg, base, c, BWD ? c : n, pol_last, pol_first, pol_first, ring_slot, two, one);
      };
      if (inner) pass(std::bool_constant<MW == 32>{});
      else pass(std::false_type{});
      shift = kk.x;
    }
    __syncwarp();
    float warp_shift = shift;
#pragma unroll 1
    for (int i = lane; i < n_mine; i += 32)      // (a segment may have nothing but listed elements and masked ones)
      warp_shift = fminf(warp_shift, -ceilf(c32 * fminf(sh.x[parity][mine[i] & 255u], 1e30f)));
    __syncwarp();
    warp_shift = warp_least(warp_shift);
    double outside = (((double)S0.x + (double)S0.y) + ((double)S1.x + (double)S1.y)) * (double)ex2f(fmaxf(warp_shift - shift, -200.f));
    double inside = 0, cross = 0;
#pragma unroll 1
    for (int i = lane; i < n_mine; i += 32) {
      const int j = (int)(mine[i] & 255u);
      const float x = sh.x[parity][j];
      const float2 w = sh.w[b][j];
      const float e = ex2f(fmaf(x, c32, warp_shift));
      // (a listed token that the student's row has masked, or not finite: the float64 kernel decides)
      inside += fabsf(x) < CUDART_INF_F ? (double)e : CUDART_NAN;
      cross += reverse ? (double)e * ((double)x * rtau - (double)w.y) : (double)w.x * ((double)x * rtau);
    }
    __syncwarp();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {      // (three chains side by side)
      outside += __shfl_xor_sync(0xffffffffu, outside, o);
      inside += __shfl_xor_sync(0xffffffffu, inside, o);
      cross += __shfl_xor_sync(0xffffffffu, cross, o);
    }
    if (lane == 0) { sh.red[0][warp] = outside; sh.red[1][warp] = (double)warp_shift; sh.red[2][warp] = inside; sh.red[3][warp] = cross; }
    __syncthreads();
    if (warp == 0) {
      const int wl = lane < MW ? lane : 0;
      const bool part = lane < MW;
      const double ks = sh.red[1][wl];
      const double kr = (double)warp_least(part ? (float)ks : CUDART_INF_F);
      const double f = part ? pow2_exact((int)fmax(kr - ks, -1000.0)) : 0;
      // (a warp whose share is nothing beside the others' may have an infinite one; a NaN counts everywhere)
      auto share = [&](double x) { return f > 0 ? x * f : part && x != x ? CUDART_NAN : 0.0; };
      double out = share(sh.red[0][wl]), in = share(sh.red[2][wl]);
      double sum_cross = part ? sh.red[3][wl] * (reverse ? f : 1.0) : 0;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        out += __shfl_xor_sync(0xffffffffu, out, o);
        in += __shfl_xor_sync(0xffffffffu, in, o);
        sum_cross += __shfl_xor_sync(0xffffffffu, sum_cross, o);
      }
      if (lane == 0) {
        float scale_out = 0.f, Zs = 0.f, kg = 0.f, lse_f = 0.f, loss_f = 0.f, grad_shift = 0.f;
        const ListRow& list = sh.list[b];
        if (live) {
          const double sum = out + in;
          const bool has_rest = list.R > 0 && out > 0;
          // not finite (or nothing but masked entries), or a share outside K so small that the sum may have lost terms of it,
          // or logits of millions, whose shifts are no exact float32: the float64 kernel decides
          if (!(sum > 0) || !(sum < CUDART_INF) || !(fabs(sum_cross) < CUDART_INF) || (list.R > 0 && out < sum * 0x1p-60) || !(fabs(kr) < 8e6)) {
            P.redo_list[atomicAdd(P.redo_count, 1u)] = (int32_t)row;
          } else {
            // sum of exp(x / tau) = exp(x0 / tau) sum of 2^(c (x - x0)) with x0 = -kr / c, up to what c as a float32 is off over distances from x0
            const double l2 = log2_fast(sum), lo2 = has_rest ? log2_fast(out) : l2, lse = LN2 * l2 - kr * x0_tau;
            const double rsum = rcp_near(sum);
            const double lS = LN2 * (lo2 - l2);
            const double Z = list.W + (has_rest ? list.R : 0);
            double loss, c_out;
            if (reverse) {
              loss = sum_cross * rsum - lse * (in * rsum) + (has_rest ? out * rsum * (lS - list.log_R) : 0);
              c_out = (has_rest ? lS - list.log_R : 0) - loss;
            } else {
              loss = list.H - sum_cross + lse * list.W + (has_rest ? list.R * (list.log_R - lS) : 0);
              c_out = Z - (has_rest ? list.R * sum * rcp_near(out) : 0);
            }
            const int e = (int)floor(l2);
            const double kgd = (double)P.grad_scale * rtau;
            const double unit = rsum * pow2_near(e);      // 1 over sum 2^-e, which is 1 to 2
            grad_shift = (float)(kr - (double)e);
            scale_out = (float)(kgd * c_out * unit);
            Zs = (float)unit;
            kg = (float)kgd;
            lse_f = (float)lse; loss_f = (float)loss;
            sh.dc[parity][0] = lse; sh.dc[parity][1] = loss; sh.dc[parity][2] = Z;
            if (BWD && !(fabsf(scale_out) < CUDART_INF_F && fabsf(kg) < CUDART_INF_F)) {      // factors beyond float32, of gradients that need not be
              P.redo_list[atomicAdd(P.redo_count, 1u)] = (int32_t)row;
              scale_out = Zs = 0.f;
            } else write_result(P, row, loss_f, lse_f, 0u);
          }
        } else write_result(P, row, 0.f, 0.f, list.status);
        float* const bc = sh.bc[parity];
        bc[0] = grad_shift; bc[1] = scale_out; bc[2] = Zs; bc[3] = kg;
      }
    }
    if (few_groups) {
      copies_commit();      // (a warp without a step has made no visit, which would have committed its copies of the next row's list)
      copies_wait<0>();
    }
    __syncthreads();

    // ------------------------------------------------ pass 2: the gradient
    if constexpr (BWD) {
      const float* const bc = sh.bc[parity];
      const float kr = bc[0], scale = bc[1], unit = bc[2], kg = bc[3];
      const bool zero = unit == 0.f;      // a row that contributes nothing (or waits for the float64 kernel): zeros, whatever its logits
      {
        const double lse = sh.dc[parity][0], loss = sh.dc[parity][1], Z = sh.dc[parity][2];
#pragma unroll 1
        for (int i = lane; i < n_mine; i += 32) {
          const int j = (int)(mine[i] & 255u);
          const float x = sh.x[parity][j];
          const float2 w = sh.w[b][j];
          const float p = ex2f(fmaf(x, c32, kr)) * unit;
          // (p 0: of a token masked by the lowest value, say, whose log-ratio is beyond float32)
          const float v = !reverse ? (float)(Z * (double)p - (double)w.x) : p > 0.f ? p * (float)((double)x * rtau - lse - (double)w.y - loss) : 0.f;
          sh.g[j] = zero ? 0.f : kg * v;
        }
      }
      __syncwarp();
      bits = here;
      const float2 cc = splat(c32), kk = splat(kr), sc = splat(scale);
      T* const g_row = (T*)P.dlogits + row * P.ld_g;
      char* const g_base = (char*)((uintptr_t)g_row & ~(uintptr_t)15);
      const bool alike = ((uintptr_t)g_row & 15) == cur.head * sizeof(T);      // the gradient's pieces lie like the row's
      auto plain = [&](const uint4& w) -> uint4 {
        float2 v[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) v[i] = fmul2(ex2f2(ffma2(El::pair(w, i), cc, kk)), sc);
        if constexpr (E == 8) return make_uint4(pack_bf16x2(v[0].x, v[0].y), pack_bf16x2(v[1].x, v[1].y), pack_bf16x2(v[2].x, v[2].y), pack_bf16x2(v[3].x, v[3].y));
        else return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
      };
      auto put_listed = [&](auto steps, uint4& g0, uint4& g1, int step) {
        each_listed<steps.value, El::STEP_LOG>(mine, n_mine, step, lane, [&](int e, int j) {
          if (lane == (e >> El::LOG & 31)) {
            const float x = sh.g[j];
            if (e >> El::STEP_LOG) El::put(g1, e & (E - 1), x);
            else El::put(g0, e & (E - 1), x);
          }
        });
      };
      auto pass = [&](auto in) {
        const Source<T, in.value> c(cur, V, sg.c0, lane), n(nxt, V, sg.c0, lane);
        char* const to = g_base + (int64_t)c.c0 * 16;
        auto store = [&](const uint4& g, int step) {
          const int p = c.c0 + 32 * step;
          if (in.value || (alike && (c.whole(step) || (unsigned)(p - cur.full0) < (unsigned)cur.full))) st_stream(to + (uint32_t)step * 512u, g, pol_first);
          else if (p < cur.n)
#pragma unroll 1
            for (int e = 0; e < E; ++e)
              if ((unsigned)(p * E + e - cur.head) < (unsigned)V) st_from_float(g_row, p * E + e - cur.head, El::get(g, e));
        };
        visit<true>(sg, base, c, n, pol_first, pol_last, pol_first, ring_slot,
          [&](const uint4& w0, const uint4& w1, int step) {
            uint4 g0 = make_uint4(0u, 0u, 0u, 0u), g1 = g0;
            if (!zero) {
              g0 = plain(w0); g1 = plain(w1);
              if (bits & 3ull) put_listed(Two{}, g0, g1, step);
            }
            bits >>= 2;
            store(g0, step); store(g1, step + 1);
          },
          [&](const uint4& w, int step) {
            uint4 g = make_uint4(0u, 0u, 0u, 0u);
            if (!zero) {
              g = plain(w);
              if (bits & 1ull) put_listed(One{}, g, g, step);
            }
            bits >>= 1;
            store(g, step);
          });
      };
      if (inner && alike) pass(std::bool_constant<MW == 32>{});
      else pass(std::false_type{});
    }
    cur = nxt;
    b = next_b;
  }
  copies_wait<0>();
}

template <typename T, int MW, bool BWD> cudaError_t launch_stream_as(const DistillParams& p, cudaStream_t st) {
  static std::mutex mu;
  static int known_dev = -1, known = 0;
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  constexpr int smem = stream_smem<MW>;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (known_dev != dev) {
      cudaError_t e = cudaFuncSetAttribute(distill_stream_kernel<T, MW, BWD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e == cudaSuccess) e = cudaDeviceGetAttribute(&known, cudaDevAttrMultiProcessorCount, dev);
      if (e != cudaSuccess) return e;
      known_dev = dev;
    }
    sms = known;
  }
  const int grid = (int)std::min<int64_t>(p.in.N, (int64_t)sms * BLOCKS<MW>);
  return launch_pdl(distill_stream_kernel<T, MW, BWD>, dim3((unsigned)grid), MW * 32, smem, st, true, p);
}
template <typename T, int MW> cudaError_t launch_with(const DistillParams& p, cudaStream_t st) { return p.dlogits ? launch_stream_as<T, MW, true>(p, st) : launch_stream_as<T, MW, false>(p, st); }
// Warps to a row: as few as keep it in shared memory (several blocks on an SM: one's barriers under another's passes), all 32 where none do; 16 where there are no more rows than blocks.
// (2960 bf16 rows with lists of 32, us: 2048 entries 52 with 4 warps, 70 with 16, 122 with 32; 16384 92 with 8, 100, 125; 32003 156 with 16, 174; 65536, which 16 do not
// keep, 230 and 198; float32 rows of 32003, which they do not keep either, 214 and 193.)
template <typename T> cudaError_t launch_stream(const DistillParams& p, cudaStream_t st, int sms) {
  const int64_t bytes = ((int64_t)p.in.V + 2 * Elem<T>::E) * (int64_t)sizeof(T), N = p.in.N;
  if (bytes <= 4 * KEEP * 512 && N > sms * BLOCKS<8>) return launch_with<T, 4>(p, st);
  if (bytes <= 8 * KEEP * 512 && N > sms * BLOCKS<16>) return launch_with<T, 8>(p, st);
  if (bytes <= 16 * KEEP * 512) return launch_with<T, 16>(p, st);
  return launch_with<T, 32>(p, st);
}

int64_t round256(int64_t x) { return (x + 255) & ~(int64_t)255; }

}  // namespace

int64_t distill_scratch_bytes(int64_t N, int32_t k) { return 256 + round256(N * 4) + round256(N * (int64_t)sizeof(ListRow)) + round256(N * k * 4) + round256(N * k * 8); }

// rows of up to 64 steps a warp, in both types
bool distill_stream_can_serve(const saki_distill_in& in) {
  const int e = in.dtype == SAKI_BF16 ? 8 : 4;
  return in.N <= 0x7fffffff && ((int64_t)in.V + 2 * e - 2) / e <= (int64_t)MAX_STEPS * 32 * 32;
}

cudaError_t launch_distill(const saki_distill_in& in, const saki_distill_out& out, void* dlogits, int64_t ld_g, float grad_scale, void* scratch, bool stream,
                           unsigned long long* flagged, int* n_launches, cudaStream_t st) {
  DistillParams p = {};
  p.in = in; p.out = out; p.dlogits = dlogits; p.ld_g = ld_g; p.grad_scale = grad_scale; p.flagged = flagged;
  char* s = (char*)scratch;
  p.redo_count = (unsigned int*)s; s += 256;
  p.redo_list = (int32_t*)s; s += round256(in.N * 4);
  p.rows = (ListRow*)s; s += round256(in.N * (int64_t)sizeof(ListRow));
  p.id = (int*)s; s += round256(in.N * in.k * 4);
  p.w = (float2*)s;
  cudaError_t e = launch_pdl(distill_lists_kernel, dim3((unsigned)((in.N + 7) / 8)), 256, 0, st, true, p);
  ++*n_launches;
  if (e != cudaSuccess) return e;
  if (stream) {
    int dev = 0, sms = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    e = in.dtype == SAKI_BF16 ? launch_stream<__nv_bfloat16>(p, st, sms) : launch_stream<float>(p, st, sms);
    ++*n_launches;
    if (e != cudaSuccess) return e;
    p.from_list = 1;
  }
  const int grid = (int)std::min<int64_t>(in.N, p.from_list ? 148 : 1 << 20);
  ++*n_launches;
  e = in.dtype == SAKI_BF16 ? launch_pdl(distill_general_kernel<__nv_bfloat16>, dim3((unsigned)grid), DG_THREADS, 0, st, true, p)
                            : launch_pdl(distill_general_kernel<float>, dim3((unsigned)grid), DG_THREADS, 0, st, true, p);
  return e;
}

}  // namespace saki
