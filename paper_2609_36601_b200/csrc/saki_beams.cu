// Beam selection over vocabulary rows: the n best continuations of a group of W beams by the sum of the beam's score and the
// log-probability of the token.
//
// What bounds it: issue slots (60 % of them filled; some 860 instructions a warp and 64 elements a thread, 17 us of exponentials) and the barriers between a slice's phases, not HBM:
// 64 groups of 8 beams, 151936 bf16 logits each, a quarter of the beams finished, 50 us where the bytes that are read (not those of finished beams) take 18, the joining kernel 8 of it (52 and 59 with four
// and three blocks an SM instead of five); none finished 58 where they take 24, float32 70 and 84 where they take 36 and 48; 1 group of 4 beams 14 us, two launches and the chains of one slice and of the join.
//
// Within a beam the order of the keys is that of the logits, so a row is read once: a block holds a slice of it in registers, sums
// its exponentials, and picks the slice's n best logits.  For those, a bar: of the maxima of the 64 groups of four threads the n-th
// largest is at most the slice's n-th largest logit, and little below it as a rule.  What reaches the bar (about n elements) goes to a list in
// shared memory, is ranked by counting, and leaves as n sorted pairs.  Slices that would overflow the list (hundreds of equal logits) are picked one
// by one instead.  A second, small kernel joins the slices of a beam (log-sum-exp in float64) and the beams of a group (float64 keys).
#include "saki_device.cuh"
#include <algorithm>
#include <cmath>
#include <limits>

namespace saki {

namespace {

constexpr int BT = 256, BWARPS = BT / 32, GROUPS = 64, LIST = 512;

struct BeamParams {
  saki_beam_in in;
  saki_beam_out out;
  int slices, slice;        // per row, and elements of one
  float c_hi, c_lo;         // log2(e) / temperature
  double inv_tau;
  uint64_t* cand;           // [B * W][slices][n] pairs of a slice, best first; 0: none
  double2* part;            // [B * W][slices] (maximum, sum of 2^(c (x - maximum))) of a slice
  unsigned long long* flagged;
};

// a pair (logit, token) as one word: larger logits first, then lower tokens; never 0 for a logit above -inf
__device__ __forceinline__ uint64_t pair_word(float x, uint32_t v) {
  const uint32_t u = __float_as_uint(x + 0.f);      // (-0 counts as 0)
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return ((uint64_t)o << 32) | (0xffffffffu - v);
}
__device__ __forceinline__ float pair_logit(uint64_t w) {
  const uint32_t o = (uint32_t)(w >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t pair_token(uint64_t w) { return 0xffffffffu - (uint32_t)w; }

template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
  static constexpr int E = 8;
  uint32_t r[4];
  __device__ __forceinline__ float2 pair(int i) const { return unpack_bf16x2(r[i]); }
  __device__ __forceinline__ void set(int i, float x, float y) { r[i] = pack_bf16x2(x, y); }
  __device__ __forceinline__ float top() const {      // (of a pair with a NaN the other)
    auto h = [](uint32_t a) { return *reinterpret_cast<const __nv_bfloat162*>(&a); };
    const float2 a = __bfloat1622float2(__hmax2(__hmax2(h(r[0]), h(r[1])), __hmax2(h(r[2]), h(r[3]))));
    return fmaxf(a.x, a.y);
  }
};
template <> struct Vec<float> {
  static constexpr int E = 4;
  uint32_t r[4];
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])); }
  __device__ __forceinline__ void set(int i, float x, float y) { r[2 * i] = __float_as_uint(x); r[2 * i + 1] = __float_as_uint(y); }
  __device__ __forceinline__ float top() const { return fmaxf(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])), fmaxf(__uint_as_float(r[2]), __uint_as_float(r[3]))); }
};

// what was unpacked from x before is not kept for what comes: 64 elements as floats are more than the registers hold
template <typename T, int NV> __device__ __forceinline__ void keep_packed(Vec<T> (&x)[NV]) {
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+r"(x[k].r[i]));
}

// a vector that is not aligned, or ends behind V: -inf there.  (Out of line: with eight of these in place warps waited for instructions more than for anything else.)
template <typename T> __device__ __noinline__ Vec<T> one_by_one(const T* s, int v, int V) {
  Vec<T> x;
#pragma unroll
  for (int i = 0; i < Vec<T>::E / 2; ++i)
    x.set(i, v + 2 * i < V ? ld_as_float(s, v + 2 * i) : -CUDART_INF_F, v + 2 * i + 1 < V ? ld_as_float(s, v + 2 * i + 1) : -CUDART_INF_F);
  return x;
}

struct BeamShared {
  alignas(16) float group_max[GROUPS];
  float warp_max[BWARPS];
  double warp_sum[BWARPS];
  uint64_t warp_best[BWARPS];
  float bar;
  unsigned vectors, count;
  alignas(16) uint4 vector[LIST];
  int vector_at[LIST];
  uint64_t list[LIST];
};

// NV: 16-byte vectors that a thread holds
template <typename T, int NV> __global__ void __launch_bounds__(BT, 5) beam_rows_kernel(const BeamParams p) {
  constexpr int E = Vec<T>::E;
  __shared__ BeamShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = p.in.V, n = p.in.n;
  const int64_t row = blockIdx.x / p.slices;
  const int slice = (int)(blockIdx.x - row * p.slices);
  wait_for_predecessor();
  launch_dependents();
  uint64_t* const cand = p.cand + (row * p.slices + slice) * n;
  double2* const part = p.part + row * p.slices + slice;
  if ((p.in.finished && p.in.finished[row]) || !(fabsf(p.in.score[row]) < CUDART_INF_F)) return;      // (the joining kernel does not look at its slices)
  const int64_t b = row / p.in.W;
  const T* const s = (const T*)p.in.logits + b * p.in.ld_seq + (row - b * p.in.W) * p.in.ld_beam;
  const bool vec = ((uintptr_t)s & 15) == 0;
  const int v0 = slice * p.slice;
  if (tid == 0) sh.count = sh.vectors = 0;
  Vec<T> x[NV];
  if (vec && v0 + NV * BT * E <= V) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint4 a = __ldg((const uint4*)(s + v0) + k * BT + tid);
      x[k].r[0] = a.x; x[k].r[1] = a.y; x[k].r[2] = a.z; x[k].r[3] = a.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = v0 + (k * BT + tid) * E;
      if (vec && v + E <= V) {
        const uint4 a = __ldg((const uint4*)(s + v));
        x[k].r[0] = a.x; x[k].r[1] = a.y; x[k].r[2] = a.z; x[k].r[3] = a.w;
      } else x[k] = one_by_one(s, v, V);
    }
  }
  float top[NV], mine = -CUDART_INF_F;
#pragma unroll
  for (int k = 0; k < NV; ++k) { top[k] = x[k].top(); mine = fmaxf(mine, top[k]); }
  float m = mine;
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
  if ((lane & 3) == 0) sh.group_max[tid >> 2] = m;
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh.warp_max[warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < BWARPS; ++w) m = fmaxf(m, sh.warp_max[w]);
  if (m == -CUDART_INF_F) {        // nothing but -inf (or NaN)
    bool nan = false;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) { const float2 a = x[k].pair(i); nan = nan || a.x != a.x || a.y != a.y; }
    nan = __syncthreads_or(nan);
    if (tid == 0) *part = make_double2(m, nan ? CUDART_NAN : 0.);
    for (int i = tid; i < n; i += BT) cand[i] = 0;
    return;
  }
  {                                // the bar: thread t compares group t / 4 with a quarter of the groups
    const float g = sh.group_max[tid >> 2];
    int more = 0, least = 0;       // groups above g, and those and its equals
#pragma unroll
    for (int i = 0; i < GROUPS / 4; i += 4) {
      const float4 y = *(const float4*)(sh.group_max + (tid & 3) * (GROUPS / 4) + i);
      more += (y.x > g) + (y.y > g) + (y.z > g) + (y.w > g);
      least += (y.x >= g) + (y.y >= g) + (y.z >= g) + (y.w >= g);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) { more += __shfl_xor_sync(0xffffffffu, more, o); least += __shfl_xor_sync(0xffffffffu, least, o); }
    if (more < n && n <= least) sh.bar = g;      // (the same value, whoever writes it)
  }
  // 2^(c x - r), r = c m as rounded to float32: what the rounding did is put right once, below.  The constant has two terms, as an error of the argument that is
  // the same for all elements would not average out; both are above 0, so that -inf stays -inf.
  float2 sum = make_float2(0.f, 0.f);
  const float2 hi = splat(p.c_hi), lo = splat(p.c_lo);
  const float r = fmaf(m, p.c_hi, m * p.c_lo);
  const bool far = !(fabsf(r) < 4096.f);      // the rounding is no small thing, or c x overflows: x - m first (where -inf must not meet the second term)
  if (!far) {
    const float2 nr = splat(-r);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const float2 y = x[k].pair(i);
        sum = fadd2(sum, ex2f2(ffma2(y, lo, ffma2(y, hi, nr))));
      }
  } else {
#pragma unroll 1
    for (int k = 0; k < NV * E / 2; ++k) {
      float2 y = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NV * E / 2; ++i)
        if (i == k) y = x[i / (E / 2)].pair(i % (E / 2));
      const float2 d = fadd2(y, splat(-m));
      sum = fadd2(sum, ex2f2(ffma2(d, hi, fmul2(make_float2(fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f)), lo))));
    }
  }
  double total = warp_sum((double)sum.x + (double)sum.y);
  if (lane == 0) sh.warp_sum[warp] = total;
  __syncthreads();
  const float bar = sh.bar;
  if (tid == 0) {
    total = 0;
    for (int w = 0; w < BWARPS; ++w) total += sh.warp_sum[w];
    if (!far) {                    // r - c m, of terms that are exact in float64
      const double t = (double)r - (double)m * ((double)p.c_hi + (double)p.c_lo);
      total *= fabs(t) < 1e-5 ? 1. + t * (0.69314718055994531 + t * 0.24022650695910071) : exp2(t);      // (two terms of the series, 6e-17 off)
    }
    *part = make_double2(m, total);
  }
  keep_packed(x);
  // vectors with an element that reaches the bar, then their elements, a thread each
  if (mine >= bar && mine > -CUDART_INF_F) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (top[k] >= bar) {
        const unsigned at = atomicAdd(&sh.vectors, 1u);
        if (at < LIST) {
          sh.vector[at] = make_uint4(x[k].r[0], x[k].r[1], x[k].r[2], x[k].r[3]);
          sh.vector_at[at] = v0 + (k * BT + tid) * E;
        }
      }
  }
  __syncthreads();
  const int vectors = (int)sh.vectors;
  for (int i = tid; i < min(vectors, LIST) * E; i += BT) {
    const float e = ld_as_float((const T*)(sh.vector + i / E), i % E);
    if (e >= bar && e > -CUDART_INF_F) {
      const unsigned at = atomicAdd(&sh.count, 1u);
      if (at < LIST) sh.list[at] = pair_word(e, (uint32_t)(sh.vector_at[i / E] + i % E));
    }
  }
  __syncthreads();
  const int count = (int)sh.count;
  if (count <= LIST && vectors <= LIST) {
    for (int i = tid; i < count; i += BT) {
      const uint64_t w = sh.list[i];
      int r = 0;
      for (int j = 0; j < count; ++j) r += sh.list[j] > w;
      if (r < n) cand[r] = w;
    }
    for (int i = count + tid; i < n; i += BT) cand[i] = 0;
  } else {                          // one by one: the largest word below the last
    uint64_t last = ~0ull;
#pragma unroll 1
    for (int r = 0; r < n; ++r) {
      uint64_t best = 0;
      keep_packed(x);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float2 a = x[k].pair(i >> 1);
          const float e = i & 1 ? a.y : a.x;
          const uint64_t w = e > -CUDART_INF_F ? pair_word(e, (uint32_t)(v0 + (k * BT + tid) * E + i)) : 0;
          if (w < last && w > best) best = w;
        }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = max(best, (uint64_t)__shfl_xor_sync(0xffffffffu, best, o));
      if (lane == 0) sh.warp_best[warp] = best;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < BWARPS; ++w) best = max(best, sh.warp_best[w]);
      __syncthreads();
      if (tid == 0) cand[r] = best;
      last = best;
    }
  }
}

// A candidate of a group.  `order` decides between equal keys: lower beams, then larger logits (keys of theirs may round to the same), then lower tokens first: an order
// that a beam's slices are sorted by as they are.  0: none.
struct Best { double key; uint64_t order; };
constexpr int TOKEN_BITS = 22, FEW = BT;
__device__ __forceinline__ uint64_t order_of(int w, uint32_t logit, uint32_t v) { return (uint64_t)(63 - w) << (32 + TOKEN_BITS) | (uint64_t)logit << TOKEN_BITS | ((1u << TOKEN_BITS) - 1 - v); }
__device__ __forceinline__ bool before(const Best& a, const Best& b) { return a.key > b.key || (a.key == b.key && a.order > b.order); }
__device__ __forceinline__ Best warp_first(Best a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Best u = {__shfl_xor_sync(0xffffffffu, a.key, o), __shfl_xor_sync(0xffffffffu, a.order, o)};
    if (before(u, a)) a = u;
  }
  return a;
}

__host__ __device__ constexpr int join_items(int n, int lists) { return lists <= FEW && lists > n * n ? lists : n * n; }

// A block per group.  Its n best lie in the n lists (one per beam and slice) whose heads are the best; those lists' elements are ranked by counting, each list being sorted.
// (Head after head, with a list's next element fetched when its head was taken, took 15 us for 64 groups of 80 lists, 8 to choose.)
__global__ void __launch_bounds__(BT) beam_join_kernel(const BeamParams p) {
  __shared__ double top[64], rest[64];     // the log-sum-exp of a beam is top / tau + rest
  __shared__ int how[64];           // 0: nothing to choose, 1: slices, 2: finished
  __shared__ Best first[2][BWARPS];
  __shared__ int list_of[64];
  __shared__ Best below[1];         // the last of n heads
  __shared__ int total;
  extern __shared__ __align__(16) unsigned char join_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = p.in.W, n = p.in.n, lists = W * p.slices;
  Best* const item = (Best*)join_smem;     // [n][n]; the heads of few lists before
  unsigned char* const taken = join_smem + join_items(n, lists) * sizeof(Best);      // of every list
  const int64_t b = blockIdx.x;
  wait_for_predecessor();
  launch_dependents();
  for (int i = tid; i < lists; i += BT) taken[i] = 0;
  if (tid == 0) total = 0;
  for (int w = warp; w < W; w += BWARPS) {
    const int64_t row = b * W + w;
    const float score = p.in.score[row];
    const bool done = p.in.finished && p.in.finished[row];
    bool bad = !(score < CUDART_INF_F);
    int h = 0;
    if (!bad && score > -CUDART_INF_F) {
      h = 2;
      if (!done) {
        float m = -CUDART_INF_F;
        bool nan = false;
        for (int s = lane; s < p.slices; s += 32) { const double2 a = p.part[row * p.slices + s]; m = fmaxf(m, (float)a.x); nan = nan || a.y != a.y; }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        bad = __any_sync(0xffffffffu, nan) || m == CUDART_INF_F;
        h = bad || m == -CUDART_INF_F ? 0 : 1;
        if (h) {
          double sum = 0;
          for (int s = lane; s < p.slices; s += 32) {
            const double2 a = p.part[row * p.slices + s];
            if (a.x > -CUDART_INF) sum += a.y * exp((a.x - (double)m) * p.inv_tau);
          }
          sum = warp_sum(sum);
          if (lane == 0) { top[w] = m; rest[w] = log(sum); }
        }
      }
    }
    if (lane == 0) {
      how[w] = h;
      if (p.out.row_status) p.out.row_status[row] = bad ? SAKI_ROW_NONFINITE : 0u;
      if (bad) atomicAdd(p.flagged, 1ull);
    }
  }
  __syncthreads();
  const Best none = {-CUDART_INF, 0};
  auto element = [&](int l, int k) -> Best {
    const int w = l / p.slices, s = l - w * p.slices;
    const double score = (double)p.in.score[b * W + w];
    if (how[w] == 2) return s == 0 && k == 0 ? Best{score, order_of(w, 0x80000000u, p.in.pad)} : none;
    if (how[w] == 0) return none;
    const uint64_t c = p.cand[((b * W + w) * p.slices + s) * n + k];
    return c == 0 ? none : Best{score + (((double)pair_logit(c) - top[w]) * p.inv_tau - rest[w]), order_of(w, (uint32_t)(c >> 32), pair_token(c))};
  };
  // the best heads
  Best mine = none;
  int from = -1;
  auto look = [&] {
    mine = none;
    for (int l = tid; l < lists; l += BT) {
      const Best h = taken[l] ? none : element(l, 0);
      if (before(h, mine)) { mine = h; from = l; }
    }
  };
  int chosen = 0;
  Best last = none;
  if (lists <= FEW) {              // a thread a list: by counting
    if (tid < lists) item[tid] = mine = element(tid, 0);
    if (tid == 0) below[0] = none;
    __syncthreads();
    if (tid < lists && mine.order != 0) {
      int rank = 0;
#pragma unroll 4
      for (int l = 0; l < lists; ++l) rank += before(item[l], mine);
      if (rank < n) list_of[rank] = tid;
      if (rank == n - 1) below[0] = mine;
    }
    chosen = min(n, __syncthreads_count(mine.order != 0));
    last = below[0];
    __syncthreads();
  } else look();
#pragma unroll 1
  for (; lists > FEW && chosen < n; ++chosen) {
    Best a = warp_first(mine);
    if (lane == 0) first[chosen & 1][warp] = a;
    __syncthreads();               // (the other half is written only behind the next)
    a = first[chosen & 1][0];
#pragma unroll
    for (int w = 1; w < BWARPS; ++w)
      if (before(first[chosen & 1][w], a)) a = first[chosen & 1][w];
    if (a.order == 0) break;
    if (mine.order == a.order) { list_of[chosen] = from; taken[from] = 1; look(); }
    last = a;
  }
  __syncthreads();
  int there = 0;
  for (int i = tid; i < chosen * n; i += BT) {
    const Best e = element(list_of[i / n], i % n);
    item[i] = e;
    there += e.order != 0;
  }
  if (there) atomicAdd(&total, there);
  __syncthreads();
  for (int i = tid; i < chosen * n; i += BT) {
    const Best e = item[i];
    if (e.order == 0 || (chosen == n && before(last, e))) continue;      // (n heads come before it)
    const int j = i / n;
    int rank = i - j * n;
    for (int o = 0; o < chosen && rank < n; ++o) {
      if (o == j) continue;
      int lo = 0, hi = n;          // elements of list o before e
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (before(item[o * n + mid], e)) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank < n) {
      p.out.parent[b * n + rank] = 63 - (int)(e.order >> (32 + TOKEN_BITS));
      p.out.token[b * n + rank] = (1 << TOKEN_BITS) - 1 - (int)(e.order & ((1u << TOKEN_BITS) - 1));
      p.out.score[b * n + rank] = (float)e.key;
    }
  }
  for (int r = total + tid; r < n; r += BT) {
    p.out.parent[b * n + r] = -1;
    p.out.token[b * n + r] = -1;
    p.out.score[b * n + r] = -CUDART_INF_F;
  }
}

struct Layout { int nv, slice, slices; };
constexpr int MAX_SMS = 256;
// Slices as long as a thread's registers hold (eight vectors); shorter ones for few rows, so that there are two blocks for every
// SM.  (V has at most 2^22 entries, so the lists of a group fit into the joining kernel's shared memory.)
Layout layout(int64_t rows, int V, int dtype, int sms) {
  const int e = dtype == SAKI_BF16 ? 8 : 4;
  for (int nv = 8;; nv /= 2) {
    const int slice = BT * nv * e, slices = (V + slice - 1) / slice;
    if (nv == 1 || rows * slices >= 2 * std::min(sms, MAX_SMS)) return {nv, slice, slices};
  }
}
int sm_count() {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
int64_t round256(int64_t x) { return (x + 255) & ~(int64_t)255; }

}  // namespace

// enough for either type and any number of SMs: slices of eight vectors, or, shorter, fewer than four for every SM
int64_t beam_scratch_bytes(int64_t B, int32_t W, int32_t V, int32_t n) {
  const int64_t rows = B * W, longest = BT * 8 * 4, most = std::max<int64_t>(rows * ((V + longest - 1) / longest), 4 * MAX_SMS);
  return round256(most * n * 8) + round256(most * 16);
}

cudaError_t launch_beams(const saki_beam_in& in, const saki_beam_out& out, void* scratch, unsigned long long* flagged, cudaStream_t st) {
  const int64_t rows = in.B * in.W;
  const Layout l = layout(rows, in.V, in.dtype, sm_count());
  BeamParams p = {};
  p.in = in; p.out = out; p.slices = l.slices; p.slice = l.slice; p.flagged = flagged;
  const double c = 1.4426950408889634 / (double)in.temperature;
  p.inv_tau = 1.0 / (double)in.temperature;
  p.c_hi = (float)c;
  if ((double)p.c_hi >= c) p.c_hi = std::nextafter(p.c_hi, 0.f);
  p.c_lo = std::max((float)(c - (double)p.c_hi), std::numeric_limits<float>::denorm_min());      // above 0
  p.cand = (uint64_t*)scratch;
  p.part = (double2*)((char*)scratch + round256(rows * l.slices * in.n * 8));
  const dim3 grid((unsigned)(rows * l.slices));
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, BT, 0, st, true, p); };
  cudaError_t e;
  if (in.dtype == SAKI_BF16) {
    using T = __nv_bfloat16;
    e = l.nv == 8 ? go(beam_rows_kernel<T, 8>) : l.nv == 4 ? go(beam_rows_kernel<T, 4>) : l.nv == 2 ? go(beam_rows_kernel<T, 2>) : go(beam_rows_kernel<T, 1>);
  } else
    e = l.nv == 8 ? go(beam_rows_kernel<float, 8>) : l.nv == 4 ? go(beam_rows_kernel<float, 4>) : l.nv == 2 ? go(beam_rows_kernel<float, 2>) : go(beam_rows_kernel<float, 1>);
  if (e != cudaSuccess) return e;
  const size_t bytes = join_items(in.n, in.W * l.slices) * sizeof(Best) + (size_t)in.W * l.slices;
  constexpr int most = 64 * 64 * (int)sizeof(Best) + 64 * 512;      // (the same for every call: two threads may be here; 64 beams of 512 slices)
  e = cudaFuncSetAttribute(beam_join_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  return e != cudaSuccess ? e : launch_pdl(beam_join_kernel, dim3((unsigned)in.B), BT, bytes, st, true, p);
}

}  // namespace saki
