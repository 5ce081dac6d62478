// The k largest logits of every row, sorted, and the row's log-sum-exp: what is kept of a teacher's row for distillation.
//
// A row (or a slice of it, where there are few rows) is read once by a block of 256 threads: every thread takes 16-byte pieces 256 apart, sums their exponentials
// under a shift of its own, and leaves the upper 16 bits of the largest element of each group of its pieces, as an ordered key, in shared memory.  The k-th largest of the threads'
// maxima is a bar that the slice's k-th largest logit reaches, and that little more than k elements reach: only the groups that reach it are read again (some k of
// ten thousand), what reaches it in them is ranked by counting.  Where the largest lie in few threads' pieces the list overflows, and the bar is found by counting elements; where hundreds
// of them are equal, too, the best are taken one by one, each thread offering its best that is left.
// Slices of a row are joined by a second kernel.
//
// What bounds it: 4096 bf16 rows of 151936, 64 best, 234 to 245 us (by card) where the bytes take 190 (80 %): the special-function pipe at 60 % in the pass, and a row's tail (bar, second reading, ranks: some 5 us that other
// blocks of the SM cover in part).  float32 rows of 151936: 95 %.  2960 rows of 2048: 30 us, all tails.  8 rows: 13 us, two launches and the two tails' chains.
#include "saki_device.cuh"
#include <algorithm>
#include <climits>

namespace saki {

namespace {

constexpr int TT = 256, TWARPS = TT / 32, LIST = 512, KMAX = 128;
constexpr int MAX_ENTRIES = 10240;          // groups of a slice: 20 KB of keys
static_assert(((1 << 22) / (MAX_ENTRIES * 16) + 2) * KMAX * 8 + LIST * 8 + 64 <= 48 * 1024, "the lists of a row's slices are joined in shared memory");
constexpr int MIN_SLICES = 16;              // a row is cut in so many at the most, unless it is longer than that
constexpr float MARGIN = 60.f;

struct TopParams {
  saki_top_in in;
  saki_top_out out;
  int slices, pieces;       // per row, and 16-byte pieces of one
  float c;                  // log2(e) / temperature
  uint64_t* cand;           // [N][slices][k] a slice's best, 0: none (slices > 1)
  double2* part;            // [N][slices] (shift, sum); a NaN: flagged
  unsigned long long* flagged;
};

// a pair (logit, token) as one word: larger logits first, then lower tokens
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);      // (-0 counts as 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t pair_word(float x, int v) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - (uint32_t)v); }
__device__ __forceinline__ float pair_logit(uint64_t w) {
  const uint32_t o = (uint32_t)(w >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int pair_token(uint64_t w) { return (int)(0xffffffffu - (uint32_t)w); }
constexpr uint32_t LEAST = 0x0080u;                 // key of the lowest finite value; of -inf: 0x007f, of no element: 0

template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> {
  static constexpr int E = 8;
  static constexpr uint32_t FILLER = 0xFF80FF80u;   // -inf
  static __device__ __forceinline__ float2 pair(const uint4& w, int i) { return unpack_bf16x2(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
  template <int GROUP> static __device__ __forceinline__ float top(const uint4 (&w)[GROUP]) {      // (of a pair with a NaN the other)
    uint32_t a = w[0].x;
#pragma unroll
    for (int g = 0; g < GROUP; ++g) a = max_bf16x2(a, max_bf16x2(max_bf16x2(w[g].x, w[g].y), max_bf16x2(w[g].z, w[g].w)));
    const float2 f = unpack_bf16x2(a);
    return fmaxf(f.x, f.y);
  }
};
template <> struct Piece<float> {
  static constexpr int E = 4;
  static constexpr uint32_t FILLER = 0xFF800000u;
  static __device__ __forceinline__ float2 pair(const uint4& w, int i) { return i == 0 ? make_float2(__uint_as_float(w.x), __uint_as_float(w.y)) : make_float2(__uint_as_float(w.z), __uint_as_float(w.w)); }
  template <int GROUP> static __device__ __forceinline__ float top(const uint4 (&w)[GROUP]) {
    float m = -CUDART_INF_F;
#pragma unroll
    for (int g = 0; g < GROUP; ++g) m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[g].x), __uint_as_float(w[g].y)), fmaxf(__uint_as_float(w[g].z), __uint_as_float(w[g].w))));
    return m;
  }
};

struct TopShared {
  uint64_t list[LIST], best[KMAX];
  double sum[TWARPS];
  float shift[TWARPS];
  uint64_t warp_best[TWARPS];
  uint32_t top[TT];
  uint32_t bar, most, groups, count;
  int warp_count[TWARPS];
  double slice_shift, slice_sum;
  int group[LIST];
  uint16_t key[MAX_ENTRIES];
};

// GROUP: pieces to a key.  (With four of them a thread holds too many for six blocks on an SM.)
template <typename T, int GROUP>
__global__ void __launch_bounds__(TT, GROUP == 2 ? 6 : 5) top_rows_kernel(const TopParams P) {
  using Pc = Piece<T>;
  constexpr int E = Pc::E;
  __shared__ TopShared sh;
  launch_dependents();
  wait_for_predecessor();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = P.in.V, k = P.in.k;
  const int64_t row = blockIdx.x / P.slices;
  const int slice = (int)(blockIdx.x - row * P.slices);
  // the row in pieces that start on 16-byte boundaries; the first and the last may hold elements of other rows
  const uintptr_t addr = (uintptr_t)((const T*)P.in.logits + row * P.in.ld);
  const uint4* const base = (const uint4*)(addr & ~(uintptr_t)15);
  const int head = (int)((addr & 15) / sizeof(T));
  const int p0 = slice * P.pieces, p1 = min((V + head + E - 1) / E, slice == P.slices - 1 ? INT_MAX : p0 + P.pieces);
  const int f0 = head ? 1 : 0, f1 = (V + head) / E;      // whole pieces
  const int entries = (p1 - p0 + TT * GROUP - 1) / (TT * GROUP);      // groups of a thread
  auto load = [&](int p) -> uint4 {
    if (p >= f0 && p < f1 && p < p1) return __ldg(base + p);
    uint4 w = make_uint4(Pc::FILLER, Pc::FILLER, Pc::FILLER, Pc::FILLER);
    if (p < p1) {
      T* const e = (T*)&w;
      const T* const s = (const T*)(base + p);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (p * E + i >= head && p * E + i < head + V) e[i] = s[i];
    }
    return w;
  };
  if (tid == 0) sh.groups = sh.count = 0;

  // ------------------------------------------------ the pass over the slice
  float2 S0 = splat(0.f), S1 = splat(0.f);
  float shift = 0.f, limit = -CUDART_INF_F;      // (the first group sets them)
  uint32_t mine = 0;
  const float2 cc = splat(P.c);
  uint4 next[GROUP];                   // on their way
#pragma unroll
  for (int g = 0; g < GROUP; ++g) next[g] = load(p0 + g * TT + tid);
#pragma unroll 1
  for (int i = 0; i < entries; ++i) {
    uint4 w[GROUP];
#pragma unroll
    for (int g = 0; g < GROUP; ++g) w[g] = next[g];
    if (i + 1 < entries) {
#pragma unroll
      for (int g = 0; g < GROUP; ++g) next[g] = load(p0 + ((i + 1) * GROUP + g) * TT + tid);
    }
    const float top = Pc::top(w);
    const uint32_t key = order_of(top) >> 16;
    sh.key[i * TT + tid] = (uint16_t)key;
    mine = max(mine, key);
    if (top > limit) {                 // a new shift; sums so far go along
      const float to = -ceilf(fminf(fmaxf(P.c * top, -1e8f), 3e38f)), f = ex2f(fmaxf(to - shift, -200.f));
      if (limit > -CUDART_INF_F) { S0 = fmul2(S0, splat(f)); S1 = fmul2(S1, splat(f)); }
      shift = to;
      limit = (MARGIN - shift) / P.c;
    }
    const float2 kk = splat(shift);
#pragma unroll
    for (int g = 0; g < GROUP; ++g)
#pragma unroll
      for (int j = 0; j < E / 2; j += 2) {
        S0 = fadd2(S0, ex2f2(ffma2(Pc::pair(w[g], j), cc, kk)));
        S1 = fadd2(S1, ex2f2(ffma2(Pc::pair(w[g], j + 1), cc, kk)));
      }
  }
  // the sum, under the lowest shift
  float low = limit > -CUDART_INF_F ? shift : CUDART_INF_F;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
  double total = ((double)S0.x + (double)S0.y) + ((double)S1.x + (double)S1.y);
  if (limit > -CUDART_INF_F) total *= (double)ex2f(fmaxf(low - shift, -200.f));
  total = warp_sum(total);
  if (lane == 0) { sh.sum[warp] = total; sh.shift[warp] = low; }
  sh.top[tid] = mine;
  __syncthreads();
  if (warp == 0) {
    // the k-th largest of the threads' maxima: bisection between the smallest and the largest of them
    uint32_t x[TT / 32], lo = ~0u, hi = 0;
#pragma unroll
    for (int i = 0; i < TT / 32; ++i) { x[i] = sh.top[i * 32 + lane]; lo = min(lo, x[i]); hi = max(hi, x[i]); }
    uint32_t bar = __reduce_min_sync(0xffffffffu, lo);      // (k of them reach it: there are more than k threads)
    hi = __reduce_max_sync(0xffffffffu, hi);
#pragma unroll 1
    while (bar < hi) {
      const uint32_t to = (bar + hi + 1) >> 1;
      int n = 0;
#pragma unroll
      for (int i = 0; i < TT / 32; ++i) n += x[i] >= to;
      if (__reduce_add_sync(0xffffffffu, n) >= k) bar = to;
      else hi = to - 1;
    }
    if (lane == 0) sh.bar = max(bar, LEAST);
  } else if (warp == 1) {
    const float s = lane < TWARPS ? sh.shift[lane] : CUDART_INF_F;
    float m = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fminf(m, __shfl_xor_sync(0xffffffffu, m, o));
    double t = lane < TWARPS ? sh.sum[lane] * (s < CUDART_INF_F ? (double)ex2f(fmaxf(m - s, -200.f)) : 1.0) : 0;      // (without a shift: 0, or a NaN)
    t = warp_sum(t);
    uint32_t most = 0;
    for (int i = lane; i < TT; i += 32) most = max(most, sh.top[i]);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) { sh.slice_shift = (double)m; sh.slice_sum = t; sh.most = most; }
  }
  __syncthreads();
  const uint32_t bar = sh.bar;
  double slice_shift = sh.slice_shift, slice_sum = sh.slice_sum;
  if (!(fabs(slice_shift) < 4e6) && slice_shift < CUDART_INF) {
    // logits of millions, where 2^(c x + shift) would take a difference of rounded numbers: once more, under the largest itself
    float m = -CUDART_INF_F;
    auto each = [&](auto&& body) {
#pragma unroll 1
      for (int p = p0 + tid; p < p1; p += TT) {
        const uint4 w = load(p);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) { const float2 a = Pc::pair(w, j); body(a.x); body(a.y); }
      }
    };
    each([&](float x) { m = fmaxf(m, x); });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) sh.shift[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TWARPS; ++w) m = fmaxf(m, sh.shift[w]);
    float part = 0.f;
    each([&](float x) { part += ex2f((x - m) * P.c); });
    const double t = warp_sum((double)part);
    if (lane == 0) sh.sum[warp] = t;
    __syncthreads();
    slice_sum = 0;
#pragma unroll
    for (int w = 0; w < TWARPS; ++w) slice_sum += sh.sum[w];
    slice_shift = -(double)P.c * (double)m;
  }
  // sum of exp(x / tau) = exp(x0 / tau) sum of 2^(c (x - x0)), x0 = -shift / c
  const double lse = slice_sum > 0 ? LN2 * log2(slice_sum) - slice_shift / (double)P.c / (double)P.in.temperature : -CUDART_INF;
  const bool bad = !(slice_sum < CUDART_INF) || sh.most >= 0xff80u || (float)lse == CUDART_INF_F;      // NaN, +inf (whose key is 0xff80)
  if (tid == 0) {
    if (P.slices > 1) P.part[row * P.slices + slice] = make_double2(bad ? CUDART_NAN : slice_shift, slice_sum);
    else {
      if (P.out.lse) P.out.lse[row] = bad ? 0.f : (float)lse;
      if (P.out.row_status) P.out.row_status[row] = bad ? SAKI_ROW_NONFINITE : 0u;
      if (bad) atomicAdd(P.flagged, 1ull);
    }
  }
  if (!bad) {
    // ------------------------------------------------ groups that reach the bar, and what reaches it in them
    auto collect = [&](uint32_t bar) -> bool {      // whether it is all in the list
      if (mine >= bar)
        for (int i = 0; i < entries; ++i)
          if (sh.key[i * TT + tid] >= bar) {
            const unsigned at = atomicAdd(&sh.groups, 1u);
            if (at < LIST) sh.group[at] = i * TT + tid;
          }
      __syncthreads();
      const int groups = (int)sh.groups;
      if (groups <= LIST)
        for (int i = tid; i < groups * GROUP; i += TT) {
          const int g = sh.group[i / GROUP], at = g / TT, p = p0 + (at * GROUP + i % GROUP) * TT + (g - at * TT);
          const uint4 w = load(p);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float2 a = Pc::pair(w, j >> 1);
            const float x = j & 1 ? a.y : a.x;
            if (order_of(x) >> 16 >= bar && x > -CUDART_INF_F) {
              const unsigned n = atomicAdd(&sh.count, 1u);
              if (n < LIST) sh.list[n] = pair_word(x, p * E + j - head);
            }
          }
        }
      __syncthreads();
      return groups <= LIST && sh.count <= LIST;
    };
    bool all = collect(bar);
    if (!all) {
      // the largest lie in few threads' pieces (or there are fewer threads with any than k): the bar goes up to the k-th largest itself, by counting what reaches it
      uint32_t lo = bar, hi = sh.most;
#pragma unroll 1
      while (lo < hi) {
        const uint32_t to = (lo + hi + 1) >> 1;
        int n = 0;
        if (mine >= to)
#pragma unroll 1
          for (int i = 0; i < entries; ++i)
            if (sh.key[i * TT + tid] >= to)
#pragma unroll
              for (int g = 0; g < GROUP; ++g) {
                const uint4 w = load(p0 + (i * GROUP + g) * TT + tid);
#pragma unroll
                for (int j = 0; j < E / 2; ++j) { const float2 a = Pc::pair(w, j); n += (order_of(a.x) >> 16 >= to) + (order_of(a.y) >> 16 >= to); }
              }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) sh.warp_count[warp] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int w = 0; w < TWARPS; ++w) n += sh.warp_count[w];
        __syncthreads();
        if (n >= k) lo = to;
        else hi = to - 1;
      }
      __syncthreads();      // (all have read the counts, also where there was nothing to bisect)
      if (tid == 0) sh.groups = sh.count = 0;
      __syncthreads();
      all = collect(lo);
    }
    const int count = (int)sh.count;
    if (all) {
      // ranks by counting, one to four threads an element
      const int parts = count <= TT / 4 ? 4 : count <= TT / 2 ? 2 : 1, step = TT / parts;
      for (int i0 = warp * 32 / parts; i0 < count; i0 += step) {      // (the same for all threads of a warp: they exchange)
        const int i = i0 + lane / parts;
        const uint64_t w = sh.list[min(i, count - 1)];
        int r = 0;
#pragma unroll 4
        for (int j = tid % parts; j < count; j += parts) r += sh.list[j] > w;
        if (parts > 1) r += __shfl_xor_sync(0xffffffffu, r, 1);
        if (parts > 2) r += __shfl_xor_sync(0xffffffffu, r, 2);
        if (i < count && r < k && tid % parts == 0) sh.best[r] = w;
      }
      for (int i = count + tid; i < k; i += TT) sh.best[i] = 0;
    } else {
      // one by one: every thread offers the best of its pieces that comes behind the last one taken
      uint64_t last = ~0ull, offer = 0;
      bool look = true;
#pragma unroll 1
      for (int r = 0; r < k; ++r) {
        if (look) {
          offer = 0;
          bool done = false;
#pragma unroll 1
          for (int i = 0; i < entries && !done; ++i) {
            if (sh.key[i * TT + tid] < (uint32_t)(offer >> 48)) continue;
#pragma unroll 1
            for (int g = 0; g < GROUP && !done; ++g) {
              const int p = p0 + (i * GROUP + g) * TT + tid;
              if (p >= p1) break;
              const uint4 w = load(p);
#pragma unroll
              for (int j = 0; j < E; ++j) {
                const float2 a = Pc::pair(w, j >> 1);
                const float x = j & 1 ? a.y : a.x;
                const uint64_t word = x > -CUDART_INF_F ? pair_word(x, p * E + j - head) : 0;
                if (word < last && word > offer) offer = word;
              }
              done = (uint32_t)(offer >> 32) == (uint32_t)(last >> 32);      // an equal of the last: no better one is behind it
            }
          }
          look = false;
        }
        uint64_t a = offer;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a = max(a, (uint64_t)__shfl_xor_sync(0xffffffffu, a, o));
        if (lane == 0) sh.warp_best[warp] = a;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TWARPS; ++w) a = max(a, sh.warp_best[w]);
        __syncthreads();
        if (tid == 0) sh.best[r] = a;
        last = a;
        look = a != 0 && a == offer;
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < k; i += TT) {
    const uint64_t w = bad ? 0 : sh.best[i];
    if (P.slices > 1) P.cand[(row * P.slices + slice) * k + i] = w;
    else {
      P.out.token[row * k + i] = w ? pair_token(w) : -1;
      P.out.logit[row * k + i] = w ? pair_logit(w) : bad ? 0.f : -CUDART_INF_F;
    }
  }
}

// A block a row: the slices' sorted lists become one.  The least of the lists' ceil(k / slices)-th elements is a bar that k elements reach, and twice as many or so do: those are ranked by counting.
// Where more of them do than LIST, by their places in all lists.
__global__ void __launch_bounds__(TT) top_join_kernel(const TopParams P) {
  __shared__ int total, above;
  __shared__ bool bad;
  __shared__ unsigned long long bar;
  __shared__ uint64_t list[LIST];
  extern __shared__ uint64_t c[];      // [slices][k]
  launch_dependents();
  wait_for_predecessor();
  const int tid = threadIdx.x, lane = tid & 31, k = P.in.k, n = P.slices;
  const int64_t row = blockIdx.x;
  for (int i = tid; i < n * k; i += TT) c[i] = P.cand[row * n * k + i];
  if (tid == 0) { total = above = 0; bar = ~0ull; }
  __syncthreads();
  if (tid < 32) {
    double m = CUDART_INF, s = 0;
    bool nan = false;
    for (int i = lane; i < n; i += 32) { const double2 a = P.part[row * n + i]; nan |= a.x != a.x; m = fmin(m, a.x); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmin(m, __shfl_xor_sync(0xffffffffu, m, o));
    nan = __any_sync(0xffffffffu, nan);
    for (int i = lane; i < n; i += 32) {
      const double2 a = P.part[row * n + i];
      if (a.y > 0) s += a.y * exp2(m - a.x);
    }
    s = warp_sum(s);
    if (lane == 0) {
      bad = nan;
      const double lse = s > 0 ? LN2 * log2(s) - m / (double)P.c / (double)P.in.temperature : -CUDART_INF;
      if (P.out.lse) P.out.lse[row] = nan ? 0.f : (float)lse;
      if (P.out.row_status) P.out.row_status[row] = nan ? SAKI_ROW_NONFINITE : 0u;
      if (nan) atomicAdd(P.flagged, 1ull);
    }
  } else if (tid < 64) {
    unsigned long long b = ~0ull;
    for (int l = lane; l < n; l += 32) b = min(b, (unsigned long long)c[l * k + (k + n - 1) / n - 1]);
    atomicMin(&bar, b);
  }
  __syncthreads();
  if (!bad) {
    const uint64_t least = max((unsigned long long)bar, 1ull);      // (0: a list falls short)
    int there = 0;
    for (int i = tid; i < n * k; i += TT) {
      const uint64_t w = c[i];
      there += w != 0;
      if (w >= least) {
        const int at = atomicAdd(&above, 1);
        if (at < LIST) list[at] = w;
      }
    }
    if (there) atomicAdd(&total, there);
    __syncthreads();
    const int m = above;
    auto write = [&](int rank, uint64_t w) {
      P.out.token[row * k + rank] = pair_token(w);
      P.out.logit[row * k + rank] = pair_logit(w);
    };
    if (m <= LIST) {
      for (int i = tid; i < m; i += TT) {
        const uint64_t w = list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < m; ++j) rank += list[j] > w;
        if (rank < k) write(rank, w);
      }
    } else {
      for (int i = tid; i < n * k; i += TT) {
        const uint64_t w = c[i];
        if (w < least) continue;
        const int own = i / k;
        int rank = i - own * k;
        for (int l = 0; l < n && rank < k; ++l) {
          if (l == own) continue;
          int lo = 0, hi = k;            // elements of list l before w
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (c[l * k + mid] > w) lo = mid + 1;
            else hi = mid;
          }
          rank += lo;
        }
        if (rank < k) write(rank, w);
      }
    }
  }
  __syncthreads();
  for (int i = (bad ? 0 : total) + tid; i < k; i += TT) {
    P.out.token[row * k + i] = -1;
    P.out.logit[row * k + i] = bad ? 0.f : -CUDART_INF_F;
  }
}

struct Cut { int slices, pieces, group; };
constexpr int MAX_SMS = 256;
// Slices as long as the keys' room; shorter ones for few rows, so that there are two blocks for every SM, of 256 pieces (one a thread) at the least and MIN_SLICES at the most.
Cut cut(int64_t rows, int V, int dtype, int sms) {
  const int e = dtype == SAKI_BF16 ? 8 : 4, all = (V + 2 * e - 2) / e;
  // float32: four pieces to a key keep more bytes on their way, two leave room for six blocks on an SM, not five (2960 rows, 64 best: of 2048 32 and 27 us, of 16384 54 and 53, of 32003 84 and 88, of
  // 65536 142 and 150).  Rows of up to 65536 take two where that is a round of blocks less (1500 rows of 32003 52 and 48, 760 of 65536 53 and 43, 1700 92 and 85; longer rows gain too
  // little by it: 1500 of 100000 124 and 132).
  auto rounds = [&](int blocks) { return (rows + (int64_t)blocks * sms - 1) / ((int64_t)blocks * sms); };
  const int group = dtype == SAKI_BF16 || V <= 20480 || (V <= 65536 && rounds(6) < rounds(5)) ? 2 : 4, longest = MAX_ENTRIES * group;
  const int need = (all + longest - 1) / longest;
  int64_t want = (2 * (int64_t)std::min(sms, MAX_SMS) + rows - 1) / std::max<int64_t>(rows, 1);
  want = std::max<int64_t>(need, std::min<int64_t>({want, (int64_t)std::max(MIN_SLICES, need), (int64_t)std::max(1, all / TT)}));
  const int pieces = (int)((all + want - 1) / want);
  return {(all + pieces - 1) / pieces, pieces, group};
}
int sm_count() {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
int64_t round256(int64_t x) { return (x + 255) & ~(int64_t)255; }

}  // namespace

// enough for either type and any number of SMs up to MAX_SMS
int64_t top_scratch_bytes(int64_t N, int32_t V, int32_t k) {
  int64_t most = 0;
  for (int dtype : {SAKI_F32, SAKI_BF16}) most = std::max<int64_t>(most, cut(N, V, dtype, MAX_SMS).slices);
  return 256 + (most > 1 ? round256(N * most * k * 8) + round256(N * most * 16) : 0);
}

cudaError_t launch_top(const saki_top_in& in, const saki_top_out& out, void* scratch, unsigned long long* flagged, int* n_launches, cudaStream_t st) {
  const Cut c = cut(in.N, in.V, in.dtype, sm_count());
  TopParams p = {};
  p.in = in; p.out = out; p.slices = c.slices; p.pieces = c.pieces; p.flagged = flagged;
  p.c = (float)(INV_LN2 / (double)in.temperature);
  p.cand = (uint64_t*)scratch;
  p.part = (double2*)((char*)scratch + round256(in.N * c.slices * in.k * 8));
  const dim3 grid((unsigned)(in.N * c.slices));
  cudaError_t e = in.dtype == SAKI_BF16 ? launch_pdl(top_rows_kernel<__nv_bfloat16, 2>, grid, TT, 0, st, true, p)
                  : c.group == 2    ? launch_pdl(top_rows_kernel<float, 2>, grid, TT, 0, st, true, p)
                                    : launch_pdl(top_rows_kernel<float, 4>, grid, TT, 0, st, true, p);
  *n_launches = 1;
  if (e != cudaSuccess || c.slices == 1) return e;
  ++*n_launches;
  return launch_pdl(top_join_kernel, dim3((unsigned)in.N), TT, (size_t)c.slices * in.k * 8, st, true, p);
}

}  // namespace saki
