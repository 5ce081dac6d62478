// What the attention kernels share: the line of tiles and its pieces, what a query sees, how results are written or left to be joined.
#pragma once
#include "saki_device.cuh"
#include "saki_tensor_map.cuh"
#include <algorithm>
#include <cmath>

namespace saki {

namespace attn {

// Tensor maps of a pool.  MAP_BOXES: (column, head, position, page), boxes of 128 bytes by `box` positions.  The others, for D = 128: (column of a half, position
// of eight, half, eights of positions, the rest), boxes of all 256 bytes of their positions, where five dimensions say where these lie: heads are
// side by side (halves and heads are one dimension), pages hold one head after the other (pages and heads are one), or positions run on from page to page (eights
// and pages are one).
enum { MAP_BOXES = 0, MAP_HEADS, MAP_PAGES, MAP_RUN };

struct AttnParams {
  saki_attn_in in;
  saki_attn_out out;
  int G, R, RB;             // query heads per key head; rows of a key head (Q * G); blocks of rows
  int q_vec;                // q can be read in 16-byte pieces
  int box;                  // positions of a TMA box
  int map_mode;             // how the tensor maps see a pool: MAP_*
  int page_shift;           // page_size is 1 << page_shift; -1: no power of two
  uint32_t q_sign;          // a negative scale turns the queries' signs
  float c;                  // |scale| * log2(e), above 0
  int4* desc;               // [workers] the segment that starts in a piece and goes on: (b, head and row block, pieces behind, status)
  float* part;              // [workers][2] partial results: of the segment that goes on from the piece before, of the one that goes on behind
  int2* late;               // [workers] first and last sequence of those with a segment for which a wait of the worker ran out; (0, -1): none
  unsigned long long* flagged;
  long long wait_limit;
};

__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int x, int head, int slot, int page, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(head), "r"(slot), "r"(page), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tma_eights(uint32_t dst, const CUtensorMap* map, int c2, int c3, int c4, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(0), "r"(c2), "r"(c3), "r"(c4), "r"(smem_addr(bar)) : "memory");
}
// What the queries of a sequence see, in tiles of T positions: the tiles of the first `sk` positions, then those from tile m0 on.  (Positions are
// below 2^31.)
struct Span {
  int n, p0, nq, lo, sk, ns, m0, nt;
  uint32_t status;
};
template <int T> __device__ __forceinline__ Span span_of(const AttnParams& p, int64_t b) {
  Span s;
  s.n = p.in.length[b];
  s.nq = p.in.n_query ? p.in.n_query[b] : p.in.Q;
  s.status = p.in.row_status ? p.in.row_status[b] : 0u;      // (refused when positions were reserved)
  if (s.status) s.n = s.nq = 0;
  else if (s.n < 0 || (int64_t)s.n > (int64_t)p.in.max_pages * p.in.page_size || s.nq < 0 || s.nq > p.in.Q) { s.status = SAKI_ROW_BAD_LENGTH; s.n = 0; s.nq = 0; }
  s.p0 = s.n - s.nq;
  s.lo = p.in.window > 0 ? (int)max((int64_t)0, (int64_t)s.p0 - p.in.window + 1) : 0;
  if (s.nq == 0) s.lo = s.n;
  s.sk = s.nq == 0 ? 0 : min(p.in.sinks, s.lo);
  s.ns = (int)(((unsigned)s.sk + T - 1) / T);
  s.m0 = max(s.lo / T, s.ns);
  s.nt = max(1, s.ns + max(0, (int)(((unsigned)s.n + T - 1) / T) - s.m0));
  return s;
}
template <int T> __device__ __forceinline__ int tile_start(const Span& s, int t) { return (t < s.ns ? t : s.m0 + t - s.ns) * T; }

// A place on the line of tiles: sequence, key head and row block, tile.
template <int T> struct Cursor {
  int b, hr, t;
  Span s;
  __device__ __forceinline__ void at(const AttnParams& p, int64_t b_, int64_t offset) {
    b = (int)b_;
    s = span_of<T>(p, b);
    hr = (int)(offset / s.nt);
    t = (int)(offset - (int64_t)hr * s.nt);
  }
  __device__ __forceinline__ void next(const AttnParams& p) {
    if (++t < s.nt) return;
    t = 0;
    if (++hr < p.in.H * p.RB) return;
    hr = 0;
    if (++b < p.in.B) s = span_of<T>(p, b);
  }
};

template <int THREADS> struct LineShared {
  long long sum[THREADS / 32];
  long long b[THREADS / 32], before[THREADS / 32];      // by worker of the block: the sequence of its first tile, tiles in front of it
};
// The pieces of a block's workers [u0, u0 + chunk) of the line: worker w of block i is number w * blocks + i (few tiles: one worker on each SM).  Every
// block adds up all sequences' tiles, a few per thread.
template <int T, int THREADS, int WORKERS> __device__ __forceinline__ void pieces(const AttnParams& p, LineShared<THREADS>& sh, long long& chunk, long long& total) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t per = (p.in.B + THREADS - 1) / THREADS, b0 = min((int64_t)tid * per, p.in.B), b1 = min(b0 + per, p.in.B);
  const int each = p.in.H * p.RB;
  long long mine = 0;
#pragma unroll 1
  for (int64_t b = b0; b < b1; ++b) mine += (long long)span_of<T>(p, b).nt * each;
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh.sum[warp] = upto;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) upto += sh.sum[w];
    total += sh.sum[w];
  }
  chunk = max(1ll, (total + gridDim.x * WORKERS - 1) / (gridDim.x * WORKERS));
#pragma unroll 1
  for (int w = 0; w < WORKERS; ++w) {
    const long long u0 = ((long long)w * gridDim.x + blockIdx.x) * chunk;
    if (upto - mine <= u0 && u0 < upto) {
      long long at = upto - mine;
      int64_t b = b0;
#pragma unroll 1
      for (;; ++b) {
        const long long n = (long long)span_of<T>(p, b).nt * each;
        if (u0 < at + n) break;
        at += n;
      }
      sh.b[w] = b; sh.before[w] = at;
    }
  }
  __syncthreads();
}

__device__ __forceinline__ int64_t out_at(const AttnParams& p, int64_t b, int h, int r) {
  const int j = r / p.G;
  return b * p.out.o_seq + j * p.out.o_pos + (int64_t)(h * p.G + r - j * p.G) * p.out.o_head;
}
__device__ __forceinline__ float lse_of(float m, float l) { return l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F; }
__device__ __forceinline__ void put_lse(const AttnParams& p, int64_t b, int h, int r, float m, float l) {
  if (!p.out.lse) return;
  const int j = r / p.G;
  p.out.lse[(b * p.in.Q + j) * p.in.Hq + h * p.G + r - j * p.G] = lse_of(m, l);
}
// (by the worker that has the sequence's first tile; what comes to light elsewhere is added by the joining kernel)
__device__ __forceinline__ void put_status(const AttnParams& p, int64_t b, uint32_t st) {
  if (p.out.row_status) p.out.row_status[b] = st;
  if (st && !(p.in.row_status && p.in.row_status[b])) atomicAdd(p.flagged, 1ull);      // (a flag that came with the call is counted already)
}

__device__ __forceinline__ void add_status(const AttnParams& p, int64_t b, uint32_t st) {
  if (!p.out.row_status || atomicOr(p.out.row_status + b, st) == 0) atomicAdd(p.flagged, 1ull);
}

// Segments (sequence, key head, row block) that several workers had a part of: ROWS rows of DP values, then ROWS pairs (m, l); l = -1: a bad
// page, -2: a wait ran out.
template <int ROWS, int DP> constexpr int PART = ROWS * (DP + 2);
__device__ __forceinline__ uint32_t status_of(float l) { return l == -1.f ? SAKI_ROW_BAD_PAGE : l == -2.f ? SAKI_ROW_TIMEOUT : 0u; }

// The exponent of a weight is c s - m in one fused operation, whatever tile it is in and whatever the maximum was taken to be by then: equal scores weigh the same.  m is the
// largest c s rounded downwards, so the largest exponent is what the rounding took away: below 1 for |c s| < 2^24, up to 64 for 2^30, where a step of the score itself is 64 and more.
// Beyond that it is cut, for the sums' sake: scores that equal the largest still weigh the same, and one a step of float32 below it may weigh as much.  (NaN stays.)
constexpr float MOST_EXPONENT = 64.f;
__device__ __forceinline__ float cut_exponent(float x) { return x > MOST_EXPONENT ? MOST_EXPONENT : x; }

// what a row sees: positions up to `to`, from `from` on or below `first`
struct Sight {
  int to, from, first;
  __device__ __forceinline__ bool operator()(int x) const { return x <= to && (x >= from || x < first); }
};
__device__ __forceinline__ Sight sight_of(const AttnParams& p, const Span& s, int r) {      // r: row within the key head
  const int j = r / p.G;
  if (r >= p.R || j >= s.nq) return {-1, 0, 0};
  const int at = s.p0 + j;
  return {at, p.in.window > 0 ? (int)max((int64_t)0, (int64_t)at - p.in.window + 1) : 0, p.in.window > 0 ? p.in.sinks : 0};
}
// all rows see all of a tile's positions
template <int T> __device__ __forceinline__ bool whole(const AttnParams& p, const Span& s, int x0) {
  return s.nq == p.in.Q && x0 + (T - 1) <= s.p0 && (p.in.window <= 0 || x0 > s.n - 1 - p.in.window || x0 + T <= s.sk);
}

// The kernel on tcgen05 (saki_attention_umma.cu): bf16, D up to 128, boxes of at least eight positions; rows of a row block, and the launch.
constexpr int UMMA_T = 128;
int umma_rows(const saki_attn_in& in);
cudaError_t launch_umma(const AttnParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, int blocks, cudaStream_t st);

}  // namespace attn

}  // namespace saki
