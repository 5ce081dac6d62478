// The pages of a key-value cache: page tables, lengths and counts of holders (integers, a few thousand to a few hundred
// thousand of them), and the two calls that move keys and values.
//
// The integer calls are bound by latency, not by what they read.  Which page a sequence gets depends on all sequences before
// it and on all pages below, so reserving and compacting are a handful of scans: one cluster of blocks does them in one launch,
// with cluster barriers where a grid would need further launches (2 to 3 us each): a reservation for 512 sequences over 40000 pages takes 15 us, of which the scans, five waits
// for L2 and three cluster barriers are nearly all; for 8 sequences over 2048 pages 12.  The write of 512 x 7 positions of 8 heads of 128 takes 11.5 us (29 MB: 4.5 at the copy rate), copies run at it where pages are runs of whole 16 bytes (others go byte
// by byte: 1024 pages of 2160 bytes in 4 pools at 3.2 TB/s; rows apart, 128 runs a page of 32 KB and two launches a pool, at 0.5).  Every result is a function of the call's inputs
// alone: pages are dealt out by rank, and the only atomics are sums and minima of integers.
#include "saki_common.cuh"
#include <cooperative_groups.h>
#include <algorithm>
#include <climits>

namespace cg = cooperative_groups;

namespace saki {

namespace {

constexpr int CT = 1024, CWARPS = CT / 32, CCS = 8;        // threads of a block, blocks of the cluster
constexpr uint32_t NOT_SERVED = 0xffffffffu;

__device__ __forceinline__ int pages_of(int64_t positions, int page) { return (int)((positions + page - 1) / page); }
__device__ __forceinline__ bool in_pool(int id, int n_pages) { return (unsigned)id < (unsigned)n_pages; }
__device__ __forceinline__ bool length_ok(const saki_cache& c, int64_t L) { return L >= 0 && L <= (int64_t)c.max_pages * c.page_size; }

// What a sequence asks for.
struct Plan { int64_t L, n; int have, want, last; uint32_t status; };
__device__ __forceinline__ Plan plan(const saki_cache& c, const int32_t* n_new, int32_t n_all, int64_t b) {
  Plan p;
  p.L = c.length[b]; p.n = n_new ? n_new[b] : n_all;
  p.have = p.want = 0; p.last = -1; p.status = 0;
  if (!length_ok(c, p.L) || p.n < 0 || !length_ok(c, p.L + p.n)) { p.status = SAKI_ROW_BAD_LENGTH; return p; }
  p.have = pages_of(p.L, c.page_size); p.want = pages_of(p.L + p.n, c.page_size);
  if (p.n > 0 && p.L % c.page_size != 0) {               // goes on in its last page
    p.last = c.page_table[b * c.ld_table + p.have - 1];
    if (!in_pool(p.last, c.n_pages)) { p.status = SAKI_ROW_BAD_PAGE; p.last = -1; p.want = p.have; }
  }
  return p;
}

// inclusive sum over the block in thread order; every thread gets the total too
__device__ __forceinline__ long long block_scan(long long v, long long* warps, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  long long before = 0;
  total = 0;
  for (int w = 0; w < CWARPS; ++w) {
    const long long s = warps[w];
    if (w < warp) before += s;
    total += s;
  }
  return v + before;
}

struct ClusterShared {
  long long scan[CWARPS];
  int warp_count[2][CWARPS];
  int count[2];            // of the block, read by the others
  int need;                // pages that are dealt out (first block)
};

// The pages are split over the cluster's warps in runs of whole 32s, in order.
struct Run { int from, to; };
__device__ __forceinline__ Run run_of(int n_pages, int rank) {
  const int per = (int)(((int64_t)n_pages + CCS * CWARPS - 1) / (CCS * CWARPS) + 31) & ~31;
  const int64_t from = (int64_t)(rank * CWARPS + (threadIdx.x >> 5)) * per;
  return {(int)min(from, (int64_t)n_pages), (int)min(from + per, (int64_t)n_pages)};
}
// pages of a run that `is` says yes to, counted into sh.warp_count[k] and, for the block, sh.count[k] (ends with a barrier)
// Eight loads are on their way at a time: a run of a few hundred pages costs one wait, not one for every 32.
constexpr int AHEAD = 8;
template <typename F, typename G> __device__ __forceinline__ void each_32(Run r, F&& is, G&& take) {      // take(i, is(i), mask of the warp's)
  const int lane = threadIdx.x & 31;
  for (unsigned i0 = (unsigned)r.from; i0 < (unsigned)r.to; i0 += 32 * AHEAD) {      // (unsigned: behind the last page may be 2^31)
    bool yes[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const unsigned i = i0 + 32 * k + lane;
      yes[k] = i < (unsigned)r.to && is((int)i);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) take((int)(i0 + 32 * k + lane), yes[k], __ballot_sync(0xffffffffu, yes[k]));
  }
}
template <typename F> __device__ __forceinline__ void count_run(ClusterShared& sh, int k, Run r, F&& is) {
  const int lane = threadIdx.x & 31;
  int n = 0;
  each_32(r, is, [&](int, bool, unsigned m) { n += __popc(m); });
  if (lane == 0) sh.warp_count[k][threadIdx.x >> 5] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    int t = 0;
    for (int w = 0; w < CWARPS; ++w) t += sh.warp_count[k][w];
    sh.count[k] = t;
  }
  __syncthreads();
}
// rank of this warp's first page among those that were counted, and the total, over the cluster
__device__ __forceinline__ int rank_of_run(cg::cluster_group& cl, ClusterShared& sh, int k, int* total) {
  int before = 0, all = 0;
  for (int r = 0; r < CCS; ++r) {
    const int n = cl.map_shared_rank(&sh, r)->count[k];
    if (r < (int)cl.block_rank()) before += n;
    all += n;
  }
  for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) before += sh.warp_count[k][w];
  *total = all;
  return before;
}
template <typename F, typename G> __device__ __forceinline__ void each_ranked(Run r, int rank, F&& is, G&& take) {
  const int lane = threadIdx.x & 31;
  each_32(r, is, [&](int i, bool yes, unsigned m) {
    if (yes) take(i, rank + __popc(m & ((1u << lane) - 1u)));
    rank += __popc(m);
  });
}

// scratch of a reservation: free pages by rank; per shared last page the first sequence that goes on in it, and how many do; per
// sequence how it is served
struct ReserveScratch { int32_t *order, *first, *going; uint32_t* seq; };
__device__ __forceinline__ ReserveScratch reserve_scratch(const saki_cache& c) {
  int32_t* const w = (int32_t*)c.scratch;
  return {w, w + c.n_pages, w + 2 * (int64_t)c.n_pages, (uint32_t*)(w + 3 * (int64_t)c.n_pages)};
}

// 1. the free pages are counted; the first block looks at the sequences.  2. which sequences find room (in order, one page counted
// for each shared last page), who keeps such a page, where each sequence's share of the free pages starts.  3. the free pages by
// rank.  4. tables, lengths, counts.
__global__ void __launch_bounds__(CT) reserve_kernel(const saki_cache c, const int32_t* n_new, int32_t n_all, int32_t* copy_src,
                                                     int32_t* copy_dst, uint32_t* row_status, unsigned long long* flagged) {
  __shared__ ClusterShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), tid = threadIdx.x;
  wait_for_predecessor();
  launch_dependents();
  const ReserveScratch w = reserve_scratch(c);
  const Run run = run_of(c.n_pages, rank);
  auto free_page = [&](int id) { return c.ref_count[id] == 0; };
  // (the first block's plan of the first CT sequences stays in registers)
  Plan own = {};
  bool own_shared = false, shared = false;                // goes on in a page with other holders; any sequence does
  if (rank == 0) {
    if (tid == 0) sh.need = 0;
    for (int64_t b = tid; b < c.B; b += CT) {
      const Plan p = plan(c, n_new, n_all, b);
      const bool parted = p.last >= 0 && c.ref_count[p.last] > 1;
      if (parted) { w.first[p.last] = INT_MAX; w.going[p.last] = 0; }
      if (b == tid) { own = p; own_shared = parted; }
      shared = shared || parted;
    }
    shared = __syncthreads_or(shared);
  }
  count_run(sh, 0, run, free_page);
  cl.sync();
  int n_free = 0;
  const int my_rank = rank_of_run(cl, sh, 0, &n_free);
  if (rank == 0) {
    long long carry = 0, total = 0;
    for (int64_t b0 = 0; b0 < c.B; b0 += CT) {
      const int64_t b = b0 + tid;
      Plan p = own;
      bool parted = own_shared;
      if (b0 > 0) {
        p = b < c.B ? plan(c, n_new, n_all, b) : Plan{};
        parted = b < c.B && p.last >= 0 && c.ref_count[p.last] > 1;
      }
      const long long need = b < c.B && !p.status ? p.want - p.have + (parted ? 1 : 0) : 0;
      const long long upto = carry + block_scan(need, sh.scan, total);
      carry += total;
      const bool ok = b < c.B && !p.status && upto <= n_free;
      if (shared) {
        if (b < c.B) w.seq[b] = ok ? (parted ? 3u : 1u) : 0u;
        if (ok && parted) { atomicMin(w.first + p.last, (int)b); atomicAdd(w.going + p.last, 1); }
      } else {                     // no page is shared: that is all
        if (b < c.B) w.seq[b] = ok ? (uint32_t)((upto - need) * 2) : NOT_SERVED;
        const int most = __reduce_max_sync(0xffffffffu, ok ? (int)upto : 0);
        if ((tid & 31) == 0) atomicMax(&sh.need, most);
      }
    }
    if (shared) {
      __syncthreads();
      carry = 0;
      for (int64_t b0 = 0; b0 < c.B; b0 += CT) {
        const int64_t b = b0 + tid;
        long long need = 0;
        uint32_t how = 0;
        bool copies = false;
        if (b < c.B && (how = w.seq[b])) {
          const Plan p = b0 == 0 ? own : plan(c, n_new, n_all, b);
          copies = how == 3u && !(w.going[p.last] == c.ref_count[p.last] && w.first[p.last] == (int)b);
          need = p.want - p.have + (copies ? 1 : 0);
        }
        const long long upto = carry + block_scan(need, sh.scan, total);
        carry += total;
        if (b < c.B) w.seq[b] = how ? (uint32_t)((upto - need) * 2 + (copies ? 1 : 0)) : NOT_SERVED;
      }
      if (tid == 0) sh.need = (int)carry;
    }
  }
  cl.sync();
  const int dealt = cl.map_shared_rank(&sh, 0)->need;
  if (my_rank < dealt)
    each_ranked(run, my_rank, free_page, [&](int id, int r) {
      if (r < dealt) { w.order[r] = id; c.ref_count[id] = 1; }
    });
  cl.sync();
  const int lane = tid & 31;
  for (int64_t b = rank * CWARPS + (tid >> 5); b < c.B; b += CCS * CWARPS) {
    const Plan p = plan(c, n_new, n_all, b);
    const uint32_t s = w.seq[b];
    const bool ok = s != NOT_SERVED, copies = ok && (s & 1u);
    __syncwarp();
    if (ok) {
      const int start = (int)(s >> 1) + (copies ? 1 : 0);
      int32_t* const row = c.page_table + b * c.ld_table;
      for (int x = p.have + lane; x < p.want; x += 32) row[x] = w.order[start + x - p.have];
      if (lane == 0 && copies) {
        row[p.have - 1] = w.order[s >> 1];
        atomicSub(c.ref_count + p.last, 1);
      }
    }
    if (lane == 0) {
      copy_src[b] = copies ? p.last : -1;
      copy_dst[b] = copies ? w.order[s >> 1] : -1;
      const uint32_t st = ok ? 0u : p.status ? p.status : SAKI_ROW_NO_PAGES;
      if (ok) c.length[b] = (int32_t)(p.L + p.n);
      if (row_status) row_status[b] = st;
      if (st) atomicAdd(flagged, 1ull);
    }
  }
}

// a warp per sequence
__global__ void __launch_bounds__(256) truncate_kernel(const saki_cache c, const int32_t* keep, int32_t keep_add, int32_t of, uint32_t* row_status,
                                                       unsigned long long* flagged) {
  wait_for_predecessor();
  launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (b >= c.B) return;
  if (const uint32_t refused = c.row_status ? c.row_status[b] : 0u) {      // what is to be cut is not there
    __syncwarp();
    if (lane == 0 && row_status) row_status[b] = refused;
    return;
  }
  const int64_t L = c.length[b], k = (int64_t)keep[b] + keep_add, last = of < 0 ? L : of;
  __syncwarp();
  uint32_t st = 0;
  if (!length_ok(c, L) || last > L || k < 0 || k > last) st = SAKI_ROW_BAD_LENGTH;
  else {
    const int64_t left = L - last + k;
    int32_t* const row = c.page_table + b * c.ld_table;
    bool bad = false;
    for (int x = pages_of(left, c.page_size) + lane; x < pages_of(L, c.page_size); x += 32) {
      const int id = row[x];
      if (in_pool(id, c.n_pages)) atomicSub(c.ref_count + id, 1);
      else bad = true;
      row[x] = -1;
    }
    if (__any_sync(0xffffffffu, bad)) st = SAKI_ROW_BAD_PAGE;
    if (lane == 0) c.length[b] = (int32_t)left;
  }
  if (lane == 0) {
    if (row_status) row_status[b] = st;
    if (st) atomicAdd(flagged, 1ull);
  }
}

// the row that row b becomes: -1 none (st: why), else its number
__device__ __forceinline__ int64_t parent_row(const saki_cache& c, const int32_t* parent, int64_t group, int64_t b, uint32_t& st) {
  const int64_t base = b / group * group, p = parent[b];
  if (p >= 0 && p < group && base + p < c.B) return base + p;
  if (p != -1) st = SAKI_ROW_BAD_ID;
  return -1;
}
// The new rows go to scratch first: a row is read by others while it gets its own.  Counts: plus one for every page of the
// parent, minus one for every page that the row held.
__global__ void __launch_bounds__(128) fork_kernel(const saki_cache c, const int32_t* parent, int64_t group, uint32_t* row_status,
                                                   unsigned long long* flagged) {
  wait_for_predecessor();
  launch_dependents();
  const int64_t b = blockIdx.x;
  uint32_t st = 0;
  const int64_t p = parent_row(c, parent, group, b, st);
  bool bad = false;
  if (p != b) {
    int32_t* const to = (int32_t*)c.scratch + b * c.max_pages;
    int64_t Lp = p >= 0 ? c.length[p] : 0, Lb = c.length[b];
    if (!length_ok(c, Lp)) { Lp = 0; st |= SAKI_ROW_BAD_LENGTH; }
    if (!length_ok(c, Lb)) { Lb = 0; st |= SAKI_ROW_BAD_LENGTH; }
    const int np = pages_of(Lp, c.page_size), nb = pages_of(Lb, c.page_size);
    for (int x = threadIdx.x; x < c.max_pages; x += blockDim.x) {
      int id = -1;
      if (x < np) {
        id = c.page_table[p * c.ld_table + x];
        if (in_pool(id, c.n_pages)) atomicAdd(c.ref_count + id, 1);
        else bad = true;
      }
      to[x] = id;
      if (x < nb) {
        const int old = c.page_table[b * c.ld_table + x];
        if (in_pool(old, c.n_pages)) atomicSub(c.ref_count + old, 1);
        else bad = true;
      }
    }
    if (threadIdx.x == 0) ((int32_t*)c.scratch)[c.B * c.max_pages + b] = (int32_t)Lp;
  }
  if (__syncthreads_or(bad)) st |= SAKI_ROW_BAD_PAGE;
  if (threadIdx.x == 0) {
    if (row_status) row_status[b] = st;
    if (st) atomicAdd(flagged, 1ull);
  }
}
__global__ void __launch_bounds__(128) fork_rows_kernel(const saki_cache c, const int32_t* parent, int64_t group) {
  wait_for_predecessor();
  launch_dependents();
  const int64_t b = blockIdx.x;
  uint32_t st = 0;
  if (parent_row(c, parent, group, b, st) == b) return;
  const int32_t* const from = (const int32_t*)c.scratch + b * c.max_pages;
  for (int x = threadIdx.x; x < c.max_pages; x += blockDim.x) c.page_table[b * c.ld_table + x] = from[x];
  if (threadIdx.x == 0) c.length[b] = ((const int32_t*)c.scratch)[c.B * c.max_pages + b];
}

__global__ void __launch_bounds__(CT) compact_kernel(const saki_cache c, int32_t* copy_src, int32_t* copy_dst, int32_t* n_moves) {
  __shared__ ClusterShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), half = c.n_pages / 2;
  wait_for_predecessor();
  launch_dependents();
  int32_t* const to = (int32_t*)c.scratch;              // [n_pages] where each page goes
  const Run run = run_of(c.n_pages, rank);
  int used = 0, moves = 0, rooms = 0;
  count_run(sh, 0, run, [&](int id) { return c.ref_count[id] != 0; });
  cl.sync();
  rank_of_run(cl, sh, 0, &used);
  cl.sync();
  auto moved = [&](int id) { return id >= used && c.ref_count[id] != 0; };
  auto room = [&](int id) { return id < used && c.ref_count[id] == 0; };
  count_run(sh, 0, run, moved);
  count_run(sh, 1, run, room);
  cl.sync();
  const int from_move = rank_of_run(cl, sh, 0, &moves), from_room = rank_of_run(cl, sh, 1, &rooms);   // (as many of one as of the other)
  each_ranked(run, from_move, moved, [&](int id, int r) { copy_src[r] = id; });
  each_ranked(run, from_room, room, [&](int id, int r) { copy_dst[r] = id; });
  for (int i = run.from + (threadIdx.x & 31); i < run.to; i += 32) to[i] = i;
  for (int i = moves + rank * CT + threadIdx.x; i < half; i += CCS * CT) { copy_src[i] = -1; copy_dst[i] = -1; }
  if (rank == 0 && threadIdx.x == 0 && n_moves) *n_moves = moves;
  cl.sync();
  for (int i = rank * CT + threadIdx.x; i < moves; i += CCS * CT) {
    const int s = copy_src[i], d = copy_dst[i];
    to[s] = d;
    c.ref_count[d] = c.ref_count[s];
    c.ref_count[s] = 0;
  }
}
__global__ void __launch_bounds__(128) compact_rows_kernel(const saki_cache c, uint32_t* row_status, unsigned long long* flagged) {
  wait_for_predecessor();
  launch_dependents();
  const int64_t b = blockIdx.x, L = c.length[b];
  uint32_t st = 0;
  bool bad = false;
  if (!length_ok(c, L)) st = SAKI_ROW_BAD_LENGTH;
  else
    for (int x = threadIdx.x; x < pages_of(L, c.page_size); x += blockDim.x) {
      const int id = c.page_table[b * c.ld_table + x];
      if (in_pool(id, c.n_pages)) c.page_table[b * c.ld_table + x] = ((const int32_t*)c.scratch)[id];
      else bad = true;
    }
  if (__syncthreads_or(bad)) st |= SAKI_ROW_BAD_PAGE;
  if (threadIdx.x == 0) {
    if (row_status) row_status[b] = st;
    if (st) atomicAdd(flagged, 1ull);
  }
}

constexpr int POOLS = 64;          // pools of one launch
struct CopyParams {
  char* pool[POOLS];
  int64_t stride[POOLS], bytes[POOLS];
  const int32_t *src, *dst;
  int64_t n;
  int32_t n_pages;
};
// a block per pair and pool
template <typename V> __global__ void __launch_bounds__(256) copy_pages_kernel(const __grid_constant__ CopyParams p) {
  wait_for_predecessor();
  launch_dependents();
  char* const pool = p.pool[blockIdx.y];
  const int64_t stride = p.stride[blockIdx.y], n = p.bytes[blockIdx.y] / (int64_t)sizeof(V);
  for (int64_t i = blockIdx.x; i < p.n; i += gridDim.x) {
    const int s = p.src[i], d = p.dst[i];
    if (!in_pool(s, p.n_pages) || !in_pool(d, p.n_pages)) continue;
    const V* const from = (const V*)(pool + s * stride);
    V* const to = (V*)(pool + d * stride);
    int64_t x = threadIdx.x;
    for (; x + 3 * 256 < n; x += 4 * 256) {
      V v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = from[x + k * 256];
#pragma unroll
      for (int k = 0; k < 4; ++k) to[x + k * 256] = v[k];
    }
    for (; x < n; x += 256) to[x] = from[x];
  }
}

// a block per new position; E: elements of V
template <typename V, int E> __global__ void __launch_bounds__(256) write_kernel(const saki_cache c, const saki_cache_kv w) {
  wait_for_predecessor();
  launch_dependents();
  const int64_t b = blockIdx.x / w.Q;
  const int j = (int)(blockIdx.x - b * w.Q);
  constexpr int SIZE = (int)sizeof(V) / E;
  const int vecs = w.D / E, half = w.H * vecs;
  const char* const k = (const char*)w.k + (b * w.k_seq + j * w.k_pos) * SIZE;
  const char* const v = (const char*)w.v + (b * w.v_seq + j * w.v_pos) * SIZE;
  auto from = [&](int i) {
    const bool second = i >= half;
    const int r = second ? i - half : i, h = r / vecs, d = (r - h * vecs) * E;
    return *(const V*)((second ? v + (h * w.v_head + d) * SIZE : k + (h * w.k_head + d) * SIZE));
  };
  // (a thread's first piece is on its way while the position is looked up, three reads one behind the other)
  const V early = from(min((int)threadIdx.x, 2 * half - 1));
  const uint32_t flag = w.row_status ? w.row_status[b] : 0u;
  const int n = w.n_new ? w.n_new[b] : w.Q;
  const int64_t L = c.length[b], x = L - n + j;
  if (flag || n < 0 || n > w.Q || j >= n || x < 0 || !length_ok(c, L)) return;
  const int64_t page = x <= INT_MAX ? (unsigned)x / (unsigned)c.page_size : x / c.page_size;
  const int id = c.page_table[b * c.ld_table + page], slot = (int)(x - page * c.page_size);
  if (!in_pool(id, c.n_pages)) return;
  char* const kp = (char*)w.k_pages + (id * w.kp_page + slot * w.kp_pos) * SIZE;
  char* const vp = (char*)w.v_pages + (id * w.vp_page + slot * w.vp_pos) * SIZE;
  for (int i = threadIdx.x; i < 2 * half; i += blockDim.x) {
    const bool second = i >= half;
    const int r = second ? i - half : i, h = r / vecs, d = (r - h * vecs) * E;
    *(V*)((second ? vp + (h * w.vp_head + d) * SIZE : kp + (h * w.kp_head + d) * SIZE)) = i == (int)threadIdx.x ? early : from(i);
  }
}

}  // namespace

int64_t cache_scratch_bytes(int64_t B, int32_t max_pages, int32_t n_pages) {
  return 4 * std::max<int64_t>(3 * (int64_t)n_pages + B, B * ((int64_t)max_pages + 1));
}

cudaError_t launch_cache_reserve(const saki_cache& c, const int32_t* n_new, int32_t n_all, int32_t* src, int32_t* dst, uint32_t* status,
                                 unsigned long long* flagged, cudaStream_t st) {
  return launch_pdl_cluster(reserve_kernel, dim3(CCS), CT, CCS, 0, st, c, n_new, n_all, src, dst, status, flagged);
}
cudaError_t launch_cache_truncate(const saki_cache& c, const int32_t* keep, int32_t add, int32_t of, uint32_t* status, unsigned long long* flagged,
                                  cudaStream_t st) {
  return launch_pdl(truncate_kernel, dim3((unsigned)((c.B + 7) / 8)), 256, 0, st, true, c, keep, add, of, status, flagged);
}
cudaError_t launch_cache_fork(const saki_cache& c, const int32_t* parent, int64_t group, uint32_t* status, unsigned long long* flagged,
                              cudaStream_t st) {
  cudaError_t e = launch_pdl(fork_kernel, dim3((unsigned)c.B), 128, 0, st, true, c, parent, group, status, flagged);
  return e != cudaSuccess ? e : launch_pdl(fork_rows_kernel, dim3((unsigned)c.B), 128, 0, st, true, c, parent, group);
}
cudaError_t launch_cache_compact(const saki_cache& c, int32_t* src, int32_t* dst, int32_t* n_moves, uint32_t* status, unsigned long long* flagged,
                                 cudaStream_t st) {
  cudaError_t e = launch_pdl_cluster(compact_kernel, dim3(CCS), CT, CCS, 0, st, c, src, dst, n_moves);
  return e != cudaSuccess || c.B == 0 ? e : launch_pdl(compact_rows_kernel, dim3((unsigned)c.B), 128, 0, st, true, c, status, flagged);
}
cudaError_t launch_copy_pages(void* const* pools, const int64_t* stride, const int64_t* bytes, int32_t n_pools, const int32_t* src,
                              const int32_t* dst, int64_t n, int32_t n_pages, int* n_launches, cudaStream_t st) {
  for (int k = 0; k < n_pools; k += POOLS) {
    CopyParams p = {};
    const int m = std::min(POOLS, n_pools - k);
    bool wide = true;
    for (int i = 0; i < m; ++i) {
      p.pool[i] = (char*)pools[k + i]; p.stride[i] = stride[k + i]; p.bytes[i] = bytes[k + i];
      wide = wide && ((uintptr_t)p.pool[i] | (uintptr_t)p.stride[i] | (uintptr_t)p.bytes[i]) % 16 == 0;
    }
    p.src = src; p.dst = dst; p.n = n; p.n_pages = n_pages;
    const dim3 grid((unsigned)std::min<int64_t>(n, 1 << 20), (unsigned)m);
    const cudaError_t e = wide ? launch_pdl(copy_pages_kernel<uint4>, grid, 256, 0, st, true, p) : launch_pdl(copy_pages_kernel<unsigned char>, grid, 256, 0, st, true, p);
    if (e != cudaSuccess) return e;
    ++*n_launches;
  }
  return cudaSuccess;
}
cudaError_t launch_cache_write(const saki_cache& c, const saki_cache_kv& w, cudaStream_t st) {
  const int size = w.dtype == SAKI_BF16 ? 2 : 4, e = 16 / size;
  uintptr_t all = (uintptr_t)w.k | (uintptr_t)w.v | (uintptr_t)w.k_pages | (uintptr_t)w.v_pages;
  for (int64_t s : {w.k_seq, w.k_pos, w.k_head, w.v_seq, w.v_pos, w.v_head, w.kp_page, w.kp_pos, w.kp_head, w.vp_page, w.vp_pos, w.vp_head, (int64_t)w.D})
    all |= (uintptr_t)(s * size);
  const bool wide = all % 16 == 0;
  const int items = 2 * w.H * (wide ? w.D / e : w.D), threads = std::min(256, (items + 31) & ~31);
  const dim3 grid((unsigned)(c.B * w.Q));
  if (wide) return size == 2 ? launch_pdl(write_kernel<uint4, 8>, grid, threads, 0, st, true, c, w) : launch_pdl(write_kernel<uint4, 4>, grid, threads, 0, st, true, c, w);
  return size == 2 ? launch_pdl(write_kernel<uint16_t, 1>, grid, threads, 0, st, true, c, w) : launch_pdl(write_kernel<uint32_t, 1>, grid, threads, 0, st, true, c, w);
}

}  // namespace saki
