// The attention of saki_attention.cu on the fifth-generation tensor cores, for bf16 with D up to 128 and pages of whole eights.
//
// A tile is 128 positions of one key head, and the products are turned round: positions and head columns are the 128 rows of tcgen05.mma, the queries
// (16, 32 or 64 rows of a key head) its columns.  So nothing is padded but the queries, and a tile costs a handful of instructions:
//   scores^T [128 positions x N]  = K [128 x D] . Q^T [D x N]              K as stored (K-major), 128-byte swizzle as TMA lays it down
//   out^T    [128 columns x 2 N] += V^T [D x 128] . P^T [128 x 2 N]        V as stored (M-major); P in two bf16 terms (16 bits), side by side: V is read once
// One block on each SM, its piece of the line, and
//   warp 0      looks pages up and loads keys and values by TMA into a ring of slots (one tile's keys or values each)
//   warps 1, 2  a thread of one issues the products for the scores, up to two tiles ahead, a thread of the other those for the outputs (one thread for both was what a tile
//               waited for: 16 products take 1200 cycles of shared memory's time, waits and commits around them as long again); warp 2 holds tensor memory
//   warp 3      loads the queries of the segments, two ahead
//   from 4 on   groups of four warps that share a tile's queries (8 each, 16 of 64), a thread per position: it reads its scores, takes 2^(c s - m), adds them up, and
//               leaves the weights in shared memory for the next product.  m is a row's maximum as of some tile: it is brought up to date (and
//               sums and outputs with it) only when a weight passes 2^8, so that a common tile needs no maximum over its positions and no pass over
//               the output.  (A group is a warp on each scheduler, which issues an instruction in four to six cycles: so few queries, and groups that
//               share a tile.  Groups that took turns, a tile each, were slower: a tile's keys and values wait twice as long for their turn in the ring.)
//   the last 4  a thread per column of the output: at a segment's end they divide and write, while the groups go on
// What bounds it: HBM where segments are long (two to three tiles of 64 KB in flight on an SM): 64 sequences of 4096 positions, 8 key heads of 128, 4 rows each 179 us, 6.0 TB/s (92 % of
// the measured copy rate), of 8192 with 28 rows 362 us (91 %), 512 of 1024 with 4 rows 353 us (93 %).  The weights' warps where segments end often or rows are many: 512 of 65 to 2048
// positions with 28 rows 568 to 590 us from run to run (59 to 61 %: the instructions of an edge, some 7 us a segment), 64 of 8192 with 64 rows 608 us (54 %).  More rows are row blocks of 64, which read keys
// and values once each: 136 rows 1776 us, on 512 of 65 to 2048 positions 2863.  One sequence of 131077, 4 key heads: 57 us (72 %: start, two ends and the joining kernel are some 15 of it).
// Every wait is bounded (by the time that no tile is finished): a wait that runs out ends all roles' waits, the segments that are left are flagged, and the block leaves.
#include "saki_attention.cuh"
#include <cfloat>
#include <climits>

namespace saki {

namespace attn {

namespace {

constexpr int UT = 128;                      // positions of a tile

template <int DP, int N> struct UShape {
  static constexpr int GROUPS = N == 16 ? 2 : 4, CW = N / GROUPS, THREADS = 256 + 128 * GROUPS;      // groups of warps, queries of a group
  static constexpr int SLABS = DP / 64, SLOT = UT * DP * 2;                // keys or values of a tile
  static constexpr int P_BYTES = 2 * N * UT * 2, P_BUFS = N <= 32 ? 2 : 1; // two terms
  static constexpr int Q_BYTES = N * DP * 2;
  static constexpr int FIXED = P_BUFS * P_BYTES + 2 * Q_BYTES + 7168 + 1024;      // and the rest, alignment
  static constexpr int FIT = (227 * 1024 - FIXED) / SLOT, SLOTS = FIT < 12 ? FIT : 12;
  static constexpr int SMEM = SLOTS * SLOT + FIXED;
  static constexpr int COLS = 6 * N <= 128 ? 128 : 6 * N <= 256 ? 256 : 512;             // two buffers of scores; by segment, outputs in two terms
  static_assert(SLOTS >= 4, "two tiles");
};

template <int THREADS> struct URest {      // of shared memory
  uint64_t full[12], empty[12], q_full[2], q_empty[2], s_full[2], p_ready[2], pv_done[2], drain[2];
  uint64_t seg_sums[2], seg_pv[2], seg_free[2];      // by segment: the groups' sums are there; so are the outputs; both have been read
  LineShared<THREADS> line;
  // by query
  alignas(16) float m[64];                   // (read four at a time)
  float factor[64], top[4][64], inverse[64];
  int to[64], from[64];
  int64_t row_at[64], q_at[64];              // where a row's output starts, where its queries are in a sequence and key head; -1: there is none
  // by segment, for the warps that write
  float end_m[2][64], end_sum[2][4][64];
  int end_bad[2];
  int bad[8];             // by tile: a page outside the pool
  int keep[2];            // by tile: its sums go on top of what is there although it is the segment's first
  int stop[2];            // a wait ran out; tiles that the groups have finished
  uint32_t tmem;
};
static_assert(sizeof(URest<768>) <= 7168, "what is left of shared memory");

// The loads of n tiles, in the order of the products: K0 K1 V0 K2 V1 ... V(n-1).  (Values with their keys would hold a slot for a tile's time longer.)
__device__ __forceinline__ int load_of_keys(int i) { return i == 0 ? 0 : 2 * i - 1; }
__device__ __forceinline__ int load_of_values(int i, int n) { return i + 1 < n ? 2 * i + 2 : 2 * n - 1; }

// Code that is rarely run, or run from many places, is kept out of line: with all of it in place a kernel had 107 to 139 KB, and its warps, each in a part of its
// own, waited for instructions more than for anything else.
// The limit is for a tile: some roles wait for a whole segment, so it starts again whenever the groups have finished one (there are so many tiles and no more).
static __device__ __noinline__ bool u_wait_long(uint64_t* bar, uint32_t parity, int* stop, long long limit) {
  const bool common = limit >= WAIT_LIMIT_CYCLES;
  if (common && mbar_try_wait(bar, parity)) return true;       // (which itself waits for a while)
  long long t0 = clock64();
  int done = *(volatile int*)(stop + 1);
  for (;;) {
    if (*(volatile int*)stop) return false;
    const int now = *(volatile int*)(stop + 1);
    if (now != done) { done = now; t0 = clock64(); }
    else if (clock64() - t0 > limit) { *(volatile int*)stop = 1; return false; }
    if (common ? mbar_try_wait(bar, parity) : mbar_test_wait(bar, parity)) return true;
  }
}
template <typename R> __device__ __forceinline__ bool u_wait(uint64_t* bar, uint32_t parity, R& r, long long limit) {
  return (limit >= WAIT_LIMIT_CYCLES && mbar_try_wait(bar, parity)) || u_wait_long(bar, parity, r.stop, limit);
}
__device__ __forceinline__ void u_arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void u_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void u_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void u_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Shared-memory matrix descriptor, 128-byte swizzle, in two words.  Lower: address and, for an M-major operand, `lead`, the bytes from 64 rows to the next, in units
// of 16 bytes; upper: `stride`, the bytes from eight rows (K-major) or eight k (M-major) to the next.  (The issuing thread takes its time for every
// word that it has to compute and move: what is constant goes into the instruction.)
__device__ __forceinline__ uint32_t u_lower(uint32_t at, uint32_t lead = 16) { return (at >> 4) | (lead >> 4) << 16; }
__host__ __device__ constexpr uint32_t u_upper(uint32_t stride) { return (stride >> 4) | 1u << 14 | 2u << 29; }
// instruction descriptor: float32 sums, bf16 operands, M = 128; A M-major if `a_m`
__host__ __device__ constexpr uint32_t u_idesc(int n, bool a_m) { return (1u << 4) | (1u << 7) | (1u << 10) | (a_m ? 1u << 15 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
template <uint32_t A, uint32_t B, uint32_t IDESC> __device__ __forceinline__ void u_mma(uint32_t d, uint32_t a, uint32_t b) {      // on top of what is there
  asm volatile("{\n\t.reg .b64 da, db;\n\t.reg .pred p;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %4};\n\tsetp.eq.u32 p, 0, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "n"(A), "n"(B), "n"(IDESC) : "memory");
}
template <uint32_t A, uint32_t B, uint32_t IDESC> __device__ __forceinline__ void u_mma(uint32_t d, uint32_t a, uint32_t b, bool on_top) {
  asm volatile("{\n\t.reg .b64 da, db;\n\t.reg .pred p;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %4};\n\tsetp.ne.u32 p, %6, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "n"(A), "n"(B), "n"(IDESC), "r"((uint32_t)on_top) : "memory");
}
// 8 or 16 columns of the thread's lane
template <int C> __device__ __forceinline__ void u_ld(uint32_t at, float* x) {
  uint32_t r[C];
  if constexpr (C == 16)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < C; ++i) x[i] = __uint_as_float(r[i]);
}
template <int C> __device__ __forceinline__ void u_st(uint32_t at, const float* x) {
  if constexpr (C == 16)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]),
                   "f"(x[8]), "f"(x[9]), "f"(x[10]), "f"(x[11]), "f"(x[12]), "f"(x[13]), "f"(x[14]), "f"(x[15]) : "memory");
  else
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ void u_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the 128 threads of group g of warps
__device__ __forceinline__ void u_sync(int g) { asm volatile("bar.sync %0, 128;" ::"r"(g + 1) : "memory"); }
__device__ __forceinline__ bool u_any(int g, bool yes, int threads = 128) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(yes ? 1u : 0u), "r"(g + 1), "r"(threads) : "memory");
  return r != 0;
}
__device__ __forceinline__ float u_warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// 16-byte piece j of row r, slabs of `rows` rows of 128 bytes
__device__ __forceinline__ uint32_t u_piece(int rows, int r, int j) { return (uint32_t)((j >> 3) * (rows * 128) + r * 128 + (((j & 7) ^ (r & 7)) << 4)); }

// sums over the warp of N values per lane, left in `to` (the next u_sync or u_any makes them seen): half of the values change hands at a time
template <int N> __device__ __forceinline__ void column_sums(float (&l)[N], float* to, int lane) {
  float x[N];
#pragma unroll
  for (int n = 0; n < N; ++n) x[n] = l[n];
  int n0 = 0;
#pragma unroll
  for (int o = 16, m = N; o > 0; o >>= 1) {
    const bool up = lane & o;
    if (m > 1) {
      m /= 2;
#pragma unroll
      for (int k = 0; k < N / 2; ++k)
        if (k < m) {
          const float give = up ? x[k] : x[m + k], mine = up ? x[m + k] : x[k];
          x[k] = mine + __shfl_xor_sync(0xffffffffu, give, o);
        }
      n0 += up ? m : 0;
    } else x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
  }
  constexpr int LEFT = N > 32 ? N / 32 : 1;
#pragma unroll
  for (int k = 0; k < LEFT; ++k) to[n0 + k] = x[k];      // (N = 16: two lanes write the same)
}

__device__ __forceinline__ __nv_bfloat162 bf16x2_of(uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); }
static __device__ __noinline__ uint4 u_eight(const uint16_t* w) {      // not aligned
  return make_uint4(w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16, w[4] | (uint32_t)w[5] << 16, w[6] | (uint32_t)w[7] << 16);
}
// (a copy goes in and out: the cursor itself stays in registers)
static __device__ __noinline__ void u_at_far(const AttnParams& p, Cursor<UT>& c, long long b, long long offset) { c.at(p, b, offset); }
static __device__ __noinline__ void u_next_row(const AttnParams& p, Cursor<UT>& c) { c.next(p); }
__device__ __forceinline__ void u_at(const AttnParams& p, Cursor<UT>& c, long long b, long long offset) {
  Cursor<UT> to;
  u_at_far(p, to, b, offset);
  c = to;
}
__device__ __forceinline__ void u_next(const AttnParams& p, Cursor<UT>& c) {
  if (c.t + 1 < c.s.nt) { ++c.t; return; }
  Cursor<UT> to = c;
  u_next_row(p, to);
  c = to;
}

constexpr float NOTHING = -FLT_MAX;     // the maximum of a row that has seen nothing so far

// GROUPED (D = 128): a box brings both slabs of its positions, [8 positions][2 slabs][8 rows of 128 bytes]; else [slab][128 rows of 128 bytes].  (Boxes of a page
// of 16 positions are 2 KB then, and 32 of them a tile take longer than the bus: 64 sequences of 4096 at 72 % of the copy rate, 88 % with pages of 64.)
template <int DP, int N, bool GROUPED> __global__ void __launch_bounds__(UShape<DP, N>::THREADS, 1) attn_umma_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = UShape<DP, N>;
  using E = __nv_bfloat16;
  constexpr int SLOTS = S::SLOTS, PIECES = DP / 8, PB = S::P_BUFS, GROUPS = S::GROUPS, THREADS = S::THREADS, CW = S::CW;
  constexpr uint32_t SLAB = GROUPED ? 1024 : UT * 128, EIGHT = GROUPED ? S::SLABS * 1024 : 1024;      // bytes from a slab to the next, from eight positions to the next
  auto piece_of = [](int t, int j) { return (uint32_t)((t >> 3) * EIGHT + (j >> 3) * SLAB + (t & 7) * 128 + (((j & 7) ^ (t & 7)) << 4)); };
  extern __shared__ char u_raw[];
  char* const smem = (char*)(((uintptr_t)u_raw + 1023) & ~(uintptr_t)1023);
  char* const p_s = smem + SLOTS * S::SLOT;
  char* const q_s = p_s + PB * S::P_BYTES;
  URest<THREADS>& r = *(URest<THREADS>*)(q_s + 2 * S::Q_BYTES);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    for (int i = 0; i < SLOTS; ++i) { mbar_init(r.full + i, 1); mbar_init(r.empty + i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(r.q_full + i, 1); mbar_init(r.q_empty + i, 1); mbar_init(r.s_full + i, 1); mbar_init(r.p_ready + i, 128 * GROUPS); mbar_init(r.pv_done + i, 1); mbar_init(r.seg_sums + i, 128 * GROUPS); mbar_init(r.seg_pv + i, 1); mbar_init(r.seg_free + i, 128); }
    mbar_init(r.drain, 1); mbar_init(r.drain + 1, 1);
    r.stop[0] = r.stop[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&r.tmem)), "n"(S::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  u_before();
  wait_for_predecessor();
  launch_dependents();
  long long chunk, total;
  pieces<UT, THREADS, 1>(p, r.line, chunk, total);        // (ends with a barrier)
  u_after();
  const uint32_t tmem = *(volatile uint32_t*)&r.tmem;
  const int number = (int)blockIdx.x;
  const long long u0 = number * chunk, limit = p.wait_limit;
  const int n_tiles = u0 < total ? (int)min(chunk, total - u0) : 0;

  if (n_tiles == 0) {
    if (tid == 0) { p.desc[number] = make_int4(0, 0, 0, 0); p.late[number] = make_int2(0, -1); }
  } else if (warp == 0) {
    // ---- loads, in the order in which the products take them up; load j goes to slot j % SLOTS
    Cursor<UT> look;
    u_at(p, look, r.line.b[0], u0 - r.line.before[0]);
    const int boxes = UT / p.box, box_x = lane % boxes * p.box, slab = lane / boxes;
    const bool loads = GROUPED ? slab == 0 : slab < S::SLABS && slab * 64 < p.in.D;
    const uint32_t box_at = (uint32_t)(slab * SLAB + box_x / 8 * EIGHT), box_bytes = (uint32_t)p.box * (GROUPED ? 256 : 128);
    struct Box { int page, x, head; };        // page as it is in the table (what is made of it here would wait for it), x -1: nothing of the lane's box is seen
    auto look_up = [&]() -> Box {             // of the tile at the cursor
      const int x = tile_start<UT>(look.s, look.t) + box_x;
      Box f = {0, -1, p.RB == 1 ? look.hr : look.hr / p.RB};
      if (loads && x < look.s.n && (x + p.box > look.s.lo || x < look.s.sk)) {
        const int page = p.page_shift >= 0 ? x >> p.page_shift : (int)((unsigned)x / (unsigned)p.in.page_size);
        f.page = p.in.page_table[look.b * p.in.ld_table + page];
        f.x = x - page * p.in.page_size;
      }
      return f;
    };
    struct Load { int c1, c2, c3; uint32_t bytes; };           // coordinates of the lane's box (c1 -1: there is none), bytes of the tile
    const int eights = p.in.page_size / 8, mode = p.map_mode;
    const uint32_t ring = smem_addr(smem) + box_at;
    int slot = 0, j = 0;                      // loads so far
    uint32_t turn = 0;
    bool ok = true;
    auto load = [&](const CUtensorMap* map, const Load& f) {
      ok = __all_sync(0xffffffffu, u_wait(r.empty + slot, turn ^ 1u, r, limit));
      if (!ok) return;
      if (lane == 0) mbar_expect_tx(r.full + slot, f.bytes);
      __syncwarp();
      if (f.c1 >= 0) {
        if constexpr (GROUPED) tma_eights(ring + slot * S::SLOT, map, f.c1, f.c2, f.c3, r.full + slot);
        else tma_box(ring + slot * S::SLOT, map, slab * 64, f.c1, f.c2, f.c3, r.full + slot);
      }
      ++j;
      if (++slot == SLOTS) { slot = 0; turn ^= 1u; }
    };
    Box ahead = look_up();                    // the boxes of the next tile, looked up a tile ahead
    Load tile = {}, before = {};              // of the tile whose keys are next or were last, of the one before
#pragma unroll 1
    for (int i = 0; i <= n_tiles && ok; ++i) {      // K0 | K1 V0 | K2 V1 | ... | V(n-1)
      before = tile;
      if (i < n_tiles) {
        const Box f = ahead;
        const bool there = f.x >= 0, in = (unsigned)f.page < (unsigned)p.in.n_pages;
        tile.bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, there && in)) * box_bytes;
        const bool bad = __any_sync(0xffffffffu, there && !in);
        if (lane == 0) { *(volatile int*)(r.bad + (i & 7)) = bad; __threadfence_block(); }
        if constexpr (GROUPED) {
          tile.c1 = mode == MAP_HEADS ? 2 * f.head : 0;
          tile.c2 = (f.x >> 3) + (mode == MAP_RUN ? f.page * eights : 0);
          tile.c3 = mode == MAP_HEADS ? f.page : mode == MAP_PAGES ? f.page * p.in.H + f.head : f.head;
        } else { tile.c1 = f.head; tile.c2 = f.x; tile.c3 = f.page; }
        if (!there || !in) tile.c1 = -1;
        if (i + 1 < n_tiles) { u_next(p, look); ahead = look_up(); }
        load(&k_map, tile);
      }
      if (i > 0 && ok) load(&v_map, before);
    }
    // all copies land before the block leaves, also where the others have given up and do not wait for them
    for (int done = max(0, j - SLOTS); done < j; ++done) mbar_wait_bounded(r.full + done % SLOTS, (uint32_t)(done / SLOTS) & 1u);
  } else if (warp == 1) {
    if (lane == 0) {
      // ---- scores: those of tile i once its keys are there and the weights of tile i - 2 have left their buffer
      constexpr uint32_t ID = u_idesc(N, false), UP_K = u_upper(EIGHT), UP_Q = u_upper(1024);
      Cursor<UT> at;
      u_at(p, at, r.line.b[0], u0 - r.line.before[0]);
      const int steps = (p.in.D + 15) / 16;
      int seg = 0;                            // segments whose queries have been used
      bool first = true;
      for (int i = 0; i < n_tiles; ++i) {
        const int load = load_of_keys(i), slot = load % SLOTS, qb = seg & 1;
        if ((i >= 2 && !u_wait(r.p_ready + (i & 1), ((i - 2) >> 1) & 1, r, limit)) || (first && !u_wait(r.q_full + qb, (seg >> 1) & 1, r, limit)) ||
            !u_wait(r.full + slot, (load / SLOTS) & 1, r, limit)) break;
        u_after();
        const uint32_t k = u_lower(smem_addr(smem + slot * S::SLOT)), q = u_lower(smem_addr(q_s + qb * S::Q_BYTES)), s_to = tmem + (i & 1) * N;
        u_mma<UP_K, UP_Q, ID>(s_to, k, q, false);
#pragma unroll
        for (int e = 1; e < DP / 16; ++e)
          if (e < steps) u_mma<UP_K, UP_Q, ID>(s_to, k + ((e >> 2) * SLAB + (e & 3) * 32) / 16, q + ((e >> 2) * (N * 128) + (e & 3) * 32) / 16);
        u_commit(r.s_full + (i & 1));
        u_commit(r.empty + slot);
        first = at.t + 1 == at.s.nt;
        if (first) { u_commit(r.q_empty + qb); ++seg; }
        u_next(p, at);
      }
      u_commit(r.drain);                      // nothing of it is under way when tensor memory goes (the others may have given up)
      mbar_wait_bounded(r.drain, 0);
    }
  } else if (warp == 2) {
    if (lane == 0) {
      // ---- outputs: tile i's once its weights are there
      constexpr uint32_t ID = u_idesc(2 * N, true), UP_V = u_upper(EIGHT), UP_P = u_upper(1024);
      Cursor<UT> at;
      u_at(p, at, r.line.b[0], u0 - r.line.before[0]);
      int seg = 0;
      bool first = true;
      for (int i = 0; i < n_tiles; ++i) {
        const int load = load_of_values(i, n_tiles), slot = load % SLOTS;
        if ((first && !u_wait(r.seg_free + (seg & 1), ((seg >> 1) & 1) ^ 1u, r, limit)) || !u_wait(r.full + slot, (load / SLOTS) & 1, r, limit) ||
            !u_wait(r.p_ready + (i & 1), (i >> 1) & 1, r, limit)) break;
        u_after();
        const bool on_top = !first || *(volatile int*)(r.keep + (i & 1));
        const uint32_t v = u_lower(smem_addr(smem + slot * S::SLOT), DP == 128 ? SLAB : 0), w = u_lower(smem_addr(p_s + i % PB * S::P_BYTES)), o = tmem + 2 * N + (seg & 1) * 2 * N;
        u_mma<UP_V, UP_P, ID>(o, v, w, on_top);
#pragma unroll
        for (int e = 1; e < 8; ++e)           // steps of 16 positions
          u_mma<UP_V, UP_P, ID>(o, v + e * 2 * EIGHT / 16, w + ((e >> 2) * (N * 256) + (e & 3) * 32) / 16);
        u_commit(r.pv_done + (i & 1));
        u_commit(r.empty + slot);
        first = at.t + 1 == at.s.nt;
        if (first || i + 1 == n_tiles) { u_commit(r.seg_pv + (seg & 1)); ++seg; }
        u_next(p, at);
      }
      u_commit(r.drain + 1);
      mbar_wait_bounded(r.drain + 1, 0);
    }
  } else if (warp == 3) {
    // ---- queries of the piece's segments
    Cursor<UT> at;
    u_at(p, at, r.line.b[0], u0 - r.line.before[0]);
    constexpr int EACH = N * PIECES / 32, BATCH = EACH < 8 ? EACH : 8;
    long long left = n_tiles;
#pragma unroll 1
    for (int seg = 0; left > 0; ++seg) {
      const int qb = seg & 1;
      if (!__all_sync(0xffffffffu, u_wait(r.q_empty + qb, ((seg >> 1) & 1) ^ 1u, r, limit))) break;
      const int h = p.RB == 1 ? at.hr : at.hr / p.RB;
      if (seg == 0 || p.RB > 1) {             // where the rows' queries are within a sequence and key head
        __syncwarp();
        for (int n = lane; n < N; n += 32) {
          const int row = at.hr % p.RB * N + n, t = row / p.G;
          r.q_at[n] = row < p.R ? t * p.in.q_pos + (int64_t)(row - t * p.G) * p.in.q_head : -1;
        }
        __syncwarp();
      }
      const E* const from = (const E*)p.in.q + at.b * p.in.q_seq + (int64_t)(h * p.G) * p.in.q_head;
      const int jj = lane % PIECES;
      const uint32_t g = p.q_sign;
      auto put = [&](int e, uint4 x) {
        *(uint4*)(q_s + qb * S::Q_BYTES + u_piece(N, e * (32 / PIECES) + lane / PIECES, jj)) = make_uint4(x.x ^ g, x.y ^ g, x.z ^ g, x.w ^ g);
      };
      auto at_of = [&](int e) -> int64_t {
        const int64_t q_at = r.q_at[e * (32 / PIECES) + lane / PIECES];
        return jj * 8 < p.in.D ? q_at : -1;
      };
      if (p.q_vec) {
#pragma unroll 1
        for (int e0 = 0; e0 < EACH; e0 += BATCH) {
          uint4 x[BATCH];                     // all on their way before the first is put down
#pragma unroll
          for (int e = 0; e < BATCH; ++e) {
            const int64_t q_at = at_of(e0 + e);
            x[e] = q_at >= 0 ? *(const uint4*)(from + q_at + jj * 8) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int e = 0; e < BATCH; ++e) put(e0 + e, x[e]);
        }
      } else {
#pragma unroll 1
        for (int e = 0; e < EACH; ++e) {
          const int64_t q_at = at_of(e);
          put(e, q_at >= 0 ? u_eight((const uint16_t*)(from + q_at + jj * 8)) : make_uint4(0, 0, 0, 0));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) u_arrive(r.q_full + qb);
      left -= at.s.nt - at.t;
      at.t = at.s.nt - 1;
      u_next(p, at);
    }
  } else if (warp >= 4 && warp < 4 + 4 * GROUPS) {
    // ---- weights: thread t of group g is position t of the tile, for queries c0 to c0 + CW
    const int t = (tid - 128) & 127, q4 = warp & 3, g = (warp - 4) >> 2, c0 = g * CW;
    const uint32_t lanes = (uint32_t)(q4 * 32) << 16;
    float* const m_s = r.m + c0;
    float* const factor_s = r.factor + c0;
    int* const to_s = r.to + c0;
    int* const from_s = r.from + c0;
    auto by_four = [&](const float* x, auto&& f) {
#pragma unroll
      for (int n = 0; n < CW; n += 4) { const float4 y = *(const float4*)(x + n); f(n, y.x); f(n + 1, y.y); f(n + 2, y.z); f(n + 3, y.w); }
    };
    Cursor<UT> now;
    u_at(p, now, r.line.b[0], u0 - r.line.before[0]);
    bool dead = false, fresh = true;          // no tile of the segment so far
    float l[CW], bad = 0.f;
    int seg = 0, my_query = 0;
#pragma unroll 1
    for (int i = 0; i < n_tiles; ++i) {
      {
        const int x0 = tile_start<UT>(now.s, now.t), x = x0 + t;
        if (fresh) {
          u_sync(g);               // (the segment before is done with what is written here)
          if (t < CW) {
            if (p.RB > 1 || seg == 0) {       // (a division)
              const int row = now.hr % p.RB * N + c0 + t;
              my_query = row < p.R ? row / p.G : INT_MAX;
            }
            const int at = my_query < now.s.nq ? now.s.p0 + my_query : -1;
            to_s[t] = at; from_s[t] = p.in.window > 0 ? (int)max((int64_t)0, (int64_t)at - p.in.window + 1) : 0;
            m_s[t] = NOTHING;
          }
#pragma unroll
          for (int n = 0; n < CW; ++n) l[n] = 0.f;
          bad = 0.f;
          u_sync(g);
        }
        if (!dead && !u_wait(r.s_full + (i & 1), (i >> 1) & 1, r, limit)) dead = true;
        u_after();
        float w[CW];
        if (*(volatile int*)(r.bad + (i & 7))) bad = -1.f;
        const bool edge = !whole<UT>(p, now.s, x0), hidden = !(x < now.s.n && (x >= now.s.lo || x < now.s.sk));
        const int sinks = p.in.window > 0 ? p.in.sinks : 0;
        // in front of some rows, behind others
        const bool partly = edge && !hidden && !(now.s.nq == p.in.Q && x <= now.s.p0 && (p.in.window <= 0 || x > now.s.n - 1 - p.in.window || x < sinks));
        auto scores = [&] {
          u_ld<CW>(tmem + lanes + (i & 1) * N + c0, w);
          if (hidden) {
#pragma unroll
            for (int n = 0; n < CW; ++n) w[n] = -CUDART_INF_F;
          } else if (partly) {
#pragma unroll
            for (int n = 0; n < CW; ++n)
              if (!(x <= to_s[n] && (x >= from_s[n] || x < sinks))) w[n] = -CUDART_INF_F;
          }
        };
        float big = 0.f;
        bool exact = fresh && edge;
        auto weights = [&] {
          by_four(m_s, [&](int n, float m) { w[n] = fmaf(w[n], p.c, -m); });
          if (exact)               // (elsewhere a weight beyond 2^8 leads here)
#pragma unroll
            for (int n = 0; n < CW; ++n) w[n] = cut_exponent(w[n]);
#pragma unroll
          for (int n = 0; n < CW; ++n) { w[n] = ex2f(w[n]); big = fmaxf(big, w[n]); }
        };
#pragma unroll 1
        for (;;) {
          scores();
          if (exact) {             // the rows' maxima
#pragma unroll
            for (int n = 0; n < CW; ++n) {
              const float top = u_warp_max(w[n]);
              if (lane == n) r.top[q4][c0 + n] = top;
            }
            u_sync(g);
            if (t < CW) {
              const int n = c0 + t;
              const float most = fmaxf(fmaxf(r.top[0][n], r.top[1][n]), fmaxf(r.top[2][n], r.top[3][n])), before = m_s[t], m = fmaxf(before, __fmul_rd(most, p.c));
              m_s[t] = m;
              factor_s[t] = ex2f(before - m);
            }
            u_sync(g);
            if (!fresh) {          // ... and what is there already
              if (!dead && !u_wait(r.pv_done + ((i - 1) & 1), ((i - 1) >> 1) & 1, r, limit)) dead = true;
              u_after();
#pragma unroll 1
              for (int k = 0; k < 2; ++k) {
                const uint32_t at = tmem + lanes + 2 * N + (seg & 1) * 2 * N + k * N + c0;
                float y[CW];
                u_ld<CW>(at, y);
#pragma unroll
                for (int e = 0; e < CW; ++e) y[e] *= factor_s[e];
                u_st<CW>(at, y);
              }
              u_st_wait();
              by_four(factor_s, [&](int n, float f) { l[n] *= f; });
            }
          } else if (fresh) {
            // any maximum will do that none of the positions passes by 2^8: that of a quarter of them, each warp for a quarter of the rows
#pragma unroll
            for (int k = 0; k < CW / 4; ++k) {
              const float top = u_warp_max(q4 == 0 ? w[k] : q4 == 1 ? w[CW / 4 + k] : q4 == 2 ? w[CW / 2 + k] : w[3 * CW / 4 + k]);
              if (lane == k) m_s[q4 * (CW / 4) + k] = fmaxf(NOTHING, __fmul_rd(top, p.c));
            }
            u_sync(g);
          }
          weights();
          if (exact || !u_any(g, big > 256.f)) break;
          exact = true;
        }
#pragma unroll
        for (int n = 0; n < CW; ++n) l[n] += w[n];
        const int v_load = load_of_values(i, n_tiles);
        char* const v_s = smem + v_load % SLOTS * S::SLOT;
        bool keep = false;
        if (edge) {
          if (!dead && !u_wait(r.full + v_load % SLOTS, (v_load / SLOTS) & 1, r, limit)) dead = true;
          if (hidden && g == 0)    // values of positions that nothing sees: whatever lies there
#pragma unroll 1
            for (int j = 0; j < PIECES; ++j) *(uint4*)(v_s + piece_of(t, j)) = make_uint4(0, 0, 0, 0);
          if (p.in.Q > 1) {        // some rows do not see all of the tile: a value that is not finite must not reach those as 0 * inf
            const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
            __nv_bfloat162 z[4] = {zero, zero, zero, zero};      // 0 x, added up: NaN once there is such a value
            if (partly)            // (each group looks at a share)
#pragma unroll
              for (int j = g; j < PIECES; j += GROUPS) {
                const uint4 y = *(const uint4*)(v_s + piece_of(t, j));
                z[0] = __hfma2(bf16x2_of(y.x), zero, z[0]); z[1] = __hfma2(bf16x2_of(y.y), zero, z[1]);
                z[2] = __hfma2(bf16x2_of(y.z), zero, z[2]); z[3] = __hfma2(bf16x2_of(y.w), zero, z[3]);
              }
            const float2 z2 = __bfloat1622float2(__hadd2(__hadd2(z[0], z[1]), __hadd2(z[2], z[3])));
            const bool strange = !(z2.x + z2.y == 0.f);
            if (u_any(6, strange, 128 * GROUPS)) { // (one answer for all groups, whatever one that has given up reads) it goes to the rows that see it by itself, and 0 takes its place
              if (!fresh) {
                if (!dead && !u_wait(r.pv_done + ((i - 1) & 1), ((i - 1) >> 1) & 1, r, limit)) dead = true;
              } else if (!dead && !u_wait(r.seg_free + (seg & 1), ((seg >> 1) & 1) ^ 1u, r, limit)) dead = true;
              u_after();
              keep = fresh;
              {
                const uint32_t o_at = tmem + lanes + 2 * N + (seg & 1) * 2 * N + c0;
                float y[CW];
                if (fresh) {
#pragma unroll
                  for (int e = 0; e < CW; ++e) y[e] = 0.f;
                  u_st<CW>(o_at + N, y);
                } else u_ld<CW>(o_at, y);
                if (t < DP)
#pragma unroll 1
                  for (int pos = 0; pos < UT; ++pos) {      // (positions that all rows see are left to the product)
                    const int xx = x0 + pos;
                    if (!(xx < now.s.n && (xx >= now.s.lo || xx < now.s.sk))) continue;
                    if (now.s.nq == p.in.Q && xx <= now.s.p0 && (p.in.window <= 0 || xx > now.s.n - 1 - p.in.window || xx < sinks)) continue;
                    const float z = __bfloat162float(*(const E*)(v_s + piece_of(pos, t >> 3) + (t & 7) * 2));
                    if (!(fabsf(z) < CUDART_INF_F))
#pragma unroll
                      for (int e = 0; e < CW; ++e)
                        if (xx <= to_s[e] && (xx >= from_s[e] || xx < sinks)) y[e] += z;
                  }
                u_st<CW>(o_at, y);
              }
              u_st_wait();
              asm volatile("bar.sync 7, %0;" ::"n"(128 * GROUPS) : "memory");      // (all groups have it)
              if (partly && g == 0)
#pragma unroll 1
                for (int j = 0; j < PIECES; ++j) {
                  uint4* const at = (uint4*)(v_s + piece_of(t, j));
                  auto clean = [](uint32_t y) { return ((y & 0x7f800000u) == 0x7f800000u ? 0u : y & 0xffff0000u) | ((y & 0x7f80u) == 0x7f80u ? 0u : y & 0xffffu); };
                  const uint4 y = *at;
                  *at = make_uint4(clean(y.x), clean(y.y), clean(y.z), clean(y.w));
                }
            }
          }
        }
        if (i >= PB && !dead && !u_wait(r.pv_done + ((i - PB) & 1), ((i - PB) >> 1) & 1, r, limit)) dead = true;      // the buffer's last product
        if (t == 0 && g == 0) {
          *(volatile int*)(r.keep + (i & 1)) = keep;      // (only now: before that product was issued, tile i - 2's word was still to be read)
          *(volatile int*)(r.stop + 1) = i + 1;
        }
        {
          char* const at = p_s + (i % PB) * S::P_BYTES + (t >> 6) * (N * 256) + (t & 7) * 2 + c0 * 128;
          const uint32_t piece = (uint32_t)((t >> 3) & 7) << 4;
#pragma unroll
          for (int n = 0; n < CW; n += 2) {
            const uint32_t a = __float_as_uint(w[n]), b = __float_as_uint(w[n + 1]);
            const float2 rest = fadd2(make_float2(w[n], w[n + 1]), make_float2(-__uint_as_float(a & 0xffff0000u), -__uint_as_float(b & 0xffff0000u)));
            const uint32_t lo = pack_bf16x2(rest.x, rest.y);
            char* const p0 = at + n * 128 + (piece ^ (uint32_t)((n & 7) << 4));
            char* const p1 = at + (n + 1) * 128 + (piece ^ (uint32_t)(((n + 1) & 7) << 4));
            *(uint16_t*)p0 = (uint16_t)(a >> 16);
            *(uint16_t*)p1 = (uint16_t)(b >> 16);
            *(uint16_t*)(p0 + N * 128) = (uint16_t)lo;
            *(uint16_t*)(p1 + N * 128) = (uint16_t)(lo >> 16);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        u_before();
        u_arrive(r.p_ready + (i & 1));
        fresh = false;
      }
      if (now.t + 1 == now.s.nt || i + 1 == n_tiles) {        // the segment ends, or the piece does: to the warps that write
        const int sb = seg & 1;
        if (!dead && !u_wait(r.seg_free + sb, ((seg >> 1) & 1) ^ 1u, r, limit)) dead = true;
        column_sums<CW>(l, r.end_sum[sb][q4] + c0, lane);
        if (t < CW) r.end_m[sb][c0 + t] = m_s[t];
        if (t == 0 && g == 0) r.end_bad[sb] = bad < 0.f;
        u_arrive(r.seg_sums + sb);
        fresh = true;
        ++seg;
      }
      u_next(p, now);
    }
  } else if (warp >= 4 + 4 * GROUPS) {
    // ---- results: thread t is column t of the output
    const int t = tid & 127, q4 = warp & 3;
    const uint32_t lanes = (uint32_t)(q4 * 32) << 16;
    Cursor<UT> at;
    u_at(p, at, r.line.b[0], u0 - r.line.before[0]);
    bool dead = false;
    int left = n_tiles, row = 0, j = 0;
    int2 late = make_int2(INT_MAX, -1);
#pragma unroll 1
    for (int seg = 0; left > 0; ++seg) {
      const int sb = seg & 1, rest = at.s.nt - at.t;
      const bool head = at.t > 0, tail = left < rest;        // the segment goes on from the piece before, or behind
      const int h = p.RB == 1 ? at.hr : at.hr / p.RB;
      const int n = t;
      if (t < N) {
        if (seg == 0 || p.RB > 1) {           // (a division)
          row = at.hr % p.RB * N + t;
          j = row / p.G;
        }
        r.row_at[t] = row < p.R ? at.b * p.out.o_seq + j * p.out.o_pos + (int64_t)(h * p.G + row - j * p.G) * p.out.o_head : -1;
      }
      if (!dead && !u_wait(r.seg_sums + sb, (seg >> 1) & 1, r, limit)) dead = true;
      if (!dead && !u_wait(r.seg_pv + sb, (seg >> 1) & 1, r, limit)) dead = true;
      u_after();
      // (a group that gave up goes on without waiting, so the rest may have come from nothing: it said so before)
      const float b = u_any(GROUPS, dead || *(volatile int*)r.stop) ? -2.f : r.end_bad[sb] ? -1.f : 0.f;
      const uint32_t st = at.s.status | status_of(b);
      const bool partial = head || tail;
      float* const part = p.part + (number * 2 + (head ? 0 : 1)) * (int64_t)PART<N, DP>;
      if (t < N) {
        const float m = r.end_m[sb][n], sum = (r.end_sum[sb][0][n] + r.end_sum[sb][1][n]) + (r.end_sum[sb][2][n] + r.end_sum[sb][3][n]);
        r.inverse[n] = partial ? 1.f : st || sum == 0.f ? 0.f : 1.f / sum;      // (of a flagged segment nothing is used, whatever it is)
        if (row < p.R) {
          if (partial) *(float2*)(part + N * DP + n * 2) = make_float2(m, b < 0.f ? b : sum);
          else if (p.out.lse) p.out.lse[((int64_t)at.b * p.in.Q + j) * p.in.Hq + h * p.G + row - j * p.G] = lse_of(m, st ? 0.f : sum);
        }
      }
      u_sync(GROUPS);
      const int D = partial ? DP : p.in.D;
#pragma unroll 1
      for (int n0 = 0; n0 < N; n0 += 8) {
        if (r.row_at[n0] < 0) break;          // (rows that there are come first)
        float o[8], y[8];
        const uint32_t o_at = tmem + lanes + 2 * N + sb * 2 * N + n0;
        u_ld<8>(o_at, o);
        u_ld<8>(o_at + N, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int64_t to = r.row_at[n0 + e];
          const float f = r.inverse[n0 + e], x = f == 0.f ? 0.f : (o[e] + y[e]) * f;
          if (to >= 0 && t < D) {
            if (partial) part[(n0 + e) * DP + t] = x;
            else ((E*)p.out.out)[to + t] = __float2bfloat16_rn(x);
          }
        }
      }
      u_before();
      u_arrive(r.seg_free + sb);
      if (t == 0) {
        if (!head && at.hr == 0) put_status(p, at.b, tail ? at.s.status : st);
        if (b == -2.f) { late.x = min(late.x, at.b); late.y = at.b; }
        if (left <= rest)          // a segment that starts here and goes on: how many pieces behind have a share of it
          p.desc[number] = tail && !head ? make_int4(at.b, at.hr, (int)((u0 + n_tiles - left - at.t + at.s.nt - 1) / chunk) - number, (int)at.s.status) : make_int4(0, 0, 0, 0);
      }
      left -= rest;
      at.t = at.s.nt - 1;
      u_next(p, at);
      u_sync(GROUPS);              // (row_at and inverse are written again)
    }
    if (t == 0) p.late[number] = late;
  }
  u_before();
  __syncthreads();
  if (warp == 2) {
    u_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS) : "memory");
  }
}

template <int DP, int N, bool GROUPED> cudaError_t launch(const AttnParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, int blocks, cudaStream_t st) {
  using S = UShape<DP, N>;
  auto* const fn = attn_umma_kernel<DP, N, GROUPED>;
  const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  return e != cudaSuccess ? e : launch_pdl(fn, dim3((unsigned)blocks), S::THREADS, S::SMEM, st, true, p, k_map, v_map);
}
template <int DP, bool GROUPED> cudaError_t launch(const AttnParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, int blocks, cudaStream_t st) {
  const int n = umma_rows(p.in);
  return n == 16 ? launch<DP, 16, GROUPED>(p, k_map, v_map, blocks, st) : n == 32 ? launch<DP, 32, GROUPED>(p, k_map, v_map, blocks, st) : launch<DP, 64, GROUPED>(p, k_map, v_map, blocks, st);
}

}  // namespace

int umma_rows(const saki_attn_in& in) {
  const int R = in.Q * (in.Hq / in.H);
  return R <= 16 ? 16 : R <= 32 ? 32 : 64;
}

cudaError_t launch_umma(const AttnParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, int blocks, cudaStream_t st) {
  return p.in.D <= 64 ? launch<64, false>(p, k_map, v_map, blocks, st) : p.map_mode ? launch<128, true>(p, k_map, v_map, blocks, st) : launch<128, false>(p, k_map, v_map, blocks, st);
}

}  // namespace attn

}  // namespace saki
