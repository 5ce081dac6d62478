// Attention of a few new tokens per sequence over a paged key-value cache.
//
// Every key and value is read once for all G * Q query rows that meet it (G query heads share a key head, Q new tokens), up to 128 of them (64 on tcgen05, and for float32 heads above 128; more rows are
// further row blocks, which read it again).  The work is therefore laid out by what is read: the visible positions of all sequences, key heads and row
// blocks, in tiles of T positions, form one line of tiles that is cut into equal pieces, whatever the lengths are (they are known on
// the device only).  A piece belongs to one worker: a warp (two or four warps where there are more rows than one holds) with a ring of tiles in
// shared memory of its own, which it fills by TMA ahead of its products, across the ends of sequences.  No worker waits for another; each row's running maximum, sum
// and weighted values stay in registers.  Where a cut falls inside a sequence the two sides leave partial results in scratch, which a second small
// kernel joins in the order of the line.
//
//   s = scale * q.k,   m' = max(m, s),   l = l 2^(m - m') + 2^(s - m'),   o = o 2^(m - m') + 2^(s - m') v       (s, m in units of log 2)
//
// This file's kernel runs the products on mma.sync with float32 accumulators, query rows in groups of 16: float32, bf16 heads above 128 and up to 16, pages that are no whole
// eights, and single tokens of few rows with small heads or little to see (`on_umma`); all other bf16 calls go to saki_attention_umma.cu.  bf16: m16n8k16; the weights go into the second product as two bf16 terms, so that they carry 16 bits: one
// term would add an error as large as the rounding of the output (2^-9 each).  f32: m16n8k8 on tf32 terms, x = hi + lo with 11 bits each and
// hi.hi + hi.lo + lo.hi: what is dropped is 2^-21 of a product and less, of either sign.
// What bounds it: the latency of a tile's chain of small products at two warps a scheduler.  bf16, heads of 64, 96 sequences of 8000 positions, 5 rows, pages of 32
// positions, one head after the other: 311 us, 5.1 TB/s (77 % of the measured copy rate; 406 where the heads of a position lie side by side, 128 bytes each); 96 windows of 1024: 61 us.  Heads of 256, 64
// sequences of 4096: 4 rows 560 us (59 %), 28 rows 1131 (29 %: tiles of 16 positions, one warp a scheduler).  f32, heads of 80, 24 sequences of 15000 positions, 3 rows: 217 us, 3.2 TB/s (49 %), heads
// of 128 381 (44 %; tiles of 8 positions); of up to 3001, 9 rows: 65 us (some 1400 instructions a warp and tile of 16 positions, half of them the splitting into terms and their products; 251 registers, so eight warps).
#include "saki_attention.cuh"
#include <algorithm>
#include <climits>
#include <cmath>

namespace saki {

using namespace attn;

namespace {

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool real) {      // zeros where not real
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_arrive(uint64_t* bar) {      // once the thread's copies so far are there
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm2(uint32_t (&r)[2], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x as two tf32 terms.  The first factor of a product (queries, weights): the nearest number of 11 bits and the rest, of either sign and at most 2^-11 of x, of which the product keeps 11 bits
// (2^-23 of x is cut).  Numbers from (2 - 2^-11) 2^127 on become infinite.
__device__ __forceinline__ void two_nearest(uint32_t x, uint32_t& hi, uint32_t& lo) {
  hi = (x + 0x1000u) & 0xffffe000u;
  lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi));
}
// The second (keys, values, which may hold the largest numbers where some rows do not look): the upper 11 bits, and the rest (exact, below 2^-10 of x) with half a unit added, as the product cuts
// it to 11 bits: 2^-22 of x.  With both factors split like this what is dropped, lo.lo, would be up to 2^-20 and always of the product's sign (the error against 64 bits 6.7e-7 where it is 5.4e-7; a
// plain float32 form has 6.0e-7).
__device__ __forceinline__ void two_terms(uint32_t x, uint32_t& hi, uint32_t& lo) {
  hi = x & 0xffffe000u;
  lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi)) + 0x1000u;
}

// NW: warps of a worker, 16 rows each
template <typename E, int DP, int NW_> struct Shape {
  static constexpr bool F32 = sizeof(E) == 4;
  static constexpr int NW = NW_, WARPS = DP == 256 && NW <= 4 ? 4 : 8, THREADS = 32 * WARPS, WORKERS = WARPS / NW, ROWS = 16 * NW;
  static constexpr int T = F32 ? (DP <= 96 ? 16 : 8) : (DP == 64 ? 32 : 16);         // positions of a tile (f32, heads of 80, 8 and 16: 294 and 217 us at 24 sequences of 15000)
  static constexpr int COLS = 128 / (int)sizeof(E), SLABS = DP / COLS;               // columns of a 128-byte slab [T][128 bytes]
  static constexpr int HALF = T * DP * (int)sizeof(E), STAGE = 2 * HALF;             // keys, then values
  static constexpr bool Q_REGS = F32 && DP <= 128;                                   // queries in registers: the room is for the ring
  static constexpr int Q_BYTES = Q_REGS ? 0 : ROWS * DP * (int)sizeof(E);            // of a worker
  static constexpr int FIT = (226 * 1024 - WORKERS * Q_BYTES - 1024 - 8 * THREADS) / (WORKERS * (STAGE + 8));
  static constexpr int MOST = NW == 8 ? 24 : 4 * NW, STAGES = FIT < MOST ? FIT : MOST;
  static constexpr int SMEM = WORKERS * (STAGES * (STAGE + 8) + Q_BYTES) + (int)sizeof(LineShared<THREADS>) + 1024;
  static_assert(STAGES >= 2 && STAGES < 32 && SMEM <= 227 * 1024, "a block's shared memory");
  static_assert(2 * SMEM > 227 * 1024, "one block on each SM");
};
// 16-byte piece j of row r in a slab layout with `rows` rows a slab: eight pieces of a row are swizzled by the row, as TMA lays them down
template <int ROWS> __device__ __forceinline__ uint32_t piece_at(int r, int j) { return (uint32_t)((j >> 3) * (ROWS * 128) + r * 128 + (((j & 7) ^ (r & 7)) << 4)); }
// ... piece 2 k + e of a lane's row, from the address of piece e: the slab's rows are eight times 128 bytes and the base a multiple of 1024, so that the swizzle
// is an exclusive or with a constant
template <int ROWS> __device__ __forceinline__ uint32_t pair_at(uint32_t first, int k) { return (first ^ (uint32_t)(((2 * k) & 7) << 4)) + (uint32_t)((k >> 2) * (ROWS * 128)); }

// TMA: tiles come as boxes of `box` positions (a page is a multiple of eight positions); else 16 bytes at a time.
template <typename E, int DP, int NW, bool TMA>
__global__ void __launch_bounds__(Shape<E, DP, NW>::THREADS) attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = Shape<E, DP, NW>;
  constexpr int T = S::T, ST = S::STAGES, ND = DP / 8, NT = T / 8, PE = 16 / (int)sizeof(E), PIECES = DP / PE, THREADS = S::THREADS;
  constexpr bool F32 = S::F32;
  extern __shared__ char smem_raw[];
  char* const smem = (char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, worker = warp / NW, part_of = warp % NW;
  char* const ring = smem + worker * ST * S::STAGE;
  char* const q_s = smem + S::WORKERS * ST * S::STAGE + worker * S::Q_BYTES;
  char* const rest = smem + S::WORKERS * (ST * S::STAGE + S::Q_BYTES);
  uint64_t* const full = (uint64_t*)rest + worker * ST;
  LineShared<THREADS>& line = *(LineShared<THREADS>*)(rest + S::WORKERS * ST * 8);
  const uint32_t ring_a = smem_addr(ring), q_a = smem_addr(q_s);
  auto together = [&] {            // the worker's warps
    if constexpr (NW == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(worker + 1), "r"(32 * NW) : "memory");
  };
  auto any_of_us = [&](bool yes) -> bool {      // one answer for all threads of the worker, who meet there
    if constexpr (NW == 1) return __any_sync(0xffffffffu, yes);
    else {
      uint32_t any;
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                   : "=r"(any) : "r"(yes ? 1u : 0u), "r"(worker + 1), "r"(32 * NW) : "memory");
      return any != 0;
    }
  };

  // columns behind D stay zero (TMA fills a slab that it loads)
  if (TMA ? p.in.D <= DP - S::COLS : p.in.D < DP) {
    for (int i = tid; i < S::WORKERS * ST * 2 * T * PIECES; i += THREADS) {
      const int r = i / PIECES, j = i % PIECES;
      if ((TMA ? j / 8 * 8 : j) * PE >= p.in.D) *(uint4*)(smem + r / T * S::HALF + piece_at<T>(r % T, j)) = make_uint4(0, 0, 0, 0);
    }
  }
  if (part_of == 0 && lane < ST) mbar_init(full + lane, TMA ? 1 : 32);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  wait_for_predecessor();
  launch_dependents();
  const int number = worker * (int)gridDim.x + (int)blockIdx.x;
  long long chunk, total;
  pieces<T, THREADS, S::WORKERS>(p, line, chunk, total);        // (ends with a barrier: the mbarriers are there for all)
  const long long u0 = number * chunk;
  if (u0 >= total) {
    if (part_of == 0 && lane == 0) { p.desc[number] = make_int4(0, 0, 0, 0); p.late[number] = make_int2(0, -1); }
    return;
  }
  const int n_tiles = (int)min(chunk, total - u0);
  Cursor<T> now;
  now.at(p, line.b[worker], u0 - line.before[worker]);

  // The ring: tile i of the piece lies in stage i % ST.  The pages of a tile are looked up one tile ahead of its load.
  Cursor<T> look = now;
  int looked = 0, loaded = 0, load_stage = 0;
  const int boxes = TMA ? T / p.box : 1, box_x = TMA ? lane % boxes * p.box : 0, slab_i = TMA ? lane / boxes % S::SLABS : 0, second = TMA ? lane / (boxes * S::SLABS) : 0;
  const bool loads = TMA ? second < 2 && slab_i * S::COLS < p.in.D : lane < T;
  const CUtensorMap* const map = second ? &v_map : &k_map;
  const uint32_t box_at = TMA ? (uint32_t)(second * S::HALF + slab_i * (T * 128) + box_x * 128) : 0;
  int found = 0, found_slot = 0, found_head = 0;      // of the tile to load next: the lane's page (TMA: of its box; else of position `lane`), -1: nothing to load, -2: outside the pool
  auto look_up = [&] {
    found = -1;
    if (looked >= n_tiles) return;
    const int x = tile_start<T>(look.s, look.t) + (TMA ? box_x : lane), end = TMA ? x + p.box : x + 1;
    if (loads && x < look.s.n && (end > look.s.lo || x < look.s.sk)) {        // any of it is seen
      const int page = p.page_shift >= 0 ? x >> p.page_shift : (int)((unsigned)x / (unsigned)p.in.page_size);
      found = p.in.page_table[look.b * p.in.ld_table + page];
      found_slot = x - page * p.in.page_size;
      if ((unsigned)found >= (unsigned)p.in.n_pages) found = -2;
    }
    found_head = p.RB == 1 ? look.hr : look.hr / p.RB;
    look.next(p);
    ++looked;
  };
  uint32_t bad_tiles = 0;          // bit i % 32: a page of tile i is outside the pool
  auto load = [&] {                // the tile that was looked up
    if (loaded >= n_tiles) return;
    const bool bad = __any_sync(0xffffffffu, found == -2);
    bad_tiles = (bad_tiles & ~(1u << (loaded & 31))) | (uint32_t)bad << (loaded & 31);
    if (part_of == 0) {
      const uint32_t at = ring_a + load_stage * S::STAGE;
      if constexpr (TMA) {
        const unsigned wanted = __ballot_sync(0xffffffffu, found >= 0);
        if (lane == 0) mbar_expect_tx(full + load_stage, (uint32_t)(__popc(wanted) * p.box * 128));
        __syncwarp();
        if (found >= 0) tma_box(at + box_at, map, slab_i * S::COLS, found_head, found_slot, found, full + load_stage);
      } else {
        const int64_t k_at = found >= 0 ? found * p.in.kp_page + found_slot * p.in.kp_pos + found_head * p.in.kp_head : -1;
        const int64_t v_at = found >= 0 ? found * p.in.vp_page + found_slot * p.in.vp_pos + found_head * p.in.vp_head : -1;
#pragma unroll 4
        for (int e = lane; e < T * PIECES; e += 32) {
          const int r = e / PIECES, j = e % PIECES;
          const int64_t k = __shfl_sync(0xffffffffu, k_at, r), v = __shfl_sync(0xffffffffu, v_at, r);
          if (j * PE < p.in.D) {
            cp16(at + piece_at<T>(r, j), (const E*)p.in.k_pages + (k < 0 ? 0 : k + j * PE), k >= 0);
            cp16(at + S::HALF + piece_at<T>(r, j), (const E*)p.in.v_pages + (v < 0 ? 0 : v + j * PE), v >= 0);
          }
        }
        cp_arrive(full + load_stage);
      }
    }
    ++loaded;
    load_stage = load_stage + 1 == ST ? 0 : load_stage + 1;
  };
  look_up();
#pragma unroll 1
  for (int i = 0; i < ST - 1; ++i) { load(); look_up(); }

  uint32_t q_r[S::Q_REGS ? DP / 8 : 1][4];      // the lane's share of the queries, as the products take them
  float o[ND][4], m[2], l[2];
  Sight sight[2];
  float bad = 0.f;                 // -1: a page outside the pool, -2: a wait ran out (from then on nothing is loaded or waited for)
  bool fresh = true, gave_up = false;
  int2 late = make_int2(INT_MAX, -1);
  int stage = 0;
  uint32_t parity = 0;
  // what a lane reads: rows of eight by lane & 7, pieces and groups of eight rows by lane >> 3
  const int r7 = lane & 7, mi = lane >> 3;
  const uint32_t q_l = q_a + (uint32_t)((part_of * 16 + (mi & 1) * 8 + r7) * 128 + (((mi >> 1) ^ r7) << 4));
  const uint32_t k_l = F32 ? (uint32_t)(r7 * 128 + (((mi & 1) ^ r7) << 4)) : (uint32_t)(((mi >> 1) * 8 + r7) * 128 + (((mi & 1) ^ r7) << 4));
  const uint32_t v_l = (uint32_t)(S::HALF + ((mi & 1) * 8 + r7) * 128 + (((mi >> 1) ^ r7) << 4));
#pragma unroll 1
  for (int i = 0; i < n_tiles; ++i) {
    const int h = p.RB == 1 ? now.hr : now.hr / p.RB, row0 = (now.hr - h * p.RB) * S::ROWS;
    if (fresh) {                   // a new segment: its queries
      if constexpr (S::Q_REGS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = row0 + part_of * 16 + (lane >> 2) + 8 * i, j = r / p.G;
          const E* const q = (const E*)p.in.q + now.b * p.in.q_seq + j * p.in.q_pos + (int64_t)(h * p.G + r - j * p.G) * p.in.q_head;
#pragma unroll
          for (int k = 0; k < DP / 8; ++k)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int col = k * 8 + (lane & 3) + 4 * c;
              q_r[k][2 * c + i] = r < p.R && col < p.in.D ? __float_as_uint((float)q[col]) ^ p.q_sign : 0u;
            }
        }
      } else {
        for (int e = part_of * 32 + lane; e < S::ROWS * PIECES; e += 32 * NW) {
          const int rr = e / PIECES, jj = e % PIECES, r = row0 + rr, j = r / p.G;
          uint4 x = make_uint4(0, 0, 0, 0);
          if (r < p.R && jj * PE < p.in.D) {
            const E* const q = (const E*)p.in.q + now.b * p.in.q_seq + j * p.in.q_pos + (int64_t)(h * p.G + r - j * p.G) * p.in.q_head + jj * PE;
            if (p.q_vec) x = *(const uint4*)q;
            else if constexpr (F32) { const uint32_t* const w = (const uint32_t*)q; x = make_uint4(w[0], w[1], w[2], w[3]); }
            else {
              const uint16_t* const w = (const uint16_t*)q;
              x = make_uint4(w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16, w[4] | (uint32_t)w[5] << 16, w[6] | (uint32_t)w[7] << 16);
            }
            x.x ^= p.q_sign; x.y ^= p.q_sign; x.z ^= p.q_sign; x.w ^= p.q_sign;
          }
          *(uint4*)(q_s + piece_at<S::ROWS>(rr, jj)) = x;
        }
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        m[k] = -CUDART_INF_F; l[k] = 0.f;
        sight[k] = sight_of(p, now.s, row0 + part_of * 16 + (lane >> 2) + 8 * k);
      }
      bad = gave_up ? -2.f : 0.f;
      fresh = false;
      together();
    }
    // (a tile's page lookups are in flight while the one before is worked on)
    if (!gave_up) {
      load();
      look_up();
      gave_up = !__all_sync(0xffffffffu, mbar_wait_bounded(full + stage, parity, p.wait_limit));      // (one answer for the warp: it votes together in load())
    }
    if (gave_up) bad = -2.f;
    else if (bad_tiles >> (i & 31) & 1u) bad = bad == 0.f ? -1.f : bad;
    const uint32_t at_s = ring_a + stage * S::STAGE;
    char* const v_p = ring + stage * S::STAGE + S::HALF;
    const int x0 = tile_start<T>(now.s, now.t);
    const bool edge = !whole<T>(p, now.s, x0);
    bool wrote = false;
    if constexpr (TMA) {
      if (edge) {                  // values of positions that nothing sees: whatever lies there
        const int x = x0 + lane;
        const bool hidden = lane < T && !(x < now.s.n && (x >= now.s.lo || x < now.s.sk));
        if (__any_sync(0xffffffffu, hidden)) {
          if (part_of == 0 && hidden)
            for (int j = 0; j < PIECES; ++j) *(uint4*)(v_p + piece_at<T>(lane, j)) = make_uint4(0, 0, 0, 0);
          wrote = true;
          together();
        }
      }
    }
    // scores
    float s[NT][4];
#pragma unroll
    for (int e = 0; e < NT; ++e) s[e][0] = s[e][1] = s[e][2] = s[e][3] = 0.f;
    if constexpr (!F32) {
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        if (k * 16 >= p.in.D) break;
        uint32_t qf[4];
        ldm4(qf, pair_at<S::ROWS>(q_l, k));
#pragma unroll
        for (int e = 0; e < NT / 2; ++e) {
          uint32_t kf[4];
          ldm4(kf, pair_at<T>(at_s + k_l, k) + e * 2048);
          mma_bf16(s[2 * e], qf, kf[0], kf[1]);
          mma_bf16(s[2 * e + 1], qf, kf[2], kf[3]);
        }
      }
    } else {
      float s2[NT][4], s3[NT][4];  // the three products apart: chains a third as long, the small ones added first
#pragma unroll
      for (int e = 0; e < NT; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) s2[e][k] = s3[e][k] = 0.f;
#pragma unroll
      for (int k = 0; k < DP / 8; ++k) {
        if (k * 8 >= p.in.D) break;
        uint32_t q[4], qh[4], ql[4];
        if constexpr (!S::Q_REGS) ldm4(q, pair_at<S::ROWS>(q_l, k));
#pragma unroll
        for (int e = 0; e < 4; ++e) two_nearest(S::Q_REGS ? q_r[S::Q_REGS ? k : 0][e] : q[e], qh[e], ql[e]);
#pragma unroll
        for (int e = 0; e < NT; ++e) {
          uint32_t kf[2], kh[2], kl[2];
          ldm2(kf, pair_at<T>(at_s + k_l, k) + e * 1024);
          two_terms(kf[0], kh[0], kl[0]); two_terms(kf[1], kh[1], kl[1]);
          mma_tf32(s2[e], ql, kh[0], kh[1]);
          mma_tf32(s3[e], qh, kl[0], kl[1]);
          mma_tf32(s[e], qh, kh[0], kh[1]);
        }
      }
#pragma unroll
      for (int e = 0; e < NT; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[e][k] += s2[e][k] + s3[e][k];
    }
    // maxima, weights, sums
    {
      float top[2] = {-CUDART_INF_F, -CUDART_INF_F}, shift[2];
      if (edge)
#pragma unroll
        for (int e = 0; e < NT; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (!sight[k >> 1](x0 + e * 8 + (lane & 3) * 2 + (k & 1))) s[e][k] = -CUDART_INF_F;
#pragma unroll
      for (int e = 0; e < NT; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) top[k >> 1] = fmaxf(top[k >> 1], s[e][k]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
        top[k] = fmaxf(__fmul_rd(top[k], p.c), m[k]);          // (c > 0)
        shift[k] = top[k] == -CUDART_INF_F ? 0.f : top[k];
      }
      if (__any_sync(0xffffffffu, top[0] != m[0] || top[1] != m[1])) {
        const float a0 = ex2f(m[0] - shift[0]), a1 = ex2f(m[1] - shift[1]);
#pragma unroll
        for (int d = 0; d < ND; ++d) { o[d][0] *= a0; o[d][1] *= a0; o[d][2] *= a1; o[d][3] *= a1; }
        l[0] *= a0; l[1] *= a1;
        m[0] = top[0]; m[1] = top[1];
      }
#pragma unroll
      for (int e = 0; e < NT; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          s[e][k] = ex2f(cut_exponent(fmaf(s[e][k], p.c, -shift[k >> 1])));
          l[k >> 1] += s[e][k];
        }
    }
    // the weights times the values
    if (edge && p.in.Q > 1) {      // some rows do not see all of the tile: a value that is not finite must not reach those as 0 * inf
      bool strange = false;
      auto odd = [](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u || (!F32 && (w & 0x7f80u) == 0x7f80u); };
      for (int e = lane; e < T * PIECES; e += 32) {
        const uint4 x = *(const uint4*)(v_p + piece_at<T>(e / PIECES, e % PIECES));
        strange = strange || odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w);
      }
      strange = any_of_us(strange);        // (whatever a warp that has given up reads)
      if (strange) {               // it goes to the rows that see it by itself, and 0 takes its place
#pragma unroll 1
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const int col = d * 8 + (lane & 3) * 2;
            float2 v;
            if constexpr (F32) v = *(const float2*)(v_p + piece_at<T>(t, col >> 2) + (col & 3) * 4);
            else v = unpack_bf16x2(*(const uint32_t*)(v_p + piece_at<T>(t, d) + (lane & 3) * 4));
            v.x = fabsf(v.x) < CUDART_INF_F ? 0.f : v.x;
            v.y = fabsf(v.y) < CUDART_INF_F ? 0.f : v.y;
            if (sight[0](x0 + t)) { o[d][0] += v.x; o[d][1] += v.y; }
            if (sight[1](x0 + t)) { o[d][2] += v.x; o[d][3] += v.y; }
          }
        together();
        for (int e = part_of * 32 + lane; e < T * PIECES; e += 32 * NW) {
          uint4* const at = (uint4*)(v_p + piece_at<T>(e / PIECES, e % PIECES));
          auto clean = [](uint32_t w) {
            if constexpr (F32) return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
            else return ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) | ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu);
          };
          const uint4 x = *at;
          *at = make_uint4(clean(x.x), clean(x.y), clean(x.z), clean(x.w));
        }
        wrote = true;
        together();
      }
    }
    if constexpr (!F32) {
#pragma unroll
      for (int e = 0; e < NT / 2; ++e) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = s[2 * e + (k >> 1)][(k & 1) * 2], y = s[2 * e + (k >> 1)][(k & 1) * 2 + 1];
          hi[k] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);        // the upper halves; the rest is exact
          const float2 r = fadd2(make_float2(x, y), make_float2(-__uint_as_float(__float_as_uint(x) & 0xffff0000u), -__uint_as_float(__float_as_uint(y) & 0xffff0000u)));
          lo[k] = pack_bf16x2(r.x, r.y);
        }
#pragma unroll
        for (int d = 0; d < ND / 2; ++d) {
          if (d * 16 >= p.in.D) break;
          uint32_t vf[4];
          ldm4t(vf, pair_at<T>(at_s + v_l, d) + e * 2048);
          mma_bf16(o[2 * d], hi, vf[0], vf[1]);
          mma_bf16(o[2 * d + 1], hi, vf[2], vf[3]);
          mma_bf16(o[2 * d], lo, vf[0], vf[1]);
          mma_bf16(o[2 * d + 1], lo, vf[2], vf[3]);
        }
      }
    } else {
      // Index k of the product stands for position 2 k (k < 4) or 2 (k - 4) + 1: so the weights are where the scores were.  A tile's
      // products are summed apart and added to what is there: the tensor cores cut where they add, and over thousands of positions that would show.
      const int t0 = (lane & 3) * 2, dc = lane >> 2;
      uint32_t wh[NT][4], wl[NT][4];
#pragma unroll
      for (int e = 0; e < NT; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) two_nearest(__float_as_uint(s[e][(k & 1) * 2 + (k >> 1)]), wh[e][k], wl[e][k]);
      const uint32_t v_0 = (uint32_t)(t0 * 128 + (((dc >> 2) ^ t0) << 4)), v_1 = (uint32_t)((t0 + 1) * 128 + (((dc >> 2) ^ (t0 + 1)) << 4));
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        if (d * 8 >= p.in.D) break;
        float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < NT; ++e) {
          uint32_t vh[2], vl[2];
          two_terms(*(const uint32_t*)(v_p + pair_at<T>(v_0, d) + e * 1024 + (dc & 3) * 4), vh[0], vl[0]);
          two_terms(*(const uint32_t*)(v_p + pair_at<T>(v_1, d) + e * 1024 + (dc & 3) * 4), vh[1], vl[1]);
          mma_tf32(add, wl[e], vh[0], vh[1]);
          mma_tf32(add, wh[e], vl[0], vl[1]);
          mma_tf32(add, wh[e], vh[0], vh[1]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) o[d][k] += add[k];
      }
    }
    if (TMA && wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the stage is written by TMA next
    // the stage may be loaded again; the warps of a worker give up on the same segment (a word in shared memory, read behind the barrier, could be a faster warp's of the tile behind)
    if constexpr (NW > 1) {
      if (any_of_us(gave_up)) { gave_up = true; bad = -2.f; }
    } else together();
    if (now.t + 1 == now.s.nt || i + 1 == n_tiles) {        // the segment ends, or the piece does
      const bool head = i < now.t, tail = now.t + 1 < now.s.nt;      // it goes on from the piece before, or behind
      const uint32_t st = now.s.status | status_of(bad);
      float* const part = p.part + (number * 2 + (head ? 0 : 1)) * (int64_t)PART<S::ROWS, DP>;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float sum = l[k];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const int rr = part_of * 16 + (lane >> 2) + 8 * k, r = row0 + rr;
        if (r >= p.R) continue;
        if (head || tail) {
#pragma unroll
          for (int d = 0; d < ND; ++d) *(float2*)(part + rr * DP + d * 8 + (lane & 3) * 2) = make_float2(o[d][2 * k], o[d][2 * k + 1]);
          if ((lane & 3) == 0) *(float2*)(part + S::ROWS * DP + rr * 2) = make_float2(m[k], bad < 0.f ? bad : sum);
        } else {
          E* const out = (E*)p.out.out + out_at(p, now.b, h, r);
          const bool none = st || sum == 0.f;
          const float inv = none ? 0.f : 1.f / sum;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const int col = d * 8 + (lane & 3) * 2;
            if (col < p.in.D) {
              st_from_float(out, col, none ? 0.f : o[d][2 * k] * inv);
              st_from_float(out, col + 1, none ? 0.f : o[d][2 * k + 1] * inv);
            }
          }
          if ((lane & 3) == 0) put_lse(p, now.b, h, r, m[k], none ? 0.f : sum);
        }
      }
      if (part_of == 0 && lane == 0) {
        if (!head && now.hr == 0) put_status(p, now.b, tail ? now.s.status : st);
        if (bad == -2.f) { late.x = min(late.x, now.b); late.y = now.b; }
        if (i + 1 == n_tiles) {    // a segment that starts here and goes on: how many pieces behind have a share of it
          const long long end = u0 + i - now.t + now.s.nt;
          p.desc[number] = tail && !head ? make_int4(now.b, now.hr, (int)((end - 1) / chunk) - number, (int)now.s.status) : make_int4(0, 0, 0, 0);
        }
      }
      fresh = true;
    }
    now.next(p);
    if (++stage == ST) { stage = 0; parity ^= 1u; }
  }
  if (part_of == 0 && lane == 0) p.late[number] = late;
  if (gave_up)                     // copies that are still on their way land before the block's shared memory goes to another
    for (int i = max(0, loaded - ST); i < loaded; ++i) mbar_wait_bounded(full + i % ST, (uint32_t)(i / ST) & 1u);
}

// Joins the segments that several workers had a part of: block i the one that starts in piece i of the line.  `share` (1, 2, 4, 8) warps take a row's partials in
// turns, in the order of the line, and put theirs together warp by warp: the same sum every time.  (Eight warps for each row whatever the number of partials: 17 us where
// 1184 pieces had 5 rows, nine blocks of ten with nothing to do.)
template <typename E, int ROWS, int DP> __global__ void __launch_bounds__(256) attn_join_kernel(const __grid_constant__ AttnParams p, int share) {
  constexpr int PER = DP / 32;
  __shared__ float o_s[8][DP];
  __shared__ float2 ml_s[8];
  __shared__ uint32_t bad_s[8];
  wait_for_predecessor();
  launch_dependents();
  const int4 d = p.desc[blockIdx.x];
  if (blockIdx.y == 0) {
    const int2 late = p.late[blockIdx.x];
    if (late.x <= late.y)
      for (int b = late.x + (int)threadIdx.x; b <= late.y; b += 256) add_status(p, b, SAKI_ROW_TIMEOUT);
  }
  if (d.z == 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = d.y / p.RB, row0 = (d.y - h * p.RB) * ROWS;
  const int w0 = warp & ~(share - 1), mine = warp - w0, at_once = 8 / share;
  const int rows = min(ROWS, p.R - row0);
  for (int r0 = blockIdx.y * at_once; r0 < rows; r0 += gridDim.y * at_once) {
    const int rr = r0 + warp / share;
    const bool there = rr < rows;
    float m = -CUDART_INF_F, l = 0.f, o[PER];
    uint32_t bad = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) o[k] = 0.f;
    if (there) {
#pragma unroll 2
      for (int i = mine; i <= d.z; i += share) {
        const float* const part = p.part + ((blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * (int64_t)PART<ROWS, DP>;
        const float2 ml = *(const float2*)(part + ROWS * DP + rr * 2);
        bad |= status_of(ml.y);
        const float top = fmaxf(m, ml.x), sh = top == -CUDART_INF_F ? 0.f : top, a = ex2f(m - sh), c = ex2f(ml.x - sh);
#pragma unroll
        for (int k = 0; k < PER; ++k) o[k] = o[k] * a + part[rr * DP + k * 32 + lane] * c;
        l = l * a + ml.y * c;
        m = top;
      }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) o_s[warp][k * 32 + lane] = o[k];
    if (lane == 0) { ml_s[warp] = make_float2(m, l); bad_s[warp] = bad; }
    __syncthreads();
    if (there) {
      float top = -CUDART_INF_F;
      for (int w = w0; w < w0 + share; ++w) { bad |= bad_s[w]; top = fmaxf(top, ml_s[w].x); }
      const float sh = top == -CUDART_INF_F ? 0.f : top;
      float sum = 0.f;
      for (int w = w0; w < w0 + share; ++w) sum += ml_s[w].y * ex2f(ml_s[w].x - sh);
      const uint32_t st = (uint32_t)d.w | bad;
      const bool none = st || sum == 0.f;
      E* const out = (E*)p.out.out + out_at(p, d.x, h, row0 + rr);
      for (int k = mine * 32 + lane; k < p.in.D; k += 32 * share) {
        float x = 0.f;
        for (int w = w0; w < w0 + share; ++w) x += o_s[w][k] * ex2f(ml_s[w].x - sh);
        st_from_float(out, k, none ? 0.f : x / sum);
      }
      if (mine == 0 && lane == 0) {
        put_lse(p, d.x, h, row0 + rr, top, none ? 0.f : sum);
        if (rr == 0 && d.y == 0 && bad) add_status(p, d.x, bad);
      }
    }
    __syncthreads();
  }
}

constexpr int MAX_SMS = 148, MAX_WORKERS = 8 * MAX_SMS;  // of a call

struct Kernel { const void *tma, *plain; int rows, dp, t, smem, workers, threads; };
template <typename E, int DP, int NW> Kernel kernel() {
  using S = Shape<E, DP, NW>;
  const void* tma = nullptr;       // (bf16 heads of 65 to 128 with more rows, boxes and all, are for tcgen05)
  if constexpr (sizeof(E) == 4 || DP != 128 || NW == 1) tma = (const void*)attn_kernel<E, DP, NW, true>;
  return {tma, (const void*)attn_kernel<E, DP, NW, false>, S::ROWS, DP, S::T, S::SMEM, S::WORKERS, S::THREADS};
}
template <typename E, int DP> Kernel pick(int R) {
  if constexpr (DP == 256 && sizeof(E) == 4) return R <= 16 ? kernel<E, DP, 1>() : R <= 32 ? kernel<E, DP, 2>() : kernel<E, DP, 4>();
  else return R <= 16 ? kernel<E, DP, 1>() : R <= 32 ? kernel<E, DP, 2>() : R <= 64 ? kernel<E, DP, 4>() : kernel<E, DP, 8>();
}
template <typename E> Kernel pick(const saki_attn_in& in) {
  const int R = in.Q * (in.Hq / in.H);
  if constexpr (sizeof(E) == 4)
    if (in.D > 64 && in.D <= 96) return pick<E, 96>(R);      // (a ring of four tiles, not three)
  return in.D <= 64 ? pick<E, 64>(R) : in.D <= 128 ? pick<E, 128>(R) : pick<E, 256>(R);
}
Kernel pick(const saki_attn_in& in) { return in.dtype == SAKI_BF16 ? pick<__nv_bfloat16>(in) : pick<float>(in); }

template <typename E, int DP> cudaError_t join(const AttnParams& p, int rows, int workers, cudaStream_t st) {
  // a warp for some four partials: as many as a segment of average length has
  const int64_t partials = workers / std::max<int64_t>(1, p.in.B * p.in.H * p.RB) + 1;
  const int share = partials <= 4 ? 1 : partials <= 8 ? 2 : partials <= 16 ? 4 : 8, at_once = 8 / share;
  const dim3 grid((unsigned)workers, (unsigned)std::min((std::min(p.R, rows) + at_once - 1) / at_once, 16));
  if (rows == 16) return launch_pdl(attn_join_kernel<E, 16, DP>, grid, 256, 0, st, true, p, share);
  if (rows == 32) return launch_pdl(attn_join_kernel<E, 32, DP>, grid, 256, 0, st, true, p, share);
  if (rows == 64) return launch_pdl(attn_join_kernel<E, 64, DP>, grid, 256, 0, st, true, p, share);
  return launch_pdl(attn_join_kernel<E, 128, DP>, grid, 256, 0, st, true, p, share);
}
template <typename E> cudaError_t join(const AttnParams& p, const Kernel& k, int workers, cudaStream_t st) {
  if constexpr (sizeof(E) == 4)
    if (k.dp == 96) return join<E, 96>(p, k.rows, workers, st);
  return k.dp == 64 ? join<E, 64>(p, k.rows, workers, st) : k.dp == 128 ? join<E, 128>(p, k.rows, workers, st) : join<E, 256>(p, k.rows, workers, st);
}

// a pool [n_pages, page_size, H, D]: boxes of 128 bytes by `box` positions of one head and page, zeros behind D
bool pool_map(CUtensorMap* map, const void* pool, int64_t page, int64_t pos, int64_t head, const saki_attn_in& in, int box) {
  const EncodeTiledFn fn = encode_fn();
  const int64_t size = in.dtype == SAKI_BF16 ? 2 : 4, row = (in.D * size + 15) & ~15ll;
  auto step = [&](int64_t s, int64_t n) { return (cuuint64_t)(n > 1 ? s * size : row); };      // (of a dimension of one: never used)
  const cuuint64_t dims[4] = {(cuuint64_t)in.D, (cuuint64_t)in.H, (cuuint64_t)in.page_size, (cuuint64_t)in.n_pages};
  const cuuint64_t strides[3] = {step(head, in.H), step(pos, in.page_size), step(page, in.n_pages)};
  const cuuint32_t boxes[4] = {(cuuint32_t)(128 / size), 1, (cuuint32_t)box, 1}, one[4] = {1, 1, 1, 1};
  return fn && fn(map, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, const_cast<void*>(pool), dims, strides, boxes, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ... as `mode` sees it (bf16, D = 128)
bool eights_map(CUtensorMap* map, const void* pool, int64_t page, int64_t pos, int64_t head, const saki_attn_in& in, int box, int mode) {
  const EncodeTiledFn fn = encode_fn();
  const cuuint64_t eights = (cuuint64_t)in.page_size / 8, pages = (cuuint64_t)in.n_pages, H = (cuuint64_t)in.H;
  auto step = [](int64_t s, cuuint64_t n) { return (cuuint64_t)(n > 1 ? s * 2 : 256); };      // (of a dimension of one: never used)
  const cuuint64_t c4 = mode == MAP_HEADS ? pages : mode == MAP_PAGES ? pages * H : H;
  const cuuint64_t dims[5] = {64, 8, mode == MAP_HEADS ? 2 * H : 2, mode == MAP_RUN ? eights * pages : eights, c4};
  const cuuint64_t strides[4] = {step(pos, 8), 128, step(8 * pos, dims[3]), step(mode == MAP_HEADS ? page : head, c4)};
  const cuuint32_t boxes[5] = {64, 8, 2, (cuuint32_t)(box / 8), 1}, one[5] = {1, 1, 1, 1, 1};
  if (!fn || dims[3] >= (1ull << 31) || c4 >= (1ull << 31)) return false;
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(pool), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// whether what `mode` takes for granted holds for a pool
bool mode_fits(int mode, int64_t page, int64_t pos, int64_t head, const saki_attn_in& in) {
  if (mode == MAP_HEADS) return in.H == 1 || head == 128;
  if (mode == MAP_PAGES) return in.H > 1 && (in.n_pages == 1 || page == in.H * head);
  return in.n_pages == 1 || page == in.page_size * pos;
}

}  // namespace

// bf16 heads of up to 128 on pages of whole eights go to the kernel on tcgen05, but for single tokens of up to 16 rows where its tiles of 128 positions cost more than they
// bring.  (us here and there, 8 key heads, pages of 16 positions.)
//  - Heads of up to 64: 96 sequences of 8000 positions, 5 rows 328 and 420, 16 rows 335 and 421; of 2000 98 and 130, 105 and 133; of 1000 60 and 83, 68 and 85.  (With the heads of a position
//    side by side the longest are alike: 418 and 418, 432 and 419; of 1000 75 and 85.)  But two tokens of 8 rows, 4000 positions: 261 and 237.
//  - Where nothing can see more than 256 positions: heads of 128, 512 sequences of 128 positions, 4 rows 83 and 104, 16 rows 111 and 109; of 256 139 and 156, 167 and 161; of 512 251 and 208.
//    What a query can see goes by the table's width: lengths are known on the device only.  (512 sequences of 128 positions in wide tables take the 104.)
static bool on_umma(const saki_attn_in& in) {
  if (in.dtype != SAKI_BF16 || in.D <= 16 || in.D > 128 || in.page_size % 8 != 0) return false;
  const int64_t table = (int64_t)in.max_pages * in.page_size, seen = in.window > 0 ? std::min<int64_t>(table, (int64_t)in.window + in.sinks) : table;
  return in.Q > 1 || in.Hq / in.H > 16 || (in.D > 64 && seen > 256);
}

int64_t attention_scratch_bytes(const saki_attn_in& in) {
  // (a block on each SM; where tcgen05 serves the call the other kernel still has to find room, should the tensor maps be refused)
  const Kernel k = pick(in);
  int64_t rows = (int64_t)k.workers * k.rows;      // with partial results, of a block
  if (on_umma(in)) rows = std::max<int64_t>(rows, umma_rows(in));
  return MAX_WORKERS * 24 + MAX_SMS * 2 * rows * (k.dp + 2) * 4;
}

cudaError_t launch_attention(const saki_attn_in& in, const saki_attn_out& out, void* scratch, unsigned long long* flagged, long long wait_limit,
                             int* n_launches, cudaStream_t st) {
  AttnParams p = {};
  p.in = in; p.out = out; p.flagged = flagged;
  p.wait_limit = wait_limit > 0 ? wait_limit : WAIT_LIMIT_CYCLES;
  p.G = in.Hq / in.H; p.R = in.Q * p.G;
  p.c = std::max(std::fabs(in.scale) * 1.4426950408889634f, 1e-37f);      // (scale 0: what is not seen has the score -inf, also times c)
  p.q_sign = in.scale < 0.f ? in.dtype == SAKI_BF16 ? 0x80008000u : 0x80000000u : 0u;
  p.page_shift = -1;
  for (int k = 0; k < 31; ++k)
    if (in.page_size == 1 << k) p.page_shift = k;
  const int size = in.dtype == SAKI_BF16 ? 2 : 4;
  p.q_vec = ((uintptr_t)in.q | (uintptr_t)(in.q_seq * size) | (uintptr_t)(in.q_pos * size) | (uintptr_t)(in.q_head * size)) % 16 == 0;
  p.desc = (int4*)scratch;
  p.late = (int2*)((char*)scratch + MAX_WORKERS * 16);
  p.part = (float*)((char*)scratch + MAX_WORKERS * 24);
  Kernel k = pick(in);
  bool umma = on_umma(in);
  // Boxes: as many positions of a page as a tile takes.  A page that is no multiple of eight, or strides that the map does not take
  // (2^40 bytes), go through the plain loads.
  p.box = 1;
  while (p.box < (umma ? UMMA_T : k.t) && in.page_size % (2 * p.box) == 0) p.box *= 2;
  CUtensorMap k_map = {}, v_map = {};
  const bool tma = p.box >= 8 && pool_map(&k_map, in.k_pages, in.kp_page, in.kp_pos, in.kp_head, in, p.box) &&
                   pool_map(&v_map, in.v_pages, in.vp_page, in.vp_pos, in.vp_head, in, p.box);
  umma = umma && tma;
  for (int mode = MAP_HEADS; umma && in.D == 128 && mode <= MAP_RUN && p.map_mode == MAP_BOXES; ++mode) {
    CUtensorMap k5 = {}, v5 = {};
    if (mode_fits(mode, in.kp_page, in.kp_pos, in.kp_head, in) && mode_fits(mode, in.vp_page, in.vp_pos, in.vp_head, in) &&
        eights_map(&k5, in.k_pages, in.kp_page, in.kp_pos, in.kp_head, in, p.box, mode) && eights_map(&v5, in.v_pages, in.vp_page, in.vp_pos, in.vp_head, in, p.box, mode)) {
      k_map = k5; v_map = v5; p.map_mode = mode;
    }
  }
  int dev = 0, sms = MAX_SMS, workers = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  sms = std::min(sms, MAX_SMS);
  if (umma) { k.rows = umma_rows(in); k.t = UMMA_T; }
  p.RB = (p.R + k.rows - 1) / k.rows;
  const int64_t most = in.B * in.H * p.RB * (((int64_t)in.max_pages * in.page_size + k.t - 1) / k.t);      // tiles, if every table were full
  if (umma) {
    workers = (int)std::min<int64_t>(most, sms);
    e = launch_umma(p, k_map, v_map, workers, st);
  } else {
    const void* const fn = tma ? k.tma : k.plain;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem);
    if (e != cudaSuccess) return e;
    const int blocks = (int)std::min<int64_t>(most, sms);
    workers = blocks * k.workers;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3((unsigned)k.threads); cfg.dynamicSmemBytes = (size_t)k.smem; cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    void* args[] = {&p, &k_map, &v_map};
    e = cudaLaunchKernelExC(&cfg, fn, args);
  }
  if (e != cudaSuccess) return e;
  ++*n_launches;
  e = in.dtype == SAKI_BF16 ? join<__nv_bfloat16>(p, k, workers, st) : join<float>(p, k, workers, st);
  if (e == cudaSuccess) ++*n_launches;
  return e;
}

}  // namespace saki
