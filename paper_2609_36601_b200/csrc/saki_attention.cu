// Attention of a few new tokens per sequence over a paged key-value cache.
//
// Every key and value is read once and meets G * Q query rows (G query heads share a key head, Q new tokens), so up to some 60
// rows the call is bound by HBM.  The work is therefore laid out by what is read: the visible positions of all sequences, key heads and row
// blocks, in tiles of T positions, form one line of tiles that is cut into equal pieces, one per thread block, whatever the lengths are
// (they are known on the device only).  A block runs along its piece with a ring of tiles in flight (cp.async), which runs
// ahead across the ends of sequences, and keeps each row's running maximum, sum and weighted values in registers.  Where a cut falls inside
// a sequence the two sides leave partial results in scratch, which a second small kernel joins in the order of the line.
//
//   s = scale * q.k,   m' = max(m, s),   l = l 2^(m - m') + 2^(s - m'),   o = o 2^(m - m') + 2^(s - m') v       (s, m in units of log 2)
//
// bf16: mma.sync m16n8k16 with float32 accumulators, a warp per 16 rows and 64 / (4 / row groups) positions.  The weights go into the second product as
// two bf16 terms, so that they carry 16 bits: one term would add an error as large as the rounding of the output (2^-9 each), and the second
// product is not what bounds the kernel.  f32: products on the FMA pipes.
#include "saki_device.cuh"
#include <algorithm>

namespace saki {

namespace {

constexpr int AT = 128;                       // threads of a block

struct AttnParams {
  saki_attn_in in;
  saki_attn_out out;
  int G, R, RB;             // query heads per key head; rows of a key head (Q * G); blocks of rows
  int q_vec;                // q can be read in 16-byte pieces
  float c;                  // scale * log2(e)
  int4* desc;               // [blocks] the segment that starts in a block and goes on: (b, head and row block, blocks behind, status)
  float* part;              // [blocks][2] partial results: of the segment that goes on from the block before, of the one that goes on behind
  unsigned long long* flagged;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool real) {      // zeros where not real
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What the queries of a sequence see, in tiles of T positions: the tiles of the first `sk` positions, then those from tile m0 on.
struct Span {
  int n, p0, nq, lo, sk, ns, m0, nt;
  uint32_t status;
};
template <int T> __device__ __forceinline__ Span span_of(const AttnParams& p, int64_t b) {
  Span s;
  s.n = p.in.length[b];
  s.nq = p.in.n_query ? p.in.n_query[b] : p.in.Q;
  s.status = 0;
  if (s.n < 0 || (int64_t)s.n > (int64_t)p.in.max_pages * p.in.page_size || s.nq < 0 || s.nq > p.in.Q) { s.status = SAKI_ROW_BAD_LENGTH; s.n = 0; s.nq = 0; }
  s.p0 = s.n - s.nq;
  s.lo = p.in.window > 0 ? (int)max((int64_t)0, (int64_t)s.p0 - p.in.window + 1) : 0;
  if (s.nq == 0) s.lo = s.n;
  s.sk = s.nq == 0 ? 0 : min(p.in.sinks, s.lo);
  s.ns = (s.sk + T - 1) / T;
  s.m0 = max(s.lo / T, s.ns);
  s.nt = max(1, s.ns + max(0, (int)(((int64_t)s.n + T - 1) / T) - s.m0));
  return s;
}
template <int T> __device__ __forceinline__ int64_t tile_start(const Span& s, int t) { return (int64_t)(t < s.ns ? t : s.m0 + t - s.ns) * T; }

// A place on the line of tiles: sequence, key head and row block, tile.
template <int T> struct Cursor {
  int64_t b;
  int hr, t;
  Span s;
  __device__ __forceinline__ void at(const AttnParams& p, int64_t b_, int64_t offset) {
    b = b_;
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

struct LineShared {
  long long sum[AT / 32];
  long long b, before;      // the sequence of the block's first tile, tiles in front of it
};
// The block's piece [u0, u1) of the line, and the cursor at its start.  Every block adds up all sequences' tiles (a few
// per thread).  false: nothing is left for the block.
template <int T> __device__ __forceinline__ bool piece(const AttnParams& p, LineShared& sh, long long& u0, long long& u1, long long& chunk, Cursor<T>& c) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t per = (p.in.B + AT - 1) / AT, b0 = min((int64_t)tid * per, p.in.B), b1 = min(b0 + per, p.in.B);
  const int each = p.in.H * p.RB;
  long long mine = 0;
  for (int64_t b = b0; b < b1; ++b) mine += (long long)span_of<T>(p, b).nt * each;
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh.sum[warp] = upto;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < AT / 32; ++w) {
    if (w < warp) upto += sh.sum[w];
    total += sh.sum[w];
  }
  chunk = max(1ll, (total + gridDim.x - 1) / gridDim.x);
  u0 = blockIdx.x * chunk;
  u1 = min(u0 + chunk, total);
  if (u0 >= total) return false;
  if (upto - mine <= u0 && u0 < upto) {
    long long at = upto - mine;
    int64_t b = b0;
    for (;; ++b) {
      const long long n = (long long)span_of<T>(p, b).nt * each;
      if (u0 < at + n) break;
      at += n;
    }
    sh.b = b; sh.before = at;
  }
  __syncthreads();
  c.at(p, sh.b, u0 - sh.before);
  return true;
}

// Where in the pools the positions of a tile lie: element offsets, -1 for positions that nothing sees, or without a page.
template <int T> struct Rows {
  int64_t k[T], v[T];
  int bad[(T + 31) / 32];        // a page id outside the pool, by warp
};
struct Found { int id; int64_t x; bool seen; };
template <int T> __device__ __forceinline__ Found find_row(const AttnParams& p, const Cursor<T>& c) {      // threads 0 .. T - 1: the page of their position
  Found f;
  f.x = tile_start<T>(c.s, c.t) + threadIdx.x;
  f.seen = f.x < c.s.n && (f.x >= c.s.lo || f.x < c.s.sk);
  f.id = f.seen ? p.in.page_table[c.b * p.in.ld_table + f.x / p.in.page_size] : 0;
  return f;
}
template <int T> __device__ __forceinline__ void put_row(const AttnParams& p, const Found& f, int head, Rows<T>& to) {
  const bool bad = f.seen && (unsigned)f.id >= (unsigned)p.in.n_pages;
  const int slot = (int)(f.x % p.in.page_size);
  to.k[threadIdx.x] = f.seen && !bad ? f.id * p.in.kp_page + slot * p.in.kp_pos + head * p.in.kp_head : -1;
  to.v[threadIdx.x] = f.seen && !bad ? f.id * p.in.vp_page + slot * p.in.vp_pos + head * p.in.vp_head : -1;
  const bool any = __any_sync(0xffffffffu, bad);
  if ((threadIdx.x & 31) == 0) to.bad[threadIdx.x >> 5] = any;
}
// A row of keys or values in shared memory: 16-byte pieces, piece j of row r at place j ^ (r & 7), so that eight rows' pieces of one
// column lie in different banks.
template <typename E, int DP> __device__ __forceinline__ uint32_t piece_at(int row, int j) { return (uint32_t)(row * DP * (int)sizeof(E) + ((j ^ (row & 7)) << 4)); }

template <typename E, int DP, int T> __device__ __forceinline__ void load_tile(const AttnParams& p, const Rows<T>& rows, uint32_t k_s, uint32_t v_s) {
  constexpr int PE = 16 / (int)sizeof(E), PIECES = DP / PE, STEP = AT / PIECES;      // rows of a pass over the threads
  static_assert(AT % PIECES == 0, "a pass covers whole rows");
  const int j = threadIdx.x % PIECES, r0 = threadIdx.x / PIECES;
  if (j * PE >= p.in.D) return;
#pragma unroll 4
  for (int r = r0; r < T; r += STEP) {
    const int64_t k = rows.k[r], v = rows.v[r];
    cp16(k_s + piece_at<E, DP>(r, j), (const E*)p.in.k_pages + (k < 0 ? 0 : k + j * PE), k >= 0);
    cp16(v_s + piece_at<E, DP>(r, j), (const E*)p.in.v_pages + (v < 0 ? 0 : v + j * PE), v >= 0);
  }
}

__device__ __forceinline__ int64_t out_at(const AttnParams& p, int64_t b, int h, int r) {
  const int j = r / p.G;
  return b * p.out.o_seq + j * p.out.o_pos + (int64_t)(h * p.G + r - j * p.G) * p.out.o_head;
}
__device__ __forceinline__ void put_lse(const AttnParams& p, int64_t b, int h, int r, float m, float l) {
  if (!p.out.lse) return;
  const int j = r / p.G;
  p.out.lse[(b * p.in.Q + j) * p.in.Hq + h * p.G + r - j * p.G] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
}
__device__ __forceinline__ void put_status(const AttnParams& p, int64_t b, uint32_t st) {
  if (p.out.row_status) p.out.row_status[b] = st;
  if (st) atomicAdd(p.flagged, 1ull);
}

// Segments (sequence, key head, row block) that several blocks worked on: ROWS rows of DP values, then ROWS pairs (m, l); l < 0: a bad page.
template <int ROWS, int DP> constexpr int PART = ROWS * (DP + 2);

// what a row sees: positions up to `to`, from `from` on or below `first`
struct Sight {
  int to, from, first;
  __device__ __forceinline__ bool operator()(int64_t x) const { return x <= to && (x >= from || x < first); }
};
__device__ __forceinline__ Sight sight_of(const AttnParams& p, const Span& s, int r) {      // r: row within the key head
  const int j = r / p.G;
  if (r >= p.R || j >= s.nq) return {-1, 0, 0};
  const int at = s.p0 + j;
  return {at, p.in.window > 0 ? (int)max((int64_t)0, (int64_t)at - p.in.window + 1) : 0, p.in.window > 0 ? p.in.sinks : 0};
}
// all rows see all of a tile's positions
template <int T> __device__ __forceinline__ bool whole(const AttnParams& p, const Span& s, int64_t x0) {
  return s.nq == p.in.Q && x0 + T - 1 <= s.p0 && (p.in.window <= 0 || x0 > (int64_t)s.n - 1 - p.in.window || x0 + T <= s.sk);
}

// ---- bf16 ----

template <int DP, int MT> struct MmaShape {
  static constexpr int T = 64, WM = MT, WN = 4 / MT, TW = T / WN, ROWS = 16 * MT;      // positions of a tile; groups of rows and of positions; positions of a warp
  static constexpr int TILE = T * DP * 2;
  static constexpr int STAGES = DP <= 128 ? 3 : 2;
  static constexpr bool Q_REGS = DP <= 128;          // the queries stay in registers
  static constexpr int SMEM = STAGES * 2 * TILE + ROWS * DP * 2 + (WN > 1 ? WM * DP * 16 * 4 + 4 * 16 * 2 * 4 : 0) + (STAGES + 1) * (int)sizeof(Rows<T>) + (int)sizeof(LineShared);
};

template <int DP, int MT> __global__ void __launch_bounds__(AT) attn_mma_kernel(const __grid_constant__ AttnParams p) {
  using S = MmaShape<DP, MT>;
  constexpr int T = S::T, ST = S::STAGES, TW = S::TW, WN = S::WN, KD = DP / 16, ND = DP / 8;
  using E = __nv_bfloat16;
  extern __shared__ __align__(128) char smem[];
  char* at = smem + ST * 2 * S::TILE;
  E* const q_s = (E*)at; at += S::ROWS * DP * 2;
  float* const o_s = (float*)at; if (WN > 1) at += S::WM * DP * 16 * 4;
  float2* const ml_s = (float2*)at; if (WN > 1) at += 4 * 16 * 2 * 4;
  Rows<T>* const rows = (Rows<T>*)at; at += (ST + 1) * sizeof(Rows<T>);
  LineShared& line = *(LineShared*)at;
  const uint32_t tiles = smem_addr(smem), q_a = smem_addr(q_s);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % S::WM, wn = warp / S::WM;

  // columns behind D stay zero
  for (int i = tid; i < ST * 2 * T * (DP / 8); i += AT) {
    const int r = i / (DP / 8), j = i % (DP / 8);
    if (j * 8 >= p.in.D) *(uint4*)(smem + r / T * S::TILE + piece_at<E, DP>(r % T, j)) = make_uint4(0, 0, 0, 0);
  }
  wait_for_predecessor();
  launch_dependents();
  long long u0, u1, chunk;
  Cursor<T> now;
  if (!piece<T>(p, line, u0, u1, chunk, now)) {
    if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  // the ring: tile u lies in stage (u - u0) % ST; where its positions lie is looked up a tile ahead of the loads
  Cursor<T> look = now;
  long long looked = u0, loaded = u0;
  auto look_up = [&] {
    if (looked < u1) {
      if (tid < T) put_row<T>(p, find_row<T>(p, look), look.hr / p.RB, rows[looked % (ST + 1)]);
      look.next(p);
      ++looked;
    }
  };
  auto load = [&] {
    if (loaded < u1) {
      const uint32_t k = tiles + (uint32_t)((loaded - u0) % ST) * (2 * S::TILE);
      load_tile<E, DP, T>(p, rows[loaded % (ST + 1)], k, k + S::TILE);
      ++loaded;
    }
    cp_commit();
  };
#pragma unroll 1
  for (int i = 0; i < ST - 1; ++i) {
    look_up();
    __syncthreads();
    load();
  }
  look_up();

  float o[ND][4], m[2], l[2];
  uint32_t qf[S::Q_REGS ? KD : 1][4];
  Sight sight[2];
  uint32_t bad = 0;
  bool fresh = true;
  const uint32_t q_row = (uint32_t)(wm * 16 + ((lane >> 3) & 1) * 8 + (lane & 7));
#pragma unroll 1
  for (long long u = u0; u < u1; ++u) {
    const int h = now.hr / p.RB, row0 = (now.hr - h * p.RB) * S::ROWS;
    if (fresh) {                    // a new segment: its queries
      for (int i = tid; i < S::ROWS * (DP / 8); i += AT) {
        const int rr = i / (DP / 8), j8 = i % (DP / 8), r = row0 + rr, j = r / p.G;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r < p.R && j8 * 8 < p.in.D) {
          const E* const q = (const E*)p.in.q + now.b * p.in.q_seq + j * p.in.q_pos + (int64_t)(h * p.G + r - j * p.G) * p.in.q_head + j8 * 8;
          if (p.q_vec) x = *(const uint4*)q;
          else {
            const uint16_t* const e = (const uint16_t*)q;
            x.x = e[0] | (uint32_t)e[1] << 16; x.y = e[2] | (uint32_t)e[3] << 16; x.z = e[4] | (uint32_t)e[5] << 16; x.w = e[6] | (uint32_t)e[7] << 16;
          }
        }
        *(uint4*)((char*)q_s + piece_at<E, DP>(rr, j8)) = x;
      }
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
      m[0] = m[1] = -CUDART_INF_F; l[0] = l[1] = 0.f;
      sight[0] = sight_of(p, now.s, row0 + wm * 16 + (lane >> 2));
      sight[1] = sight_of(p, now.s, row0 + wm * 16 + (lane >> 2) + 8);
      bad = 0;
    }
    cp_wait<ST - 2>();
    __syncthreads();
    if (fresh) {
      if constexpr (S::Q_REGS) {
#pragma unroll
        for (int k = 0; k < KD; ++k) ldm4(qf[k], q_a + piece_at<E, DP>(q_row, k * 2 + (lane >> 4)));
      }
      fresh = false;
    }
    load();
    Found ahead = {};
    const bool finding = looked < u1;
    if (finding && tid < T) ahead = find_row<T>(p, look);
    // scores of the warp's positions
    const uint32_t k_s = tiles + (uint32_t)((u - u0) % ST) * (2 * S::TILE), v_s = k_s + S::TILE;
    const int first = wn * TW;
    float s[TW / 8][4];
#pragma unroll
    for (int i = 0; i < TW / 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
    {
      const int mi = lane >> 3, tok = (mi >> 1) * 8 + (lane & 7);
#pragma unroll
      for (int k = 0; k < KD; ++k) {
        if constexpr (!S::Q_REGS) ldm4(qf[0], q_a + piece_at<E, DP>(q_row, k * 2 + (lane >> 4)));
#pragma unroll
        for (int i = 0; i < TW / 16; ++i) {
          uint32_t kf[4];
          ldm4(kf, k_s + piece_at<E, DP>(first + i * 16 + tok, k * 2 + (mi & 1)));
          mma(s[2 * i], qf[S::Q_REGS ? k : 0], kf[0], kf[1]);
          mma(s[2 * i + 1], qf[S::Q_REGS ? k : 0], kf[2], kf[3]);
        }
      }
    }
    const int64_t x0 = tile_start<T>(now.s, now.t);
    const bool edge = !whole<T>(p, now.s, x0);
    const Rows<T>& here = rows[u % (ST + 1)];
#pragma unroll
    for (int i = 0; i < (T + 31) / 32; ++i) bad |= here.bad[i];
    float top[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
    for (int i = 0; i < TW / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[i][k] *= p.c;
        if (edge && !sight[k >> 1](x0 + first + i * 8 + (lane & 3) * 2 + (k & 1))) s[i][k] = -CUDART_INF_F;
        top[k >> 1] = fmaxf(top[k >> 1], s[i][k]);
      }
    float shift[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
      top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
      top[k] = fmaxf(top[k], m[k]);
      shift[k] = top[k] == -CUDART_INF_F ? 0.f : top[k];
    }
    if (__any_sync(0xffffffffu, top[0] != m[0] || top[1] != m[1])) {
      const float a0 = ex2f(m[0] - shift[0]), a1 = ex2f(m[1] - shift[1]);
#pragma unroll
      for (int i = 0; i < ND; ++i) { o[i][0] *= a0; o[i][1] *= a0; o[i][2] *= a1; o[i][3] *= a1; }
      l[0] *= a0; l[1] *= a1;
      m[0] = top[0]; m[1] = top[1];
    }
#pragma unroll
    for (int i = 0; i < TW / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[i][k] = ex2f(s[i][k] - shift[k >> 1]);
        l[k >> 1] += s[i][k];
      }
    // the weights times the values
    bool strange = false;            // a value that is not finite, in a tile that some rows do not see all of
    if (edge && p.in.Q > 1) {
      for (int i = lane; i < TW * (DP / 8); i += 32) {
        const uint4 x = *(const uint4*)(smem + (v_s - tiles) + piece_at<E, DP>(first + i / (DP / 8), i % (DP / 8)));
        for (const uint32_t w : {x.x, x.y, x.z, x.w}) strange = strange || (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
      }
      strange = __any_sync(0xffffffffu, strange);
    }
    if (!strange) {
      const int mi = lane >> 3, tok = (mi & 1) * 8 + (lane & 7);
#pragma unroll
      for (int i = 0; i < TW / 16; ++i) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = s[2 * i + (k >> 1)][(k & 1) * 2], y = s[2 * i + (k >> 1)][(k & 1) * 2 + 1];
          hi[k] = pack_bf16x2(x, y);
          const float2 r = unpack_bf16x2(hi[k]);
          lo[k] = pack_bf16x2(x - r.x, y - r.y);
        }
#pragma unroll
        for (int d = 0; d < ND / 2; ++d) {
          uint32_t vf[4];
          ldm4t(vf, v_s + piece_at<E, DP>(first + i * 16 + tok, d * 2 + (mi >> 1)));
          mma(o[2 * d], hi, vf[0], vf[1]);
          mma(o[2 * d + 1], hi, vf[2], vf[3]);
          mma(o[2 * d], lo, vf[0], vf[1]);
          mma(o[2 * d + 1], lo, vf[2], vf[3]);
        }
      }
    } else {                         // one position at a time: what a row does not see must not reach it as 0 * inf
#pragma unroll
      for (int i = 0; i < TW / 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w0 = __shfl_sync(0xffffffffu, s[i][e & 1], (lane & ~3) | (e >> 1)), w1 = __shfl_sync(0xffffffffu, s[i][2 + (e & 1)], (lane & ~3) | (e >> 1));
          const int64_t x = x0 + first + i * 8 + e;
          const bool y0 = sight[0](x), y1 = sight[1](x);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const float2 v = unpack_bf16x2(*(const uint32_t*)(smem + (v_s - tiles) + piece_at<E, DP>(first + i * 8 + e, d) + (lane & 3) * 4));
            if (y0) { o[d][0] += w0 * v.x; o[d][1] += w0 * v.y; }
            if (y1) { o[d][2] += w1 * v.x; o[d][3] += w1 * v.y; }
          }
        }
    }
    if (finding) {
      if (tid < T) put_row<T>(p, ahead, look.hr / p.RB, rows[looked % (ST + 1)]);
      look.next(p);
      ++looked;
    }
    if (now.t + 1 == now.s.nt || u + 1 == u1) {        // the segment ends, or the piece does
      const bool head = u - now.t < u0, tail = now.t + 1 < now.s.nt;      // it goes on from the block before, or behind
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
      }
      if constexpr (WN > 1) {        // the warps that share the rows
        if ((lane & 3) == 0) {
          ml_s[warp * 16 + (lane >> 2)] = make_float2(m[0], l[0]);
          ml_s[warp * 16 + (lane >> 2) + 8] = make_float2(m[1], l[1]);
        }
        __syncthreads();
        float a[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float own = m[k];
          float best = -CUDART_INF_F, sum = 0.f;
#pragma unroll
          for (int w = 0; w < WN; ++w) best = fmaxf(best, ml_s[(w * S::WM + wm) * 16 + (lane >> 2) + 8 * k].x);
          const float sh = best == -CUDART_INF_F ? 0.f : best;
#pragma unroll
          for (int w = 0; w < WN; ++w) {
            const float2 ml = ml_s[(w * S::WM + wm) * 16 + (lane >> 2) + 8 * k];
            sum += ml.y * ex2f(ml.x - sh);
          }
          a[k] = ex2f(own - sh);
          m[k] = best; l[k] = sum;
        }
#pragma unroll
        for (int i = 0; i < ND; ++i) { o[i][0] *= a[0]; o[i][1] *= a[0]; o[i][2] *= a[1]; o[i][3] *= a[1]; }
#pragma unroll
        for (int w = WN - 1; w >= 0; --w) {
          if (wn == w) {
            float4* const at4 = (float4*)o_s + wm * ND * 32 + lane;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
              if (w < WN - 1) {
                const float4 x = at4[i * 32];
                o[i][0] += x.x; o[i][1] += x.y; o[i][2] += x.z; o[i][3] += x.w;
              }
              if (w > 0) at4[i * 32] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
            }
          }
          if (w > 0) __syncthreads();
        }
      }
      const uint32_t st = now.s.status | (bad ? SAKI_ROW_BAD_PAGE : 0u);
      if (wn == 0) {
        float* const part = p.part + (blockIdx.x * 2 + (head ? 0 : 1)) * (int64_t)PART<S::ROWS, DP>;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int rr = wm * 16 + (lane >> 2) + 8 * k, r = row0 + rr;
          if (r >= p.R) continue;
          if (head || tail) {
#pragma unroll
            for (int i = 0; i < ND; ++i) *(float2*)(part + rr * DP + i * 8 + (lane & 3) * 2) = make_float2(o[i][2 * k], o[i][2 * k + 1]);
            if ((lane & 3) == 0) *(float2*)(part + S::ROWS * DP + rr * 2) = make_float2(m[k], bad ? -1.f : l[k]);
          } else {
            E* const out = (E*)p.out.out + out_at(p, now.b, h, r);
            const bool none = st || l[k] == 0.f;
            const float inv = none ? 0.f : 1.f / l[k];
#pragma unroll
            for (int i = 0; i < ND; ++i) {
              const int d = i * 8 + (lane & 3) * 2;
              if (d < p.in.D) {
                out[d] = __float2bfloat16_rn(none ? 0.f : o[i][2 * k] * inv);
                out[d + 1] = __float2bfloat16_rn(none ? 0.f : o[i][2 * k + 1] * inv);
              }
            }
            if ((lane & 3) == 0) put_lse(p, now.b, h, r, m[k], none ? 0.f : l[k]);
          }
        }
      }
      if (!head && !tail && now.hr == 0 && tid == 0) put_status(p, now.b, st);
      if (u + 1 == u1 && tid == 0) {       // a segment that starts here and goes on: how many blocks behind have a share of it
        const long long end = u - now.t + now.s.nt;
        p.desc[blockIdx.x] = tail && !head ? make_int4((int)now.b, now.hr, (int)((end - 1) / chunk) - (int)blockIdx.x, (int)now.s.status) : make_int4(0, 0, 0, 0);
      }
      fresh = true;
      __syncthreads();                // the queries in shared memory, and what the warps exchanged, make room for the next segment's
    }
    now.next(p);
  }
  cp_wait<0>();
}

// Joins the segments that several blocks worked on: block i the one that starts in block i of the kernel above.  A row at a time, the partials
// spread over the warps (in the order of the line within a warp, then warp by warp: the same sum every time).
template <typename E, int ROWS, int DP> __global__ void __launch_bounds__(256) attn_join_kernel(const __grid_constant__ AttnParams p) {
  constexpr int PER = DP / 32;
  __shared__ float o_s[8][DP];
  __shared__ float2 ml_s[8];
  wait_for_predecessor();
  launch_dependents();
  const int4 d = p.desc[blockIdx.x];
  if (d.z == 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = d.y / p.RB, row0 = (d.y - h * p.RB) * ROWS;
  for (int rr = blockIdx.y; rr < ROWS && row0 + rr < p.R; rr += gridDim.y) {
    float m = -CUDART_INF_F, l = 0.f, o[PER];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) o[k] = 0.f;
    for (int i = warp; i <= d.z; i += 8) {
      const float* const part = p.part + ((blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * (int64_t)PART<ROWS, DP>;
      const float2 ml = *(const float2*)(part + ROWS * DP + rr * 2);
      bad = bad || ml.y < 0.f;
      const float top = fmaxf(m, ml.x), sh = top == -CUDART_INF_F ? 0.f : top, a = ex2f(m - sh), c = ex2f(ml.x - sh);
#pragma unroll
      for (int k = 0; k < PER; ++k) o[k] = o[k] * a + part[rr * DP + k * 32 + lane] * c;
      l = l * a + ml.y * c;
      m = top;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) o_s[warp][k * 32 + lane] = o[k];
    if (lane == 0) ml_s[warp] = make_float2(m, l);
    bad = __syncthreads_or(bad);
    float top = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, ml_s[w].x);
    const float sh = top == -CUDART_INF_F ? 0.f : top;
    float sum = 0.f, a[8];
#pragma unroll
    for (int w = 0; w < 8; ++w) { a[w] = ex2f(ml_s[w].x - sh); sum += ml_s[w].y * a[w]; }
    const uint32_t st = (uint32_t)d.w | (bad ? SAKI_ROW_BAD_PAGE : 0u);
    const bool none = st || sum == 0.f;
    E* const out = (E*)p.out.out + out_at(p, d.x, h, row0 + rr);
    for (int k = threadIdx.x; k < p.in.D; k += 256) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) x += o_s[w][k] * a[w];
      st_from_float(out, k, none ? 0.f : x / sum);
    }
    if (threadIdx.x == 0) {
      put_lse(p, d.x, h, row0 + rr, top, none ? 0.f : sum);
      if (rr == 0 && d.y == 0) put_status(p, d.x, st);
    }
    __syncthreads();
  }
}

// ---- f32 ----

template <int DP, int MR> struct FmaShape {
  static constexpr int T = 32, ROWS = MR, TILE = T * DP * 4;
  static constexpr int STAGES = DP <= 128 ? 3 : 2;
  static constexpr int SMEM = STAGES * 2 * TILE + MR * DP * 4 + MR * 36 * 4 + MR * 4 + (STAGES + 1) * (int)sizeof(Rows<T>) + (int)sizeof(LineShared);
};

// A thread holds a position for the scores (its key against a quarter of the rows), a warp a row at a time for the
// statistics, a thread one or two columns of the values for the sums.
template <int DP, int MR> __global__ void __launch_bounds__(AT) attn_fma_kernel(const __grid_constant__ AttnParams p) {
  using S = FmaShape<DP, MR>;
  constexpr int T = S::T, ST = S::STAGES, NC = DP < AT ? DP : AT, CP = DP / NC, GR = AT / NC, RW = MR / 4, RT = MR / GR;
  extern __shared__ __align__(128) char smem[];
  char* at = smem + ST * 2 * S::TILE;
  float* const q_s = (float*)at; at += MR * DP * 4;
  float* const w_s = (float*)at; at += MR * 36 * 4;          // weights; -1: not seen
  float* const a_s = (float*)at; at += MR * 4;               // factor of what is there already
  Rows<T>* const rows = (Rows<T>*)at; at += (ST + 1) * sizeof(Rows<T>);
  LineShared& line = *(LineShared*)at;
  const uint32_t tiles = smem_addr(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, col = tid % NC, grp = tid / NC;
  wait_for_predecessor();
  launch_dependents();
  long long u0, u1, chunk;
  Cursor<T> now;
  if (!piece<T>(p, line, u0, u1, chunk, now)) {
    if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  Cursor<T> look = now;
  long long looked = u0, loaded = u0;
  auto look_up = [&] {
    if (looked < u1) {
      if (tid < T) put_row<T>(p, find_row<T>(p, look), look.hr / p.RB, rows[looked % (ST + 1)]);
      look.next(p);
      ++looked;
    }
  };
  auto load = [&] {
    if (loaded < u1) {
      const uint32_t k = tiles + (uint32_t)((loaded - u0) % ST) * (2 * S::TILE);
      load_tile<float, DP, T>(p, rows[loaded % (ST + 1)], k, k + S::TILE);
      ++loaded;
    }
    cp_commit();
  };
#pragma unroll 1
  for (int i = 0; i < ST - 1; ++i) {
    look_up();
    __syncthreads();
    load();
  }
  look_up();
  float o[RT][CP], m[RW], l[RW];
  uint32_t bad = 0;
  bool fresh = true;
#pragma unroll 1
  for (long long u = u0; u < u1; ++u) {
    const int h = now.hr / p.RB, row0 = (now.hr - h * p.RB) * MR;
    if (fresh) {
      for (int i = tid; i < MR * DP; i += AT) {
        const int r = row0 + i / DP, d = i % DP, j = r / p.G;
        q_s[i] = r < p.R && d < p.in.D ? ((const float*)p.in.q)[now.b * p.in.q_seq + j * p.in.q_pos + (int64_t)(h * p.G + r - j * p.G) * p.in.q_head + d] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int k = 0; k < CP; ++k) o[i][k] = 0.f;
#pragma unroll
      for (int i = 0; i < RW; ++i) { m[i] = -CUDART_INF_F; l[i] = 0.f; }
      bad = 0;
      fresh = false;
    }
    cp_wait<ST - 2>();
    __syncthreads();
    load();
    Found ahead = {};
    const bool finding = looked < u1;
    if (finding && tid < T) ahead = find_row<T>(p, look);
    const char* const k_s = smem + (size_t)((u - u0) % ST) * (2 * S::TILE);
    const char* const v_s = k_s + S::TILE;
    const int64_t x0 = tile_start<T>(now.s, now.t);
    const bool edge = !whole<T>(p, now.s, x0);
    bad |= rows[u % (ST + 1)].bad[0];
    {
      float s[RW];
#pragma unroll
      for (int i = 0; i < RW; ++i) s[i] = 0.f;
#pragma unroll 4
      for (int j = 0; j * 4 < p.in.D; ++j) {
        const float4 k = *(const float4*)(k_s + piece_at<float, DP>(lane, j));
#pragma unroll
        for (int i = 0; i < RW; ++i) {
          const float4 q = *(const float4*)(q_s + (warp + 4 * i) * DP + j * 4);
          s[i] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[i]))));
        }
      }
      // the warp that has the scores of a row keeps its statistics: lane = position
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        const int r = warp + 4 * i;
        const bool seen = !edge || sight_of(p, now.s, row0 + r)(x0 + lane);
        const float x = seen ? s[i] * p.c : -CUDART_INF_F;
        float top = x;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        top = fmaxf(top, m[i]);
        const float sh = top == -CUDART_INF_F ? 0.f : top, a = ex2f(m[i] - sh), w = ex2f(x - sh);
        float sum = w;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        l[i] = l[i] * a + sum;
        m[i] = top;
        w_s[r * 36 + lane] = seen ? w : -1.f;
        if (lane == 0) a_s[r] = a;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const float a = a_s[grp + GR * i];
#pragma unroll
      for (int k = 0; k < CP; ++k) o[i][k] *= a;
    }
    auto sums = [&](bool some) {       // some: there may be positions that a row does not see
#pragma unroll 2
      for (int x = 0; x < T; x += 4) {
        float v[4][CP];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int k = 0; k < CP; ++k) v[e][k] = *(const float*)(v_s + piece_at<float, DP>(x + e, (col + k * NC) >> 2) + (col & 3) * 4);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const float4 w = *(const float4*)(w_s + (grp + GR * i) * 36 + x);
          const float ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < CP; ++k)
              if (!some || ww[e] >= 0.f || ww[e] != ww[e]) o[i][k] = fmaf(ww[e], v[e][k], o[i][k]);
        }
      }
    };
    if (col < p.in.D) { if (edge) sums(true); else sums(false); }
    if (finding) {
      if (tid < T) put_row<T>(p, ahead, look.hr / p.RB, rows[looked % (ST + 1)]);
      look.next(p);
      ++looked;
    }
    if (now.t + 1 == now.s.nt || u + 1 == u1) {
      const bool head = u - now.t < u0, tail = now.t + 1 < now.s.nt;
      const uint32_t st = now.s.status | (bad ? SAKI_ROW_BAD_PAGE : 0u);
      float* const part = p.part + (blockIdx.x * 2 + (head ? 0 : 1)) * (int64_t)PART<MR, DP>;
      // the sums of the rows, from the warps that have them
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RW; ++i)
        if (lane == 0) {
          const int r = warp + 4 * i;
          a_s[r] = l[i];
          if (row0 + r < p.R) {
            if (head || tail) *(float2*)(part + MR * DP + r * 2) = make_float2(m[i], bad ? -1.f : l[i]);
            else put_lse(p, now.b, h, row0 + r, m[i], st ? 0.f : l[i]);
          }
        }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int r = grp + GR * i;
        if (row0 + r >= p.R) continue;
        const float sum = a_s[r];
#pragma unroll
        for (int k = 0; k < CP; ++k) {
          const int d = col + k * NC;
          if (d >= p.in.D) continue;
          if (head || tail) part[r * DP + d] = o[i][k];
          else ((float*)p.out.out)[out_at(p, now.b, h, row0 + r) + d] = st || sum == 0.f ? 0.f : o[i][k] / sum;
        }
      }
      if (!head && !tail && now.hr == 0 && tid == 0) put_status(p, now.b, st);
      if (u + 1 == u1 && tid == 0) {
        const long long end = u - now.t + now.s.nt;
        p.desc[blockIdx.x] = tail && !head ? make_int4((int)now.b, now.hr, (int)((end - 1) / chunk) - (int)blockIdx.x, (int)now.s.status) : make_int4(0, 0, 0, 0);
      }
      fresh = true;
    }
    now.next(p);
    __syncthreads();
  }
  cp_wait<0>();
}

constexpr int MAX_BLOCKS = 592;       // of a call: four for each of 148 SMs

struct Kernel { const void* fn; int rows, dp, t, smem; };
template <int DP, int MT> Kernel mma_kernel() { using S = MmaShape<DP, MT>; return {(const void*)attn_mma_kernel<DP, MT>, S::ROWS, DP, S::T, S::SMEM}; }
template <int DP, int MR> Kernel fma_kernel() { using S = FmaShape<DP, MR>; return {(const void*)attn_fma_kernel<DP, MR>, S::ROWS, DP, S::T, S::SMEM}; }
template <int DP> Kernel pick(int R, int dtype) {
  if (dtype == SAKI_BF16) return R <= 16 ? mma_kernel<DP, 1>() : R <= 32 ? mma_kernel<DP, 2>() : mma_kernel<DP, 4>();
  return R <= 4 ? fma_kernel<DP, 4>() : fma_kernel<DP, 16>();
}
Kernel pick(const saki_attn_in& in) {
  const int R = in.Q * (in.Hq / in.H);
  return in.D <= 64 ? pick<64>(R, in.dtype) : in.D <= 128 ? pick<128>(R, in.dtype) : pick<256>(R, in.dtype);
}
int64_t part_floats(const Kernel& k) { return (int64_t)k.rows * (k.dp + 2); }

template <typename E, int DP> cudaError_t join(const AttnParams& p, int rows, int blocks, cudaStream_t st) {
  const dim3 grid((unsigned)blocks, (unsigned)std::min(p.R, std::min(rows, 16)));
  if constexpr (sizeof(E) == 4) {
    if (rows == 4) return launch_pdl(attn_join_kernel<E, 4, DP>, grid, 256, 0, st, true, p);
    return launch_pdl(attn_join_kernel<E, 16, DP>, grid, 256, 0, st, true, p);
  } else {
    if (rows == 16) return launch_pdl(attn_join_kernel<E, 16, DP>, grid, 256, 0, st, true, p);
    if (rows == 32) return launch_pdl(attn_join_kernel<E, 32, DP>, grid, 256, 0, st, true, p);
    return launch_pdl(attn_join_kernel<E, 64, DP>, grid, 256, 0, st, true, p);
  }
}
template <typename E> cudaError_t join(const AttnParams& p, const Kernel& k, int blocks, cudaStream_t st) {
  return k.dp == 64 ? join<E, 64>(p, k.rows, blocks, st) : k.dp == 128 ? join<E, 128>(p, k.rows, blocks, st) : join<E, 256>(p, k.rows, blocks, st);
}

}  // namespace

int64_t attention_scratch_bytes(const saki_attn_in& in) { return MAX_BLOCKS * 16 + MAX_BLOCKS * 2 * part_floats(pick(in)) * 4; }

cudaError_t launch_attention(const saki_attn_in& in, const saki_attn_out& out, void* scratch, unsigned long long* flagged, int* n_launches,
                             cudaStream_t st) {
  const Kernel k = pick(in);
  AttnParams p = {};
  p.in = in; p.out = out; p.flagged = flagged;
  p.G = in.Hq / in.H; p.R = in.Q * p.G; p.RB = (p.R + k.rows - 1) / k.rows;
  p.c = in.scale * 1.4426950408889634f;
  const int size = in.dtype == SAKI_BF16 ? 2 : 4;
  p.q_vec = ((uintptr_t)in.q | (uintptr_t)(in.q_seq * size) | (uintptr_t)(in.q_pos * size) | (uintptr_t)(in.q_head * size)) % 16 == 0;
  p.desc = (int4*)scratch;
  p.part = (float*)((char*)scratch + MAX_BLOCKS * 16);
  int dev = 0, sms = 148, per = 1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, k.fn, AT, k.smem);
  if (e != cudaSuccess) return e;
  const int64_t most = in.B * in.H * p.RB * (((int64_t)in.max_pages * in.page_size + k.t - 1) / k.t);      // tiles, if every table were full
  const int blocks = (int)std::min<int64_t>(most, std::min(sms * std::max(per, 1), MAX_BLOCKS));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(AT); cfg.dynamicSmemBytes = (size_t)k.smem; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  void* args[] = {&p};
  e = cudaLaunchKernelExC(&cfg, k.fn, args);
  if (e != cudaSuccess) return e;
  ++*n_launches;
  e = in.dtype == SAKI_BF16 ? join<__nv_bfloat16>(p, k, blocks, st) : join<float>(p, k, blocks, st);
  if (e == cudaSuccess) ++*n_launches;
  return e;
}

}  // namespace saki
