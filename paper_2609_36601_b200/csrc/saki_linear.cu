// Cross entropy straight from hidden states and an lm-head's weights (Section 3.5: the trainer's objective for freshly computed
// logits, Eqs. "k1_loss_token", "teacher_mode_loss"), without [N, V] logits or gradients in memory:
//
//   z_iv = h_i . W_v / tau,  L_i = -coef_i log pi_i(tok_i),  G_iv = coef_i (pi_iv - [v = tok_i]),
//   dH = s G W,  dW = s G^T H,  s = grad_scale / tau
//
// Rows that contribute nothing (masked, flagged) are left out before any product: the others' hidden states are gathered into a
// matrix of their own, in order, whose number of rows the products read from device memory.  (So a masked row costs nothing, and what stands in it,
// infinities among it, reaches nothing.)
//   forward    one launch over all tiles of the logits: their sums and the supervised token's logit leave, the logits do not
//   backward   the vocabulary in pieces: the logits of a piece once more, G of the piece in bf16 into a buffer; in the next launch, beside the next piece's
//              logits, its two products
// All three products are tiles of 256 x 256 on CTA pairs (tcgen05, cta_group::2), K in blocks of 64 through a TMA ring; operands that lie with their
// K outermost (W and H in the two gradients, G in dW) are read M- or N-major as they are, nothing is transposed.  Tiles are dealt out by tickets: the kinds
// differ in length.  G is rounded to bf16 (half a step, 2^-8 of an element at the most), as an operand of the tensor cores has to be next to bf16 weights; s is
// applied to the sums (in G its rounding would be the same in every unlikely target's -s: up to 2^-8 of the whole gradient).  Sums are float32 (tensor memory, and across
// pieces), the log-sum-exp float64 across tiles.
//
// What bounds it: the tensor cores at the clock that power leaves them.  4096 x 2560 x 151936, called alone: forward 2.14 ms = 1.49 PFLOP/s (89 % of the measured burst of a cuBLAS
// product), backward 6.86 ms = 1.39 PFLOP/s over its three products; called in a row forward 2.5, both 9.2.  Few rows: 64 x 1024 x 32000 111 us for both, where the weights' bytes alone take 10 and 20: seven launches, and tiles
// of 256 rows of which 192 are padding.  Vocabulary rows that start off 128-byte lines (1096 features) cost 5 % of the forward.
//
// Persistent CTAs, one per SM:
//   warp 0    one thread: TMA loads        warp 1   allocates tensor memory; in a pair's first CTA one thread issues the products
//   warps 2-5 what becomes of a tile, a row a thread         warp 6   in a pair's first CTA one thread takes the tickets and tells all roles of both CTAs
// Every wait on an mbarrier is bounded; one that runs out ends all roles, and the outputs are NaN.
#include "saki_device.cuh"
#include "saki_tensor_map.cuh"
#include <algorithm>
#include <mutex>

namespace saki {

namespace lin {

namespace {

constexpr int TILE = 256, HALF = 128, BK = 64, ACC = 2, STAGES = 6, SLOTS = 4;
constexpr int A_BYTES = HALF * BK * 2, STAGE_BYTES = 2 * A_BYTES;
constexpr int THREADS = 224;
constexpr int OUT_BYTES = 32 * 128;                          // what a warp hands to a store: 32 rows of 128 bytes
constexpr int SMEM = STAGES * STAGE_BYTES + 4 * 2 * OUT_BYTES + 512 + 1024;      // ring, two stores of each epilogue warp, barriers, alignment
constexpr int MAX_CTAS = 256, MAX_LAUNCHES = 512;
enum { KIND_LOGITS = 0, KIND_DH, KIND_DW, KINDS };

// what the products of a call share in scratch
struct Head {
  int count;                          // rows that were gathered
  unsigned char error[MAX_CTAS];      // 1: a wait of that CTA ran out
  unsigned ticket[MAX_LAUNCHES];
};

struct Rows {                         // the call's rows, and what is gathered of them
  saki_linear_in in;
  const float* lse;                   // backward: rows without a finite one contribute nothing; forward: NULL
  Head* head;
  int* rank;                          // [N] place among the gathered rows, -1: not among them
  int* tok;                           // by place
  float* coef;
  float* lse2;                        // log-sum-exp in base 2 (backward)
  double to_base2;                    // log2(e), as far as the factor of the products is off as a float32: c product - lse2 is a difference then, of which that is a share
  __nv_bfloat16* h;                   // [rows, padded to whole tiles][ld]: rows start on 128-byte boundaries
  int ld;
  int vec;                            // rows of `hidden` start at 16-byte boundaries
};

struct Tiles {
  Head* head;
  int launch;                         // which ticket counter, -1: tiles of one kind alone, dealt out in turn
  int d, V, d_tiles;
  long long wait_limit;
  // logits of columns [v0, v0 + 256 l_tiles): their sums, or G
  int l_tiles, v0;
  float c;                            // log2(e) / temperature, and what the sums lack
  float2* part;                       // forward: [rows][n_tiles] (largest product, sum of 2^(c (product - it)))
  float* z_tok;                       // forward: the supervised token's product
  int n_tiles;
  const int* tok;
  const float* coef;
  const float* lse2;
  float scale;                        // grad_scale / temperature, of dW's sums
  int grad;                           // G
  // the products of an earlier piece's G: columns [b0, b0 + 256 b_tiles)
  int b_tiles, b0, splits, first;     // dH: a tile's K in so many parts; first: the sums start here
  int dh, dw;                         // wanted
  int rows;                           // of a part of dH, [splits][rows][d]
};

// ---------------------------------------------------------------- rows
struct Row { int tok; float coef; uint32_t status; };      // tok -1: the row contributes nothing
__device__ __forceinline__ Row row_of(const Rows& P, int64_t row) {
  const saki_linear_in& in = P.in;
  Row m = {-1, 0.f, 0u};
  // (all loads first: a row's word on whether it counts takes one of them, not six in turn)
  const bool masked = in.mask && in.mask[row] == 0;
  const uint32_t rollout = in.rollout_status ? in.rollout_status[row] : 0u;
  const bool hit = in.corrected && in.corrected[row] != 0;
  const int target = in.target[row], top1 = in.corrected ? in.teacher_top1[row] : 0;
  const float advantage = in.advantage ? in.advantage[row] : 1.f, lse = P.lse ? P.lse[row] : 0.f;
  if (masked) { m.status = SAKI_ROW_MASKED; return m; }
  if (rollout & (SAKI_ROW_NONFINITE | SAKI_ROW_BAD_ID | SAKI_ROW_TIMEOUT | SAKI_ROW_NOT_COMPUTED)) { m.status = SAKI_ROW_NOT_COMPUTED; return m; }
  const int tok = hit ? top1 : target;
  const float coef = hit ? 1.f : advantage;
  if (!(fabsf(coef) < CUDART_INF_F)) { m.status = SAKI_ROW_NONFINITE; return m; }
  if (tok < 0 || tok >= in.V) { m.status = SAKI_ROW_BAD_ID; return m; }
  if (!(fabsf(lse) < CUDART_INF_F)) { m.status = SAKI_ROW_NONFINITE; return m; }
  m.tok = tok; m.coef = coef;
  return m;
}

constexpr int GT = 256;
// Gathers the rows that contribute, in order.  A block has a range of rows and counts those before it by itself (a few bytes a row): one launch.
__global__ void __launch_bounds__(GT) gather_kernel(const Rows P, int per_block) {
  __shared__ int sum[GT / 32];
  __shared__ int place[GT];
  launch_dependents();
  wait_for_predecessor();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = P.in.d;
  const int64_t N = P.in.N, r0 = min(N, (int64_t)blockIdx.x * per_block), r1 = min(N, r0 + per_block);
  if (blockIdx.x == 0) {
    for (int i = tid; i < MAX_CTAS; i += GT) P.head->error[i] = 0;
    for (int i = tid; i < MAX_LAUNCHES; i += GT) P.head->ticket[i] = 0;
  }
  int n = 0;
#pragma unroll 4
  for (int64_t i = tid; i < r0; i += GT) n += row_of(P, i).tok >= 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
  if (lane == 0) sum[warp] = n;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < GT / 32; ++w) base += sum[w];
  for (int64_t c0 = r0; c0 < r1; c0 += GT) {
    const int64_t row = c0 + tid;
    Row m = {-1, 0.f, 0u};
    if (row < r1) m = row_of(P, row);
    const unsigned have = __ballot_sync(0xffffffffu, m.tok >= 0);
    __syncthreads();                  // `sum` and `place` have been read
    if (lane == 0) sum[warp] = __popc(have);
    __syncthreads();
    int at = base + __popc(have & ((1u << lane) - 1));
    int total = 0;
#pragma unroll
    for (int w = 0; w < GT / 32; ++w) { at += w < warp ? sum[w] : 0; total += sum[w]; }
    if (m.tok < 0) at = -1;
    place[tid] = at;
    if (row < r1) P.rank[row] = at;
    if (at >= 0) {
      P.tok[at] = m.tok;
      P.coef[at] = m.coef;
      if (P.lse) P.lse2[at] = (float)((double)P.lse[row] * P.to_base2);
    }
    __syncthreads();
    const int rows = (int)min((int64_t)GT, r1 - c0);
    for (int r = warp; r < rows; r += GT / 32) {
      if (place[r] < 0) continue;
      const __nv_bfloat16* s = (const __nv_bfloat16*)P.in.hidden + (c0 + r) * P.in.ld_h;
      __nv_bfloat16* t = P.h + (int64_t)place[r] * P.ld;
      if (P.vec) {
#pragma unroll 4
        for (int j = lane; j < d / 8; j += 32) ((uint4*)t)[j] = __ldg((const uint4*)s + j);
      } else
        for (int j = lane; j < d; j += 32) t[j] = s[j];
    }
    base += total;
  }
  if (blockIdx.x == gridDim.x - 1) {  // the last rows' block of K is filled up with zeros (dW sums over whole blocks)
    const int64_t zeros = (int64_t)((base + BK - 1) / BK * BK - base) * P.ld / 8;
    uint4* t = (uint4*)(P.h + (int64_t)base * P.ld);
    for (int64_t j = tid; j < zeros; j += GT) t[j] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) P.head->count = base;
  }
}

__device__ __forceinline__ bool any_failed(const Head* h) {      // all threads of a block
  bool f = false;
  for (int k = threadIdx.x; k < MAX_CTAS; k += blockDim.x) f |= h->error[k] != 0;
  return __syncthreads_or(f);
}

// forward, a warp a row: the tiles' sums become the row's log-sum-exp and loss
__global__ void __launch_bounds__(256) loss_kernel(const Rows P, const saki_linear_out out, const float2* part, const float* z_tok, int n_tiles, float c, double rtau, unsigned long long* flagged) {
  launch_dependents();
  wait_for_predecessor();
  const bool failed = any_failed(P.head);
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= P.in.N) return;
  const Row m = row_of(P, row);
  uint32_t status = m.status;
  float loss = 0.f, logp = 0.f, lse = 0.f;
  if (m.tok >= 0) {
    const int64_t at = P.rank[row];
    const float2* pp = part + at * n_tiles;
    float mx = -CUDART_INF_F;
    bool nan = false;
    for (int t = lane; t < n_tiles; t += 32) { const float2 a = pp[t]; mx = fmaxf(mx, a.x); nan |= a.y != a.y; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    nan = __any_sync(0xffffffffu, nan);
    double s = 0.0;
    for (int t = lane; t < n_tiles; t += 32) {
      const float2 a = pp[t];
      if (a.x > -CUDART_INF_F) s += (double)(a.y * ex2f((a.x - mx) * c));
    }
    s = warp_sum(s);
    // (both from the largest product: a log-probability next to 0 is no difference of large numbers)
    const double ls = log2(s) * LN2, l = (double)mx * rtau + ls, lp = ((double)z_tok[at] - (double)mx) * rtau - ls;
    loss = (float)(-(double)m.coef * lp); logp = (float)lp; lse = (float)l;
    if (failed) status = SAKI_ROW_TIMEOUT;
    else if (nan || !(fabsf(lse) < CUDART_INF_F) || !(fabsf(logp) < CUDART_INF_F)) status = SAKI_ROW_NONFINITE;
    if (status) { loss = logp = 0.f; lse = CUDART_NAN_F; }
  }
  if (lane == 0) {
    if (out.loss) out.loss[row] = loss;
    if (out.logp_tok) out.logp_tok[row] = logp;
    out.lse[row] = lse;
    if (out.row_status) out.row_status[row] = status;
    if (status & (SAKI_ROW_NONFINITE | SAKI_ROW_BAD_ID | SAKI_ROW_TIMEOUT)) atomicAdd(flagged, 1ull);
  }
}

// backward: the parts of dH are added and rounded, rows that contribute nothing get zeros; NaN everywhere where a wait ran out.  L lanes share the parts of eight elements.
template <int L>
__global__ void __launch_bounds__(256) dhidden_kernel(const Rows P, const float* dh, int64_t dh_split, int splits, float scale, __nv_bfloat16* out, int64_t ld_out, __nv_bfloat16* dw, int64_t ld_dw) {
  launch_dependents();
  wait_for_predecessor();
  const bool failed = any_failed(P.head);
  const int d = P.in.d, d8 = d / 8, sub = threadIdx.x % L;
  const uint4 nan = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
  if (out) {
    const int64_t n = P.in.N * d8, step = (int64_t)gridDim.x * 256 / L;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 / L; i0 < n; i0 += step) {      // (the same for all threads of a block: they exchange)
      const int64_t i = i0 + threadIdx.x / L, row = min(i, n - 1) / d8;
      const int j = (int)(min(i, n - 1) - row * d8) * 8;
      const int at = P.rank[row];
      float a[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) a[k] = 0.f;
      if (at >= 0) {
        const float* s = dh + (int64_t)at * d + j + sub * dh_split;
#pragma unroll 4
        for (int p = sub; p < splits; p += L, s += L * dh_split) {
          const float4 x = *(const float4*)s, y = *(const float4*)(s + 4);
          a[0] += x.x; a[1] += x.y; a[2] += x.z; a[3] += x.w; a[4] += y.x; a[5] += y.y; a[6] += y.z; a[7] += y.w;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) a[k] += __shfl_xor_sync(0xffffffffu, a[k], o);
        a[k] *= scale;
      }
      if (i < n && sub == 0)
        *(uint4*)(out + row * ld_out + j) = failed ? nan : make_uint4(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(a[4], a[5]), pack_bf16x2(a[6], a[7]));
    }
  }
  if (failed && dw)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)P.in.V * d8; i += (int64_t)gridDim.x * 256)
      *(uint4*)(dw + i / d8 * ld_dw + i % d8 * 8) = nan;
}

// ---------------------------------------------------------------- products
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {      // the same offset in a CTA of the cluster
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ bool try_wait(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
  return ok != 0;
}
// bounded: false if the phase did not complete within the limit or another role has given up
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, volatile int* stop, long long limit) {
  if (try_wait(b, parity)) return true;
  const long long t0 = clock64();
  while (!try_wait(b, parity)) {
    if (*stop) return false;
    if (clock64() - t0 > limit) { *stop = 1; return false; }
  }
  return true;
}
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Shared-memory matrix descriptors, 128-byte swizzle, rows of 128 bytes in groups of eight 1024 bytes apart.  K-major: rows are of M or N, a row holds 64 k.
// MN-major: rows are of k, a row holds 64 of M or N, and the next 64 lie `8192` bytes on (64 rows of k in a box).
template <bool MN> __device__ __forceinline__ uint64_t desc(uint32_t at) {
  return (uint64_t)((at & 0x3FFFF) >> 4) | (uint64_t)(MN ? 8192 >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// instruction descriptor: float32 sums, bf16 operands, M = 256 (of the pair), N = 256
template <bool A_MN, bool B_MN> constexpr uint32_t IDESC =
    (1u << 4) | (1u << 7) | (1u << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
template <bool A_MN, bool B_MN> __device__ __forceinline__ void mma_block(uint32_t tmem, uint32_t at, bool on_top) {      // a block of K
  const uint64_t a = desc<A_MN>(at), b = desc<B_MN>(at + A_BYTES);
#pragma unroll
  for (int k = 0; k < BK / 16; ++k)      // 16 further along K: 32 bytes on in the swizzled row, or 16 rows on; in units of 16 bytes
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem), "l"(a + (uint64_t)(k * (A_MN ? 128 : 2))), "l"(b + (uint64_t)(k * (B_MN ? 128 : 2))), "n"(IDESC<A_MN, B_MN>), "r"((uint32_t)(on_top || k))
                 : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {      // an arrival in both CTAs when the products issued so far are done
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void ld32(uint32_t at, float (&x)[32]) {
  uint32_t r[32];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                 "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                 "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(at) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}

// A warp's 32 rows of 128 bytes to a box of 32 rows: the lanes' words go to shared memory in the box's swizzle, one lane hands them to the copy engine (rows of a warp's own
// stores would be 32 lines of 16 bytes each).  Two buffers; `add`: to what is there.
__device__ __forceinline__ uint4 pack8(const float* y) { return make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])); }
struct Out {
  uint32_t buf;                       // of the warp
  int n;                              // stores so far
  __device__ __forceinline__ void put(const uint4 (&w)[8], const CUtensorMap* map, int x, int y, bool add, int lane) {
    const uint32_t at = buf + (n & 1) * OUT_BYTES;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");      // the store before the last has been read
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(w[j].x), "r"(w[j].y), "r"(w[j].z), "r"(w[j].w) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      if (add) asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(at) : "memory");
      else asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(at) : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    ++n;
  }
};

struct Maps { CUtensorMap h_k, w_k, h_mn, w_mn, g_k, g_mn, g_out, dw_out, dh_out; };

struct Tile { int kind, m, n, k0, k1, split; };      // kind -1: there is none
// The tiles of a launch: of the two gradients the longer ones first, logits last.
struct Plan {
  int count, m_tiles, n_dw, n_dh, total, blocks;
  bool dh_first;
  __device__ __forceinline__ Plan(const Tiles& P) {
    count = *(volatile int*)&P.head->count;
    m_tiles = (count + TILE - 1) / TILE;
    n_dw = P.dw ? P.b_tiles * P.d_tiles : 0;
    n_dh = P.dh && P.b_tiles ? m_tiles * P.d_tiles * P.splits : 0;
    blocks = (min(P.V - P.b0, P.b_tiles * TILE) + BK - 1) / BK;      // of K, of dH
    dh_first = (int64_t)blocks * BK > (int64_t)count * P.splits;
    total = n_dw + n_dh + m_tiles * P.l_tiles;
  }
  __device__ __forceinline__ Tile tile(const Tiles& P, int t) const {
    Tile x = {-1, 0, 0, 0, 0, 0};
    if (t < 0) return x;
    const int first = dh_first ? n_dh : n_dw;
    if (t < n_dw + n_dh && (t < first) == dh_first) {      // 256 rows, 256 features, a part of the piece's entries
      if (!dh_first) t -= n_dw;
      x.kind = KIND_DH;
      const int per = P.d_tiles * P.splits;
      x.m = t / per; t -= x.m * per;
      x.n = t / P.splits; x.split = t - x.n * P.splits;
      x.k0 = (int)((int64_t)blocks * x.split / P.splits); x.k1 = (int)((int64_t)blocks * (x.split + 1) / P.splits);
    } else if (t < n_dw + n_dh) {     // 256 vocabulary entries, 256 features, all rows
      if (dh_first) t -= n_dh;
      x.kind = KIND_DW; x.m = t / P.d_tiles; x.n = t - x.m * P.d_tiles; x.k1 = (count + BK - 1) / BK;
    } else {                          // 256 rows, 256 vocabulary entries; row tiles innermost: a weight tile is read by neighbours
      t -= n_dw + n_dh;
      x.kind = KIND_LOGITS; x.n = t / m_tiles; x.m = t - x.n * m_tiles; x.k1 = (P.d + BK - 1) / BK;
    }
    return x;
  }
};

__global__ void __launch_bounds__(THREADS, 1) tiles_kernel(const __grid_constant__ Maps maps, const Tiles P) {
  extern __shared__ unsigned char raw[];
  unsigned char* base = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);      // (the same offset in both CTAs)
  unsigned char* const out_base = base + STAGES * STAGE_BYTES;
  uint64_t* full = (uint64_t*)(out_base + 4 * 2 * OUT_BYTES);
  uint64_t *empty = full + STAGES, *t_full = empty + STAGES, *t_empty = t_full + ACC, *s_full = t_empty + ACC, *s_empty = s_full + SLOTS;
  int* slot_tile = (int*)(s_empty + SLOTS);
  uint32_t* tmem_slot = (uint32_t*)(slot_tile + SLOTS);
  volatile int* stop = (volatile int*)(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = blockIdx.x & 1u;
  launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int a = 0; a < ACC; ++a) { mbar_init(&t_full[a], 1); mbar_init(&t_empty[a], 8); }
    for (int s = 0; s < SLOTS; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], 11); }      // producers 2, products 1, epilogues 8
    *stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(ACC * TILE) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_sync();                     // both CTAs' barriers exist before either signals the other's
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  wait_for_predecessor();
  const Plan plan(P);
  const long long limit = P.wait_limit;

  int slot = 0, in_turn = (int)blockIdx.x >> 1;
  uint32_t slot_phase = 0;
  auto next_tile = [&](bool whole_warp) -> Tile {      // of a role: waits for the next ticket, reads it, gives the slot back
    Tile x = {-1, 0, 0, 0, 0, 0};
    if (P.launch < 0) {
      x = plan.tile(P, in_turn < plan.total ? in_turn : -1);
      in_turn += (int)gridDim.x >> 1;
      return x;
    }
    const bool there = wait(&s_full[slot], slot_phase, stop, limit);
    if (whole_warp ? !__all_sync(0xffffffffu, there) : !there) return x;      // (a warp gives up as one: each lane has a clock of its own)
    x = plan.tile(P, *(volatile int*)&slot_tile[slot]);
    if (whole_warp) __syncwarp();
    if (!whole_warp || lane == 0) arrive_at(at_rank(smem_addr(&s_empty[slot]), 0));
    if (++slot == SLOTS) { slot = 0; slot_phase ^= 1u; }
    return x;
  };

  if (warp == 0) {
    if (lane == 0) {                  // ---- loads
      asm volatile("fence.proxy.async.global;" ::: "memory");      // (what the launches before have written is read by TMA)
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (Tile x = next_tile(false), next = x; ok && x.kind >= 0; x = next) {
        if (x.k0 == x.k1) next = next_tile(false);
        const int rows = x.m * TILE + (int)rank * HALF, cols = x.n * TILE + (int)rank * HALF;      // this CTA's part of M and of N
        for (int kb = x.k0; kb < x.k1; ++kb) {
          if (kb == (x.k0 + x.k1) / 2) next = next_tile(false);      // (so that there is no wait between tiles)
          if (!wait(&empty[stage], phase ^ 1u, stop, limit)) { ok = false; break; }
          const uint32_t a = smem_addr(base + stage * STAGE_BYTES), b = a + A_BYTES, bar = at_rank(smem_addr(&full[stage]), 0);
          if (rank == 0) mbar_expect_tx(&full[stage], 2 * STAGE_BYTES);
          const int k = kb * BK;
          if (x.kind == KIND_LOGITS) {
            load_box(a, &maps.h_k, k, rows, bar);
            load_box(b, &maps.w_k, k, P.v0 + cols, bar);
          } else if (x.kind == KIND_DH) {
            load_box(a, &maps.g_k, k, rows, bar);
            load_box(b, &maps.w_mn, cols, P.b0 + k, bar);
            load_box(b + A_BYTES / 2, &maps.w_mn, cols + 64, P.b0 + k, bar);
          } else {
            load_box(a, &maps.g_mn, rows, k, bar);
            load_box(a + A_BYTES / 2, &maps.g_mn, rows + 64, k, bar);
            load_box(b, &maps.h_mn, cols, k, bar);
            load_box(b + A_BYTES / 2, &maps.h_mn, cols + 64, k, bar);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {     // ---- products
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (Tile x = next_tile(false), next = x; ok && x.kind >= 0; x = next) {
        if (x.k0 == x.k1) next = next_tile(false);
        if (!wait(&t_empty[acc], acc_phase ^ 1u, stop, limit)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + (uint32_t)(acc * TILE);
        for (int kb = x.k0; kb < x.k1; ++kb) {
          if (kb == (x.k0 + x.k1) / 2) next = next_tile(false);
          if (!wait(&full[stage], phase, stop, limit)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t at = smem_addr(base + stage * STAGE_BYTES);
          if (x.kind == KIND_LOGITS) mma_block<false, false>(d, at, kb != x.k0);
          else if (x.kind == KIND_DH) mma_block<false, true>(d, at, kb != x.k0);
          else mma_block<true, true>(d, at, kb != x.k0);
          commit(&empty[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        commit(&t_full[acc]);
        if (++acc == ACC) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else if (warp == 6) {
    if (lane == 0 && rank == 0 && P.launch >= 0) {     // ---- tickets
      int s = 0;
      uint32_t phase = 0;
      for (;;) {
        if (!wait(&s_empty[s], phase ^ 1u, stop, limit)) break;
        const unsigned t = atomicAdd(&P.head->ticket[P.launch], 1u);
        const int mine = t < (unsigned)plan.total ? (int)t : -1;
        *(volatile int*)&slot_tile[s] = mine;
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at_rank(smem_addr(&slot_tile[s]), 1)), "r"(mine) : "memory");
        arrive_at(at_rank(smem_addr(&s_full[s]), 0));
        arrive_at(at_rank(smem_addr(&s_full[s]), 1));
        if (mine < 0) break;
        if (++s == SLOTS) { s = 0; phase ^= 1u; }
      }
    }
  } else {                            // ---- what becomes of a tile: tensor memory's lanes 32 (warp % 4) on, a row a thread
    const int q = warp & 3;
    int acc = 0;
    uint32_t acc_phase = 0;
    Out out = {smem_addr(out_base + q * 2 * OUT_BYTES), 0};
    for (;;) {
      const Tile x = next_tile(true);
      if (x.kind < 0) break;
      const bool done = wait(&t_full[acc], acc_phase, stop, limit);
      if (!__all_sync(0xffffffffu, done)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * TILE);
      const int row = x.m * TILE + (int)rank * HALF + q * 32 + lane;      // of H, or the vocabulary entry within the piece
      if (x.kind == KIND_LOGITS) {
        const bool there = row < plan.count;
        const int col_tile = P.v0 + x.n * TILE;
        const int tok = there ? P.tok[row] : -1;
        if (!P.grad) {
          float m = -CUDART_INF_F, s = 0.f, z = 0.f;      // m: of the products, the sum under c m
#pragma unroll 1
          for (int ch = 0; ch < TILE / 32; ++ch) {
            float y[32];
            const int col0 = col_tile + ch * 32;
            if (col0 >= P.V) break;
            ld32(from + ch * 32, y);
            if ((unsigned)(tok - col0) < 32u) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (tok - col0 == i) z = y[i];
            }
            if (col0 + 32 > P.V) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (col0 + i >= P.V) y[i] = -CUDART_INF_F;
            }
            float t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = fmaxf(y[i], y[i + 4]);
#pragma unroll
            for (int i = 8; i < 32; i += 8)
#pragma unroll
              for (int j = 0; j < 4; ++j) t[j] = fmaxf(t[j], fmaxf(y[i + j], y[i + j + 4]));
            const float cm = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
            if (cm > m) { s *= m > -CUDART_INF_F ? ex2f((m - cm) * P.c) : 0.f; m = cm; }
            const float2 cc = splat(P.c), off = splat(m > -CUDART_INF_F ? -m : 0.f);      // (nothing but -inf, or NaN, so far)
            float2 a0 = splat(0.f), a1 = splat(0.f);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              a0 = fadd2(a0, ex2f2(fmul2(fadd2(make_float2(y[i], y[i + 1]), off), cc)));
              a1 = fadd2(a1, ex2f2(fmul2(fadd2(make_float2(y[i + 2], y[i + 3]), off), cc)));
            }
            s += (a0.x + a0.y) + (a1.x + a1.y);
          }
          if (there) {
            P.part[(int64_t)row * P.n_tiles + x.n] = make_float2(m, s);
            if ((unsigned)(tok - col_tile) < (unsigned)TILE) P.z_tok[row] = z;
          }
        } else {
          const float k = there ? P.coef[row] : 0.f, l2 = there ? P.lse2[row] : 0.f;
          const bool large = __any_sync(0xffffffffu, !(fabsf(l2) < 1024.f));
#pragma unroll 1
          for (int ch = 0; ch < TILE / 64; ++ch) {
            uint4 w[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              float y[32];
              const int col0 = col_tile + ch * 64 + half * 32;
              ld32(from + ch * 64 + half * 32, y);
              const float2 cc = splat(P.c), off = splat(-l2), kk = splat(k);
              if (large) {            // a large log-sum-exp's rounding may leave a logit above it
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = k * ex2f(fminf(fmaf(y[i], P.c, -l2), 0.f));
              } else {
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                  const float2 e = fmul2(ex2f2(ffma2(make_float2(y[i], y[i + 1]), cc, off)), kk);
                  y[i] = e.x; y[i + 1] = e.y;
                }
              }
              if (!there || col0 + 32 > P.V) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (!there || col0 + i >= P.V) y[i] = 0.f;
              }
              if ((unsigned)(tok - col0) < 32u) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (tok - col0 == i) y[i] -= k;
              }
#pragma unroll
              for (int v = 0; v < 4; ++v) w[half * 4 + v] = pack8(y + 8 * v);
            }
            out.put(w, &maps.g_out, x.n * TILE + ch * 64, row - lane, false, lane);
          }
        }
      } else if (x.kind == KIND_DH) {
        const int y0 = x.split * P.rows + row - lane;
        // (rows of the warp; a part of a short last piece may be empty: nothing was summed, nothing is added.  The first piece, which stores, has 13 blocks a part at the least)
        if (x.k0 < x.k1 && row - lane < plan.count) {
#pragma unroll 1
          for (int ch = 0; ch < TILE / 32; ++ch) {
            if (x.n * TILE + ch * 32 >= P.d) break;
            float y[32];
            ld32(from + ch * 32, y);
            uint4 w[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) w[v] = make_uint4(__float_as_uint(y[4 * v]), __float_as_uint(y[4 * v + 1]), __float_as_uint(y[4 * v + 2]), __float_as_uint(y[4 * v + 3]));
            out.put(w, &maps.dh_out, x.n * TILE + ch * 32, y0, !P.first, lane);
          }
        }
      } else {
        const bool none = x.k0 == x.k1;            // no rows at all: nothing was summed
        const float k = P.scale;
        if (P.b0 + row - lane < P.V) {
#pragma unroll 1
          for (int ch = 0; ch < TILE / 64; ++ch) {
            if (x.n * TILE + ch * 64 >= P.d) break;
            uint4 w[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              float y[32];
              ld32(from + ch * 64 + half * 32, y);
#pragma unroll
              for (int i = 0; i < 32; ++i) y[i] = none ? 0.f : y[i] * k;
#pragma unroll
              for (int v = 0; v < 4; ++v) w[half * 4 + v] = pack8(y + 8 * v);
            }
            out.put(w, &maps.dw_out, x.n * TILE + ch * 64, P.b0 + row - lane, false, lane);
          }
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_at(at_rank(smem_addr(&t_empty[acc]), 0));
      if (++acc == ACC) { acc = 0; acc_phase ^= 1u; }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (*stop) {                        // copies and products that are under way end long before this
    const long long t0 = clock64();
    while (clock64() - t0 < 1000000) {}
    if (tid == 0) P.head->error[blockIdx.x] = 1;
  }
  cluster_sync();                     // neither CTA leaves while the other may still signal it
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(ACC * TILE) : "memory");
  }
}

// ---------------------------------------------------------------- host side
// a row-major matrix of bf16 (or float32): boxes of 128 bytes of box_rows rows, 128-byte swizzle, zeros outside
bool make_map(CUtensorMap* map, const void* ptr, int64_t rows, int64_t cols, int64_t ld, int box_rows, bool f32 = false) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * (f32 ? 4 : 2)};
  const cuuint32_t box[2] = {f32 ? 32u : 64u, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// The pieces of the vocabulary, and where things lie in scratch.
struct Layout {
  int64_t rows;                       // padded to whole tiles
  int n_tiles, d_tiles, ld, piece, pieces, splits;      // piece: columns, a multiple of 256
  int64_t rank, tok, coef, lse2, h, part, z_tok, g, dh, bytes;
};
Layout layout(int64_t N, int d, int V, bool backward) {
  Layout l = {};
  l.rows = up(std::max<int64_t>(N, 1), TILE);
  l.n_tiles = (V + TILE - 1) / TILE;
  l.d_tiles = (d + TILE - 1) / TILE;
  l.ld = (int)up(d, 64);
  // A piece's G takes up to 256 MB (two pieces are there at a time); the pieces are about equal.  Larger pieces mean fewer launches, each of which ends with SMs that have
  // no tile left, and fewer additions to dH in memory; that G does not stay in L2 costs less.  (2560 features, 151936 entries, backward pass of 8192 rows, with pieces of 32, 64, 128, 256
  // and 512 MB: 19.4, 16.1, 14.7, 14.3 and 14.1 ms; 4096 rows 8.3, 7.5, 7.3, 7.2, 7.2.)
  const int64_t most = std::max<int64_t>(1, (256LL << 20) / (l.rows * 2 * TILE));
  l.pieces = (int)std::max<int64_t>((l.n_tiles + most - 1) / most, 1);
  l.pieces = std::min(l.pieces, MAX_LAUNCHES - 1);
  const int tiles = (l.n_tiles + l.pieces - 1) / l.pieces;
  l.pieces = (l.n_tiles + tiles - 1) / tiles;
  l.piece = tiles * TILE;
  // few rows: the sums over the vocabulary are cut so that there is a tile for nearly every pair of SMs and no more, no part below 16 blocks of K
  const int64_t dh_tiles = l.rows / TILE * l.d_tiles;
  l.splits = (int)std::max<int64_t>(1, std::min<int64_t>(74 / dh_tiles, l.piece / BK / 16));
  int64_t at = up((int64_t)sizeof(Head), 256);
  auto take = [&](int64_t bytes) { const int64_t a = at; at += up(bytes, 256); return a; };
  l.rank = take(N * 4); l.tok = take(l.rows * 4); l.coef = take(l.rows * 4); l.lse2 = take(l.rows * 4);
  l.h = take(l.rows * l.ld * 2);
  if (!backward) { l.part = take(l.rows * l.n_tiles * 8); l.z_tok = take(l.rows * 4); }
  else { l.g = take(2 * l.rows * l.piece * 2); l.dh = take(l.splits * l.rows * d * 4); }
  l.bytes = at;
  return l;
}

cudaError_t ready(int* sms) {
  static std::mutex mu;
  static int known_dev = -1, known = 0;
  int dev = 0;
  cudaGetDevice(&dev);
  std::lock_guard<std::mutex> lock(mu);
  if (known_dev != dev) {
    cudaError_t e = cudaFuncSetAttribute(tiles_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&known, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    known_dev = dev;
  }
  *sms = known;
  return cudaSuccess;
}

cudaError_t launch_gather(const Rows& r, int sms, cudaStream_t st) {
  const int64_t blocks = std::min<int64_t>((r.in.N + 7) / 8, 2 * sms);
  const int per = (int)((r.in.N + blocks - 1) / blocks);
  return launch_pdl(gather_kernel, dim3((unsigned)((r.in.N + per - 1) / per)), GT, 0, st, true, r, per);
}

// The tensor cores cut where float32 units round: a sum that takes n additions of 16 products ends n 2^-26 of itself nearer to 0, on average.  So it was measured, for sums of dense rows of
// 256 to 8192 features and logits of 0.5 to 20 (with 0.75 and 1.25 times as much made up for, something is left in all of them), and it holds to 8 % up to 65536 features.  What is cut off is between nothing (sums that
// need no rounding, of sparse rows say: they come out that much too large) and some twice that or more (terms that are all of one sign): the factor is the middle of a fault that goes one way, not its bound.
// (Losses of 2560 features against 64 bits, as a share: 1.2e-6 without it or with twice as much, 4.6e-7 with; float32 units 4.3e-7.)
double one_over_tau(const saki_linear_in& in) { return (1.0 + (in.d + 15) / 16 * 0x1p-26) / (double)in.temperature; }
float factor(const saki_linear_in& in) { return (float)(INV_LN2 * one_over_tau(in)); }      // of the products

Rows rows_of(const saki_linear_in& in, const float* lse, char* s, const Layout& l) {
  Rows r = {};
  r.in = in; r.lse = lse; r.head = (Head*)s;
  r.rank = (int*)(s + l.rank); r.tok = (int*)(s + l.tok); r.coef = (float*)(s + l.coef); r.lse2 = (float*)(s + l.lse2);
  r.h = (__nv_bfloat16*)(s + l.h); r.ld = l.ld;
  r.to_base2 = (double)factor(in) / one_over_tau(in);
  r.vec = ((uintptr_t)in.hidden & 15) == 0 && in.ld_h % 8 == 0;
  return r;
}
Tiles tiles_of(const Rows& r, const Layout& l, long long wait_limit) {
  Tiles t = {};
  t.head = r.head; t.d = r.in.d; t.V = r.in.V; t.d_tiles = l.d_tiles; t.n_tiles = l.n_tiles;
  t.wait_limit = wait_limit > 0 ? wait_limit : WAIT_LIMIT_CYCLES;
  t.c = factor(r.in);
  t.tok = r.tok; t.coef = r.coef; t.lse2 = r.lse2;
  return t;
}

}  // namespace

}  // namespace lin

int64_t linear_scratch_bytes(int64_t N, int32_t d, int32_t V, bool backward) { return lin::layout(N, d, V, backward).bytes; }

cudaError_t launch_linear_fwd(const saki_linear_in& in, const saki_linear_out& out, void* scratch, unsigned long long* flagged, long long wait_limit, int* n_launches,
                              cudaStream_t st) {
  using namespace lin;
  int sms = 0;
  cudaError_t e = ready(&sms);
  if (e != cudaSuccess) return e;
  const Layout l = layout(in.N, in.d, in.V, false);
  char* const s = (char*)scratch;
  const Rows r = rows_of(in, nullptr, s, l);
  Maps maps = {};
  if (!make_map(&maps.h_k, r.h, l.rows, in.d, l.ld, HALF) || !make_map(&maps.w_k, in.weight, in.V, in.d, in.ld_w, HALF)) return cudaErrorInvalidValue;
  maps.h_mn = maps.w_mn = maps.g_k = maps.g_mn = maps.g_out = maps.dw_out = maps.dh_out = maps.h_k;      // (not used)
  e = launch_gather(r, sms, st);
  if (e != cudaSuccess) return e;
  Tiles t = tiles_of(r, l, wait_limit);
  t.launch = -1;
  t.l_tiles = l.n_tiles;
  t.part = (float2*)(s + l.part); t.z_tok = (float*)(s + l.z_tok);
  const int pairs = std::min(sms, MAX_CTAS) / 2;
  const int64_t tiles = l.rows / TILE * l.n_tiles;
  e = launch_pdl_cluster(tiles_kernel, dim3((unsigned)(2 * std::min<int64_t>(pairs, tiles))), THREADS, 2, SMEM, st, maps, t);
  if (e != cudaSuccess) return e;
  *n_launches = 3;
  return launch_pdl(loss_kernel, dim3((unsigned)((in.N + 7) / 8)), 256, 0, st, true, r, out, (const float2*)t.part, (const float*)t.z_tok, l.n_tiles, t.c, one_over_tau(in), flagged);
}

cudaError_t launch_linear_bwd(const saki_linear_in& in, const float* lse, void* dhidden, int64_t ld_dh, void* dweight, int64_t ld_dw, float grad_scale, void* scratch,
                              long long wait_limit, int* n_launches, cudaStream_t st) {
  using namespace lin;
  int sms = 0;
  cudaError_t e = ready(&sms);
  if (e != cudaSuccess) return e;
  const Layout l = layout(in.N, in.d, in.V, true);
  char* const s = (char*)scratch;
  const Rows r = rows_of(in, lse, s, l);
  __nv_bfloat16* const g[2] = {(__nv_bfloat16*)(s + l.g), (__nv_bfloat16*)(s + l.g) + l.rows * l.piece};
  Maps maps[2];
  for (int b = 0; b < 2; ++b)
    if (!make_map(&maps[b].h_k, r.h, l.rows, in.d, l.ld, HALF) || !make_map(&maps[b].w_k, in.weight, in.V, in.d, in.ld_w, HALF) ||
        !make_map(&maps[b].h_mn, r.h, l.rows, in.d, l.ld, BK) || !make_map(&maps[b].w_mn, in.weight, in.V, in.d, in.ld_w, BK) ||
        !make_map(&maps[b].g_k, g[b], l.rows, l.piece, l.piece, HALF) || !make_map(&maps[b].g_mn, g[b], l.rows, l.piece, l.piece, BK) ||
        !make_map(&maps[b].g_out, g[b ^ 1], l.rows, l.piece, l.piece, 32) || !make_map(&maps[b].dh_out, s + l.dh, l.rows * l.splits, in.d, in.d, 32, true) ||
        !make_map(&maps[b].dw_out, dweight ? dweight : (void*)g[b], dweight ? in.V : 32, dweight ? in.d : 64, dweight ? ld_dw : 64, 32)) return cudaErrorInvalidValue;
  e = launch_gather(r, sms, st);
  if (e != cudaSuccess) return e;
  Tiles t = tiles_of(r, l, wait_limit);
  t.scale = (float)((double)grad_scale / (double)in.temperature);
  t.splits = l.splits; t.rows = (int)l.rows; t.grad = 1;
  t.dh = dhidden != nullptr; t.dw = dweight != nullptr;
  const int pairs = std::min(sms, MAX_CTAS) / 2;
  auto columns = [&](int p) { return std::min(l.piece / TILE, l.n_tiles - p * (l.piece / TILE)); };
  for (int p = 0; p <= l.pieces; ++p) {      // the logits of piece p, the products of piece p - 1
    t.launch = p > 0 ? p : -1;
    t.l_tiles = p < l.pieces ? columns(p) : 0; t.v0 = p * l.piece;
    t.b_tiles = p > 0 ? columns(p - 1) : 0; t.b0 = (p - 1) * l.piece; t.first = p == 1;
    const int64_t tiles = l.rows / TILE * t.l_tiles + (int64_t)t.b_tiles * l.d_tiles * t.dw + (t.dh && p > 0 ? l.rows / TILE * l.d_tiles * l.splits : 0);
    e = launch_pdl_cluster(tiles_kernel, dim3((unsigned)(2 * std::min<int64_t>(pairs, tiles))), THREADS, 2, SMEM, st, maps[(p + 1) & 1], t);
    if (e != cudaSuccess) return e;
  }
  *n_launches = l.pieces + 3;
  const int lanes = l.splits >= 8 ? 8 : 1;
  const int64_t threads = in.N * (in.d / 8) * lanes;
  return launch_pdl(lanes == 8 ? dhidden_kernel<8> : dhidden_kernel<1>, dim3((unsigned)std::min<int64_t>((threads + 255) / 256, 8 * sms)), 256, 0, st, true, r, (const float*)(s + l.dh),
                    l.rows * in.d, l.splits, t.scale, (__nv_bfloat16*)dhidden, ld_dh, (__nv_bfloat16*)dweight, ld_dw);
}

}  // namespace saki
