// Newton-Schulz orthogonalisation and the Muon step of small matrices (short side m <= 128) in one launch:
// momentum update, norm, all steps and the result, one thread-block cluster per matrix.
//
// X stays in shared memory as value + remainder (two fp16 numbers, 22 bits); a CTA of the cluster has up to
// 256 of its columns (192 or 128 where A and the partial sums leave no room for more).  A step is three tcgen05 products
// with a barrier after each: the time is latency, not arithmetic, so every product has split operands
// (hi hi + hi lo + lo hi, fp32-grade) whatever precision is asked for.
//   A = X X'          K-major rows of X twice; the CTAs' partial sums are added over the cluster, in rank order: every CTA
//                     receives all of them or, where that is too much, adds its share of the elements and sends it to all
//   B = b A + c A A   every CTA for itself, in the place of A
//   X <- a X + B X    every CTA its own columns; X is MN-major here, in the same memory
// The rows of X are padded with zeros to 64 or 128, A has 128 rows.  The waits for products are bounded; when one runs out
// the results of the matrix are NaN.  The cluster barriers have no limit of their own: every CTA of a cluster reaches each of
// them, whether or not a wait of its own ran out before.
//
// Measured (B200): a step takes 1.7 us for one 8 x 8 matrix, 4.5 for 4 of 64 x 192, 3.7 for 8 of 10 x 1024 (8 CTAs each),
// 13 for 8 of 128 x 512 (5 of them the exchange of 64 KB a CTA over the cluster); what is not steps (launch, momentum, norm,
// result) 6 to 14 us.  A call of 5 steps takes 32.7 us on 4 of 64 x 192 (a Muon step 32.8) and 28.7 on 8 of 10 x 1024; with
// the launches of the general path (norm, split, steps, finish) the Muon step took 101 and the orthogonalisation 147.
#include "abs_ns.cuh"
#include "abs_pipeline.cuh"

namespace absk {
namespace {

constexpr int kWarpsS = 16;
constexpr int kThreadsS = kWarpsS * 32;
constexpr int kMaxCluster = 16;      // (beyond 8 by the non-portable attribute)
constexpr int kTogether = 8;         // CTAs whose sums a thread fetches together
constexpr size_t kSmallSmem = 224 * 1024;      // dynamic shared memory, at most
constexpr int kBatch = 2;            // groups of eight elements that a thread loads at a time

struct SmallParams {
  NsSource s;
  NsTarget t;
  int m, n;            // short and long side
  int R;               // rows of the stored matrices: 64 or 128
  int W;               // columns of a CTA
  int C;               // CTAs of a cluster
  int steps;
  float eps, sx, inv_sx;
  long long timeout_cycles;
  int gather;          // every CTA sends its partial sums of A to all (else: two-part exchange)
  int vec_src, vec_dst;   // groups of eight are 16-byte aligned in global memory
  int drop;            // test hook: no product is issued, so the first wait must run out
  NsCoef coef[kNsMaxSteps][3];
};

// ---- PTX ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void tcs_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcs_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_s() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_cluster_s() { asm volatile("fence.proxy.async.shared::cluster;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync_s() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void umma_s(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_s(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Sixteen columns of this thread's lane from each of the two accumulators, added.
__device__ __forceinline__ void tmem_ld16_sum(uint32_t main, uint32_t cross, float (&v)[2][8]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(main), "r"(cross)
      : "memory");
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e >> 3][e & 7] = __uint_as_float(r[e]) + __uint_as_float(r[16 + e]);
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, float (&v)[2][8]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e >> 3][e & 7] = __uint_as_float(r[e]);
}
__device__ __forceinline__ void sts128_s(uint32_t addr, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void st_cluster128(uint32_t addr, const uint32_t (&v)[4]) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
               : "memory");
}
__device__ __forceinline__ float4 ld_cluster128(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ unsigned ld_cluster_u32(uint32_t addr) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// Byte offset of the 16-byte chunk that holds columns 8 ch .. 8 ch + 7 of row r in a matrix stored as blocks of
// 64 columns, `block` bytes apart, with the 128-byte swizzle.  The same memory is K-major (columns are k: 8-row
// groups 1024 bytes apart) and MN-major (rows are k).
__device__ __forceinline__ uint32_t chunk_at(uint32_t block, int r, int ch) {
  return static_cast<uint32_t>(ch >> 3) * block + static_cast<uint32_t>(r) * 128u +
         ((static_cast<uint32_t>(ch & 7) ^ static_cast<uint32_t>(r & 7)) << 4);
}
__device__ __forceinline__ void split8(const float (&v)[8], uint32_t (&h)[4], uint32_t (&l)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 hv = __floats2half2_rn(v[2 * e], v[2 * e + 1]);
    const float2 f = __half22float2(hv);
    const __half2 lv = __floats2half2_rn(v[2 * e] - f.x, v[2 * e + 1] - f.y);
    h[e] = *reinterpret_cast<const uint32_t*>(&hv);
    l[e] = *reinterpret_cast<const uint32_t*>(&lv);
  }
}
__device__ __forceinline__ void join8(const uint4 h, const uint4 l, float (&x)[8]) {
  const uint32_t hh[4] = {h.x, h.y, h.z, h.w}, ll[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hh[e]));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&ll[e]));
    x[2 * e] = a.x + b.x;
    x[2 * e + 1] = a.y + b.y;
  }
}

// y <- in y + acc w for two chunks of a row, stored to `copies` rows copy_rows apart; both chunks are loaded before the
// first is used (one alone takes 260 clocks from its load to its store).
__device__ __forceinline__ void apply16(uint32_t yh, uint32_t yl, uint32_t block, int row, int ch, float acc, float in,
                                        float (&w)[2][8], int copies, int copy_rows) {
  const uint32_t o[2] = {chunk_at(block, row, ch), chunk_at(block, row, ch + 1)};
  const uint4 h0 = lds128(yh + o[0]), l0 = lds128(yl + o[0]), h1 = lds128(yh + o[1]), l1 = lds128(yl + o[1]);
  float x[2][8];
  join8(h0, l0, x[0]);
  join8(h1, l1, x[1]);
  uint32_t h[2][4], l[2][4];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[k][e] = fmaf(acc, w[k][e], in * x[k][e]);
    split8(w[k], h[k], l[k]);
  }
#pragma unroll 1
  for (int c = 0; c < copies; ++c) {                             // (the swizzle is the same: copy_rows is a multiple of 8)
    const uint32_t to = static_cast<uint32_t>(c * copy_rows) * 128u;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      sts128_s(yh + o[k] + to, h[k]);
      sts128_s(yl + o[k] + to, l[k]);
    }
  }
}

// n <= 8 consecutive elements of a matrix in global memory (zeros behind them); vec: 16-byte aligned.
__device__ __forceinline__ void load8(const float* p, int n, bool vec, float (&v)[8]) {
  if (vec && n == 8) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int n, bool vec, float (&v)[8]) {
  if (vec && n == 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? __bfloat162float(p[e]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, int n, bool vec, const float (&v)[8]) {
  if (vec && n == 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = v[e];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, int n, bool vec, const float (&v)[8]) {
  if (vec && n == 8) {
    __nv_bfloat162 w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = __float2bfloat16_rn(v[e]);
  }
}
// Eight 16-bit values to or from a stored matrix: a chunk of row o, or rows 8 g .. 8 g + 7 of column o (the first n).
__device__ __forceinline__ void put8(uint32_t matrix, uint32_t block, bool tall, int o, int g, int n, const uint32_t (&v)[4]) {
  if (!tall) {
    sts128_s(matrix + chunk_at(block, o, g), v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e < n)
      asm volatile("st.shared.b16 [%0], %1;" ::"r"(matrix + chunk_at(block, 8 * g + e, o >> 3) + 2u * static_cast<uint32_t>(o & 7)),
                   "h"(static_cast<unsigned short>(e & 1 ? v[e >> 1] >> 16 : v[e >> 1]))
                   : "memory");
  }
}
__device__ __forceinline__ void get8(uint32_t matrix, uint32_t block, bool tall, int o, int g, uint32_t (&v)[4]) {
  if (!tall) {
    const uint4 a = lds128(matrix + chunk_at(block, o, g));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {                                  // (rows up to the next multiple of eight are there)
    unsigned short a, b;
    const uint32_t at = 2u * static_cast<uint32_t>(o & 7);
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(a) : "r"(matrix + chunk_at(block, 8 * g + 2 * e, o >> 3) + at));
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(b) : "r"(matrix + chunk_at(block, 8 * g + 2 * e + 1, o >> 3) + at));
    v[e] = static_cast<uint32_t>(a) | (static_cast<uint32_t>(b) << 16);
  }
}

// CLUSTER: several CTAs a matrix.  (A kernel of its own for one CTA: what it does not need is not in its way; 4 of
// 64 x 192 32.8 us, 41.0 with one kernel for both.)
template <bool CLUSTER>
__global__ void __launch_bounds__(kThreadsS, 1)
ns_small_kernel(const __grid_constant__ SmallParams p) {
  extern __shared__ unsigned char smem_dyn[];
  __shared__ double red[kWarpsS];
  __shared__ double norm_sq;
  __shared__ unsigned long long bar_mem;
  __shared__ unsigned abort_mem, tmem_slot;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int C = CLUSTER ? p.C : 1, R = p.R;
  const int q = blockIdx.x / C, rank = static_cast<int>(blockIdx.x) - q * C;     // matrix, place in its cluster
  const int c0 = rank * p.W, wc = p.n - c0 < p.W ? p.n - c0 : p.W;               // this CTA's columns
  const int Nm = (p.m + 15) & ~15, Nw = (wc + 15) & ~15;
  const int blocks = (p.W + 63) / 64, mblocks = (p.m + 63) / 64;
  const uint32_t block_bytes = static_cast<uint32_t>(R) * 128u;
  const uint32_t raw = smem_u32(smem_dyn), base = (raw + 1023u) & ~1023u;
  // X: a block's values, its remainders, the next block's values, ...; A: values, remainders
  const uint32_t x_block = 2u * block_bytes, a_block = 128u * 128u;
  const uint32_t xh = base, xl = xh + block_bytes, ah = xh + blocks * x_block, al = ah + mblocks * a_block;
  // partial sums (C > 1): one matrix [m][Nm + 4] fp32, or two sets of one of every CTA
  const uint32_t part = al + mblocks * a_block;
  const uint32_t pitch = static_cast<uint32_t>(Nm + 4) * 4u, part_bytes = static_cast<uint32_t>(p.m) * pitch;
  volatile unsigned* abort_flag = &abort_mem;
  const uint32_t bar = smem_u32(&bar_mem);
  const uint32_t cross_off = p.W > 128 ? 256u : 128u, tmem_cols = 2u * cross_off;
  if (tid == 0) {
    mbar_init(bar, 1);
    abort_mem = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // zero X and A (the pad rows and columns stay zero)
  for (uint32_t o = tid * 16u; o < blocks * x_block + 2u * mblocks * a_block; o += kThreadsS * 16u) {
    const uint32_t z[4] = {0u, 0u, 0u, 0u};
    sts128_s(xh + o, z);
  }
  tcs_before();
  __syncthreads();
  tcs_after();
  const uint32_t tmem = tmem_slot;

  // ---- momentum update and norm, then X_0 ------------------------------------------------------------
  // This CTA's part of U goes to X's place in groups of eight elements that are consecutive in U: of columns, or, where
  // U is taller than wide, of rows of X.  (Element by element, at some 120 instructions each, the passes over the matrix
  // took longer than two steps.)
  const bool tall = p.s.rows > p.s.cols;
  const int groups = ((tall ? p.m : wc) + 7) / 8, lines = tall ? wc : p.m, units = groups * lines;
  auto unit = [&](int u, int& o, int& g, int& n) {               // line, group of eight in it and elements of that
    if (tall) {                                                  // lanes next to one another: columns of X
      g = u / lines;
      o = u - g * lines;
      n = p.m - 8 * g;
    } else {
      o = u / groups;
      g = u - o * groups;
      n = wc - 8 * g;
    }
    if (n > 8) n = 8;
  };
  auto in_matrix = [&](int o, int g, long long row_stride) {
    return (tall ? c0 + o : o) * row_stride + (tall ? 0 : c0) + 8 * g;
  };
  const long long src = matrix_base(q, p.s.L, p.s.replica_stride, p.s.matrix_stride);
  double sum = 0.0;
#pragma unroll 1
  for (int u0 = tid; u0 < units; u0 += kBatch * kThreadsS) {
    int o[kBatch], g[kBatch], n[kBatch];
    float u[kBatch][8], b[kBatch][8];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      n[x] = 0;
      if (u0 + x * kThreadsS >= units) continue;
      unit(u0 + x * kThreadsS, o[x], g[x], n[x]);
      const long long at = src + in_matrix(o[x], g[x], p.s.row_stride);
      if (p.s.src_bf16) load8(static_cast<const __nv_bfloat16*>(p.s.G) + at, n[x], p.vec_src, u[x]);
      else load8(static_cast<const float*>(p.s.G) + at, n[x], p.vec_src, u[x]);
      if (p.s.muon) load8(p.s.Buf + at, n[x], p.vec_src, b[x]);
    }
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      if (n[x] == 0) continue;
      if (p.s.muon) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          b[x][e] = fmaf(p.s.momentum, b[x][e], u[x][e]);
          u[x][e] = p.s.nesterov ? fmaf(p.s.momentum, b[x][e], u[x][e]) : b[x][e];
        }
        store8(p.s.Buf + src + in_matrix(o[x], g[x], p.s.row_stride), n[x], p.vec_src, b[x]);
      }
      uint32_t hi[4], lo[4];                                     // as it is for now: upper and lower halves of fp32
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(u[x][e]), static_cast<double>(u[x][e]), sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t f = __float_as_uint(u[x][2 * e]), s2 = __float_as_uint(u[x][2 * e + 1]);
        hi[e] = __byte_perm(f, s2, 0x7632);
        lo[e] = __byte_perm(f, s2, 0x5410);
      }
      put8(xh, x_block, tall, o[x], g[x], n[x], hi);
      put8(xl, x_block, tall, o[x], g[x], n[x], lo);
    }
  }
  sum = warp_sum(sum);
  if (lane == 0) red[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    sum = 0.0;
    for (int w = 0; w < kWarpsS; ++w) sum += red[w];
    norm_sq = sum;
  }
  if constexpr (CLUSTER) cluster_sync_s();
  else __syncthreads();
  sum = 0.0;
  if constexpr (CLUSTER) {
    for (int r = 0; r < C; ++r) sum += ld_cluster_f64(map_to_rank(smem_u32(&norm_sq), static_cast<uint32_t>(r)));
  } else {
    sum = norm_sq;
  }
  const double scale = static_cast<double>(p.sx) / (sqrt(sum) + static_cast<double>(p.eps));
#pragma unroll 1
  for (uint32_t k = tid * 16u; k < blocks * block_bytes; k += kThreadsS * 16u) {
    const uint32_t o = k + (k & ~(block_bytes - 1u));            // blocks of values are x_block apart
    const uint4 a = lds128(xh + o), b = lds128(xl + o);
    const uint32_t hi[4] = {a.x, a.y, a.z, a.w}, lo[4] = {b.x, b.y, b.z, b.w};
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = static_cast<float>(__uint_as_float((hi[e] << 16) | (lo[e] & 0xffffu)) * scale);
      v[2 * e + 1] = static_cast<float>(__uint_as_float((hi[e] & 0xffff0000u) | (lo[e] >> 16)) * scale);
    }
    uint32_t h[4], l[4];
    split8(v, h, l);
    sts128_s(xh + o, h);
    sts128_s(xl + o, l);
  }

  // ---- steps ---------------------------------------------------------------------------------------------
  // instruction descriptor: fp32 accumulator, fp16 operands, MN-major second operand (bit 16), N, M = 128; operand
  // descriptors: 128-byte swizzle, 8-row groups 1024 bytes apart, MN-major blocks of 64 columns block_bytes apart
  const uint32_t idesc0 = (1u << 4) | (8u << 24);
  const uint64_t desc_k = (1ull << 46) | (64ull << 32) | (2ull << 61) | (1ull << 16);
  const uint64_t desc_mn = (1ull << 46) | (64ull << 32) | (2ull << 61) | (static_cast<uint64_t>(x_block >> 4) << 16);
  const uint32_t cross = tmem + cross_off;
  uint32_t phase = 0;
  // The products of split operands over K: hi hi into the main accumulator, lo hi and hi lo (2^-11 of it) into one of
  // their own.  `first` and `second` (its descriptor: desc_b) are the addresses of the values, remainders are
  // first_l and second_l bytes behind.  16 of K are 32 bytes of the first operand and step_b bytes of the second; blocks of
  // 64 of K are first_block and second_block bytes apart.  One thread issues them all, so its
  // instructions count: the descriptors of a block are made once.
  auto products = [&](uint32_t first, uint32_t first_l, uint32_t first_block, uint64_t desc_b, uint32_t second, uint32_t second_l,
                      uint32_t step_b, uint32_t second_block, uint32_t idesc, int K) {
    uint64_t dah = desc_k | ((first & 0x3ffffu) >> 4), dal = dah + (first_l >> 4);
    uint64_t dbh = desc_b | ((second & 0x3ffffu) >> 4), dbl = dbh + (second_l >> 4);
#pragma unroll 1
    for (int k0 = 0; k0 < K; k0 += 64) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k0 + 16 * k >= K) break;
        const uint64_t sa = 2u * k, sb = static_cast<uint64_t>(step_b >> 4) * k;
        umma_s(tmem, dah + sa, dbh + sb, idesc, (k0 | k) ? 1u : 0u);
        umma_s(cross, dal + sa, dbh + sb, idesc, (k0 | k) ? 1u : 0u);
        umma_s(cross, dah + sa, dbl + sb, idesc, 1u);
      }
      dah += first_block >> 4;
      dal += first_block >> 4;
      dbh += second_block >> 4;
      dbl += second_block >> 4;
    }
    umma_commit_s(bar);
  };
  // X X' where X's remainders lie 64 rows behind its values: hi hi and hi lo are one product of twice the width.  One of up
  // to 128 columns costs 61 clocks (what the first operand's 128 rows take to fetch), so two of
  // them are a third faster than three: 10 x 1024 on 4 CTAs 2200 clocks, 2950.
  // Columns 128 .. 255 have an accumulator of their own: the tensor core does not round its sums to nearest, and shorter ones
  // are nearer (4 of 64 x 256, error against 64 bits 2.0e-6 with one, 1.8e-6 with two, plain fp32 1.2e-6).
  auto gram_products = [&](uint32_t idesc) {
    const uint32_t wide = idesc + (64u >> 3 << 17);
    uint64_t dh = desc_k | ((xh & 0x3ffffu) >> 4), dl = dh + (block_bytes >> 4);
#pragma unroll 1
    for (int k0 = 0; k0 < Nw; k0 += 64) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k0 + 16 * k >= Nw) break;
        umma_s(tmem + (k0 < 128 ? 0u : 128u), dh + 2u * k, dh + 2u * k, wide, ((k0 & 127) | k) ? 1u : 0u);
        umma_s(cross, dl + 2u * k, dh + 2u * k, idesc, (k0 | k) ? 1u : 0u);
      }
      dh += x_block >> 4;
      dl += x_block >> 4;
    }
    umma_commit_s(bar);
  };
  auto wait_products = [&]() {
    mbar_wait(bar, phase & 1u, abort_flag, p.timeout_cycles);
    ++phase;
    __syncwarp();
    tcs_after();
  };
  // The products read what every thread wrote to shared memory and overwrite the accumulators that every warp read.
  auto before_products = [&]() {
    fence_proxy_s();
    tcs_before();
    __syncthreads();
    tcs_after();
  };
  const int q4 = warp & 3, group = warp >> 2;                    // rows of this warp, its share of the chunks
  const int row = q4 * 32 + lane;
  const uint32_t t_row = static_cast<uint32_t>(q4 * 32) << 16;
  const bool live = q4 * 32 < p.m;                               // (whole warps)
  // Up to 64 rows B's rows are stored two or four times, so that all 128 lanes of the accumulator hold
  // B X and every warp (its lanes are the rows q4 * 32 ...) has columns to bring back: 10 x 1024, 256 columns a CTA, 3900
  // clocks with one copy, 1250 with four.
  const int copies = p.m <= 32 ? 4 : p.m <= 64 ? 2 : 1, copy_rows = 128 / copies, quarters = 4 / copies;
  const int x_row = q4 % quarters * 32 + lane, x_share = q4 / quarters * 4 + group;
  const bool joined = R == 64;

  for (int step = 0; step < p.steps; ++step) {
    // A = X X'
    before_products();
    if (tid == 0 && !p.drop) {
      fence_proxy_s();
      const uint32_t idesc = idesc0 | (static_cast<uint32_t>(Nm >> 3) << 17);
      if (joined) gram_products(idesc);
      else products(xh, block_bytes, x_block, desc_k, xh, block_bytes, 32u, x_block, idesc, Nw);
    }
    wait_products();
    const NsCoef gram = p.coef[step][0], poly = p.coef[step][1], upd = p.coef[step][2];
    if (live) {
#pragma unroll 1
      for (int ch2 = 2 * group; ch2 < Nm / 8; ch2 += 8) {
        float w[2][8];
        tmem_ld16_sum(tmem + t_row + 8u * ch2, cross + t_row + 8u * ch2, w);
        if (joined) {
          float z[2][8];
          tmem_ld16(tmem + 64u + t_row + 8u * ch2, z);
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e >> 3][e & 7] += z[e >> 3][e & 7];
          if (Nw > 128) {
            tmem_ld16_sum(tmem + 128u + t_row + 8u * ch2, tmem + 192u + t_row + 8u * ch2, z);
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e >> 3][e & 7] += z[e >> 3][e & 7];
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int ch = ch2 + x;
          float (&v)[8] = w[x];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= gram.acc;
          if constexpr (CLUSTER) {
            if (row < p.m) {
              const uint32_t at = part + static_cast<uint32_t>(row) * pitch + 32u * ch;
              const uint32_t lo[4] = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
              const uint32_t hi[4] = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
              if (p.gather) {
                const uint32_t mine = at + static_cast<uint32_t>((step & 1) * C + rank) * part_bytes;
                for (int k = 0; k < C; ++k) {
                  const uint32_t to = map_to_rank(mine, static_cast<uint32_t>(k));
                  st_cluster128(to, lo);
                  st_cluster128(to + 16u, hi);
                }
              } else {
                sts128_s(at, lo);
                sts128_s(at + 16u, hi);
              }
            }
          } else if (row < R) {
            uint32_t h[4], l[4];
            split8(v, h, l);
            sts128_s(ah + chunk_at(a_block, row, ch), h);
            sts128_s(al + chunk_at(a_block, row, ch), l);
          }
        }
      }
    }
    if constexpr (CLUSTER) cluster_sync_s();
    if (CLUSTER && p.gather) {
      // A CTA may write a set of step s + 2 once it has passed the barrier of step s + 1, which every CTA reaches with
      // the set of step s read.
      const int per_row = Nm / 8;
#pragma unroll 1
      for (int u = tid; u < p.m * per_row; u += kThreadsS) {
        const int r = u / per_row, ch = u - r * per_row;
        const uint32_t at = part + static_cast<uint32_t>((step & 1) * C) * part_bytes + static_cast<uint32_t>(r) * pitch + 32u * ch;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = 0; k < C; ++k) {
          const uint4 a = lds128(at + static_cast<uint32_t>(k) * part_bytes), b = lds128(at + static_cast<uint32_t>(k) * part_bytes + 16u);
          v[0] += __uint_as_float(a.x); v[1] += __uint_as_float(a.y); v[2] += __uint_as_float(a.z); v[3] += __uint_as_float(a.w);
          v[4] += __uint_as_float(b.x); v[5] += __uint_as_float(b.y); v[6] += __uint_as_float(b.z); v[7] += __uint_as_float(b.w);
        }
        uint32_t h[4], l[4];
        split8(v, h, l);
        sts128_s(ah + chunk_at(a_block, r, ch), h);
        sts128_s(al + chunk_at(a_block, r, ch), l);
      }
    } else if constexpr (CLUSTER) {
      const int per_row = Nm / 8, all = p.m * per_row, share = (all + C - 1) / C, stop = (rank + 1) * share < all ? (rank + 1) * share : all;
#pragma unroll 1
      for (int u = rank * share + tid; u < stop; u += kThreadsS) {      // one after the other: 128 x 512 on 4 CTAs 10000 clocks, interleaved 19000
        const int r = u / per_row, ch = u - r * per_row;
        const uint32_t at = part + static_cast<uint32_t>(r) * pitch + 32u * ch;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int k0 = 0; k0 < C; k0 += kTogether) {
          float4 a[kTogether], b[kTogether];
#pragma unroll
          for (int k = 0; k < kTogether; ++k) {
            if (k0 + k >= C) continue;
            const uint32_t from = map_to_rank(at, static_cast<uint32_t>(k0 + k));
            a[k] = ld_cluster128(from);
            b[k] = ld_cluster128(from + 16u);
          }
#pragma unroll
          for (int k = 0; k < kTogether; ++k) {
            if (k0 + k >= C) continue;
            v[0] += a[k].x; v[1] += a[k].y; v[2] += a[k].z; v[3] += a[k].w;
            v[4] += b[k].x; v[5] += b[k].y; v[6] += b[k].z; v[7] += b[k].w;
          }
        }
        uint32_t h[4], l[4];
        split8(v, h, l);
        for (int k = 0; k < C; ++k) {
          st_cluster128(map_to_rank(ah + chunk_at(a_block, r, ch), static_cast<uint32_t>(k)), h);
          st_cluster128(map_to_rank(al + chunk_at(a_block, r, ch), static_cast<uint32_t>(k)), l);
        }
      }
      fence_proxy_cluster_s();
      cluster_sync_s();
    }
    // B = b A + c A A, in the place of A
    before_products();
    if (tid == 0 && !p.drop) {
      fence_proxy_s();
      products(ah, al - ah, a_block, desc_k, ah, al - ah, 32u, a_block, idesc0 | (static_cast<uint32_t>(Nm >> 3) << 17), Nm);
    }
    wait_products();
    if (live) {
#pragma unroll 1
      for (int ch2 = 2 * group; ch2 < Nm / 8; ch2 += 8) {
        float w[2][8];
        tmem_ld16_sum(tmem + t_row + 8u * ch2, cross + t_row + 8u * ch2, w);
        if (row < R) {
          apply16(ah, al, a_block, row, ch2, row < p.m ? poly.acc : 0.f, row < p.m ? poly.in : 0.f, w, copies, copy_rows);
        }
      }
    }
    // X <- a X + B X
    before_products();
    if (tid == 0 && !p.drop) {
      fence_proxy_s();
      const uint32_t idesc = idesc0 | (1u << 16) | (static_cast<uint32_t>(Nw >> 3) << 17);
      products(ah, al - ah, a_block, desc_mn, xh, block_bytes, 16u * 128u, 64u * 128u, idesc, Nm);      // (16 rows)
    }
    wait_products();
    if (q4 % quarters * 32 < p.m) {
#pragma unroll 1
      for (int ch2 = 2 * x_share; ch2 < Nw / 8; ch2 += 8 * copies) {
        float w[2][8];
        tmem_ld16_sum(tmem + t_row + 8u * ch2, cross + t_row + 8u * ch2, w);
        if (x_row < p.m) apply16(xh, xl, x_block, x_row, ch2, upd.acc, upd.in, w, 1, 0);
      }
    }
  }
  tcs_before();
  __syncthreads();
  if (warp == 0) {
    tcs_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
  }

  // ---- the result ------------------------------------------------------------------------------------------
  unsigned failed = abort_mem;
  if constexpr (CLUSTER) {
    cluster_sync_s();
    for (int r = 0; r < C; ++r) failed |= ld_cluster_u32(map_to_rank(smem_u32(&abort_mem), static_cast<uint32_t>(r)));
  }
  const float bad = failed ? __int_as_float(0x7fc00000) : 0.f;
  const long long dst = matrix_base(q, p.s.L, p.t.replica_stride, p.t.matrix_stride);
#pragma unroll 1
  for (int u0 = tid; u0 < units; u0 += kBatch * kThreadsS) {
    int o[kBatch], g[kBatch], n[kBatch];
    float x0[kBatch][8];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      n[x] = 0;
      if (u0 + x * kThreadsS >= units) continue;
      unit(u0 + x * kThreadsS, o[x], g[x], n[x]);
      if (p.s.muon) load8(p.t.X + dst + in_matrix(o[x], g[x], p.t.row_stride), n[x], p.vec_dst, x0[x]);
    }
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      if (n[x] == 0) continue;
      const long long at = dst + in_matrix(o[x], g[x], p.t.row_stride);
      uint32_t h[4], l[4];
      get8(xh, x_block, tall, o[x], g[x], h);
      get8(xl, x_block, tall, o[x], g[x], l);
      float v[8];
      join8(make_uint4(h[0], h[1], h[2], h[3]), make_uint4(l[0], l[1], l[2], l[3]), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = v[e] * p.inv_sx + bad;
        if (p.s.muon) v[e] = fmaf(-p.t.step, v[e], p.t.decay * x0[x][e]);
      }
      if (p.s.muon) store8(p.t.X + at, n[x], p.vec_dst, v);
      else if (p.t.dst_bf16) store8(static_cast<__nv_bfloat16*>(p.t.O) + at, n[x], p.vec_dst, v);
      else store8(static_cast<float*>(p.t.O) + at, n[x], p.vec_dst, v);
    }
  }
  if constexpr (CLUSTER) cluster_sync_s();                                   // a peer may still read this CTA's abort flag
}

struct SmallPlan {
  int R, W, C, gather;
  size_t smem;
};
// `narrow`: at most 128 columns a CTA.
bool plan_columns(int count, long long rows, long long cols, bool narrow, SmallPlan* out) {
  const int m = static_cast<int>(rows < cols ? rows : cols);
  const long long n = rows < cols ? cols : rows;
  if (m > 128 || n > 256 * kMaxCluster) return false;
  SmallPlan p;
  p.R = m <= 64 ? 64 : 128;
  const int Nm = (m + 15) & ~15;
  const size_t block = static_cast<size_t>(p.R) * 128, part = static_cast<size_t>(m) * (Nm + 4) * 4;
  // with 64 rows the products read 128 of X: behind the last block lies A
  auto smem = [&](int W) { return 1024 + 2 * (static_cast<size_t>((W + 63) / 64) * block + static_cast<size_t>((m + 63) / 64) * 16384); };
  int most = narrow ? 128 : 256;                                 // columns of a CTA that fit beside A and the partial sums
  while (most > 64 && smem(most) + (n > most ? part : 0) > kSmallSmem) most -= 64;
  const long long C = (n + most - 1) / most;
  // A cluster of more than 8 CTAs has a GPC of its own, so five to eight matrices are under way at a time.  5 steps there and
  // on the general path, us.  Up to 64 rows: 18 x 2474 (10 CTAs), 8 matrices 41, 253, 16 81, 263, 32 123, 298, 48 201, 333,
  // 64 245, 380; 64 x 4000 (16), 4 60, 355, 32 296, 464, 48 417, 544; 40 x 3000 (12), 32 240, 355, 64 477, 466: the limit
  // of 32 is below where the two meet (about 64).  Up to 128 rows: 86 x 2085 (11), 5 matrices 83, 130, 8 164, 134; 128 x 2048 (16),
  // 5 102, 127, 8 201, 131: the limit of 4 is below the first number that needs a second wave.
  if (C > kMaxCluster || (C > 8 && count > (m > 64 ? 4 : 32))) return false;
  p.C = static_cast<int>(C);                                     // with W as below every CTA has columns: n > (C - 1) W
  p.W = static_cast<int>(((n + C - 1) / C + 15) / 16 * 16);
  p.smem = smem(p.W);
  // Up to 20 KB of partial sums go to all CTAs, with one barrier a step; beyond that every CTA adds its share and sends it
  // on, with two.  us a step that way and the other: 10 x 1024 as it would be on 4 CTAs (3 KB) 3.9, 4.4; 32 x 500 on 2 (9 KB) 4.2, 4.9;
  // 32 x 1000 on 4 (18 KB) 4.7, 5.0; 24 x 1500 on 6 (20 KB) 5.1, 5.1; 48 x 1000 on 4 (39 KB) 6.8, 6.4.
  p.gather = p.C * part <= 20 * 1024;
  if (p.C > 1) p.smem += p.gather ? 2 * p.C * part : part;
  // One CTA per SM: two of them could want more tensor memory than there is, and a CTA that waits for it while
  // its cluster waits for the CTA would wait for good.
  if (p.smem < 120 * 1024) p.smem = 120 * 1024;
  *out = p;
  return true;
}
// With SMs to spare, CTAs of fewer columns, where there are several anyway, us wide and narrow: 8 of 10 x 1024 (8 CTAs for 4) 30.8,
// 28.7; of 64 x 1000 50, 42; of 100 x 700 (6 for 4) 73, 68; but 4 of 64 x 192 (2 for 1) 31.7, 35.4.  The limit of 64 CTAs is on the safe
// side of how many clusters fit at a time: 10 of 64 x 1000 (80) 50, 43, 16 (128) 50, 82; 10 of 100 x 700 (60) 73, 71, 16 (96) 74, 75;
// 20 of 64 x 640 (100, clusters of 5) 48, 41, 32 (160) 49, 80.
bool plan_small(int count, long long rows, long long cols, SmallPlan* out) {
  if (!plan_columns(count, rows, cols, false, out)) return false;
  SmallPlan narrow;
  if (out->C > 2 && plan_columns(count, rows, cols, true, &narrow) && narrow.C <= 8 && count * narrow.C <= 64) *out = narrow;
  return true;
}

}  // namespace

int ns_small_cluster(int count, long long rows, long long cols) {
  SmallPlan p;
  return plan_small(count, rows, cols, &p) ? p.C : 0;
}

// Whether the device can hold a cluster of that many CTAs (of a whole SM each); asked once.
bool ns_small_resident(abs_ctx* ctx, int cluster) {
  if (cluster <= kPortableCluster) return true;
  if (ctx->tuning.ns_max_cluster != 0 && cluster > ctx->tuning.ns_max_cluster) return false;
  if (ctx->ns_clusters[cluster] == 0) {
    auto kern = ns_small_kernel<true>;
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    lc.gridDim = dim3(static_cast<unsigned>(cluster));
    lc.blockDim = dim3(kThreadsS);
    lc.dynamicSmemBytes = kSmallSmem;
    lc.attrs = attr;
    lc.numAttrs = 1;
    int clusters = 0;
    const bool ok = ensure_dynamic_smem(ctx, kern, kSmallSmem) == cudaSuccess &&
                    cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&clusters, reinterpret_cast<const void*>(kern), &lc) == cudaSuccess && clusters > 0;
    if (!ok) cudaGetLastError();
    ctx->ns_clusters[cluster] = ok ? 1 : -1;
  }
  return ctx->ns_clusters[cluster] > 0;
}

int launch_ns_small(abs_ctx* ctx, const NsSource& s, const NsTarget& t, int count, float eps, const NsScales& sc, int steps,
                    float a, float b, float c, cudaStream_t st) {
  SmallPlan plan;
  if (!plan_small(count, s.rows, s.cols, &plan) || !ns_small_resident(ctx, plan.C)) return ABS_ERR_UNSUPPORTED;
  SmallParams p = {};
  p.s = s; p.t = t;
  p.m = s.rows < s.cols ? s.rows : s.cols;
  p.n = s.rows < s.cols ? s.cols : s.rows;
  p.R = plan.R; p.W = plan.W; p.C = plan.C; p.gather = plan.gather;
  auto aligned = [](const void* a, int es, long long rs, long long ms, long long ls) {
    return ((reinterpret_cast<uintptr_t>(a) | static_cast<uintptr_t>(rs * es) | static_cast<uintptr_t>(ms * es) | static_cast<uintptr_t>(ls * es)) & 15u) == 0;
  };
  p.vec_src = aligned(s.G, s.src_bf16 ? 2 : 4, s.row_stride, s.matrix_stride, s.replica_stride) &&
              aligned(s.Buf, 4, s.row_stride, s.matrix_stride, s.replica_stride);
  p.vec_dst = aligned(s.muon ? static_cast<const void*>(t.X) : t.O, !s.muon && t.dst_bf16 ? 2 : 4, t.row_stride, t.matrix_stride, t.replica_stride);
  p.steps = steps;
  p.eps = eps;
  p.sx = sc.sx[0];
  p.inv_sx = 1.0f / sc.sx[steps];
  p.timeout_cycles = ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles;
  p.drop = ctx->tuning.stats_fault_drop_loads ? 1 : 0;
  for (int k = 0; k < steps; ++k) ns_coefs(p.coef[k], a, b, c, sc, k);
  auto kern = plan.C > 1 ? ns_small_kernel<true> : ns_small_kernel<false>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, plan.smem));
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(plan.C);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  lc.gridDim = dim3(static_cast<unsigned>(count) * plan.C);
  lc.blockDim = dim3(kThreadsS);
  lc.dynamicSmemBytes = plan.smem;
  lc.stream = st;
  lc.attrs = attr;
  lc.numAttrs = 1;
  ABS_CUDA_TRY(ctx, cudaLaunchKernelEx(&lc, kern, p));
  return ABS_OK;
}

}  // namespace absk
