// Orthogonalisation of a matrix by Newton-Schulz products, and the local Muon step built on it.
//
// From X_0 = G / (||G||_F + eps) (all singular values in [0, 1]) each step applies the odd polynomial
// p(s) = a s + b s^3 + c s^5 to the singular values:
//   A = X X',   X <- a X + (b A + c A^2) X          (on the short side, m <= n).
//
// Rounding.  The products run on fp16 operands (11 significant bits, fp32 accumulation); X itself is
// carried as value + remainder (22 bits) and the linear term uses both.  Small singular values grow by a factor a
// in every step (3.4445^5 = 485), and only through the linear term: rounding X to 11 bits there would
// lift the rounding noise of large directions into empty ones (fp16 simulation, 512 x 1024 of rank 8:
// 4e-2 of the result's norm; bfloat16 0.35), while rounding inside B X stays in proportion to B X
// (7e-4 to 1.6e-3 on Gaussian, 1/k, exponentially decaying, rank-8 and spiked spectra).  With
// ABS_NS_F32 every operand is hi + lo and a product is three tensor-core products (fp32-grade).
#include <math.h>

#include "abs_ns.cuh"

namespace absk {
namespace {

constexpr int kTile = 64;
constexpr int kPassThreads = 256;
constexpr int kTileVecs = kTile * kTile / 4 / kPassThreads;     // groups of four elements per thread

// Momentum update (Muon) and partial sums of squares in fp64 (no overflow, no lost small entries).
// V = 4: every group of four elements is 16-byte aligned and lies in one row.
template <int V>
__global__ void __launch_bounds__(kPassThreads)
ns_norm_kernel(const NsSource s, int q0, double* __restrict__ part, unsigned* __restrict__ progress, int counters,
               unsigned* flag) {
  __shared__ double red[kPassThreads / 32];
  const int z = blockIdx.y;
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x == 0 && z == 0 && threadIdx.x == 0 && q0 == 0) *flag = 0u;
  if (blockIdx.x == 0)
    for (int k = threadIdx.x; k < counters; k += kPassThreads) progress[z * counters + k] = 0u;
  const long long base = matrix_base(q0 + z, s.L, s.replica_stride, s.matrix_stride);
  const bool flat = s.row_stride == s.cols;                    // one row of rows * cols elements
  const int per_row = s.cols / V;
  const long long count = static_cast<long long>(s.rows) * per_row;
  double sum = 0.0;
  for (long long e = static_cast<long long>(blockIdx.x) * kPassThreads + threadIdx.x; e < count;
       e += static_cast<long long>(gridDim.x) * kPassThreads) {
    long long i = base;
    if (flat) {
      i += e * V;
    } else {
      const long long r = e / per_row;
      i += r * s.row_stride + (e - r * per_row) * V;
    }
    float u[V];
    load_src<V>(s, i, u);
    if (s.muon) {
      float b[V];
      load_f32<V>(s.Buf + i, b);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        b[k] = fmaf(s.momentum, b[k], u[k]);
        u[k] = s.nesterov ? fmaf(s.momentum, b[k], u[k]) : b[k];
      }
      store_f32<V>(s.Buf + i, b);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) sum = fma(static_cast<double>(u[k]), static_cast<double>(u[k]), sum);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kPassThreads / 32; ++w) sum += red[w];
    part[static_cast<long long>(z) * kNormParts + blockIdx.x] = sum;
  }
}

// X_0 = U / (||U||_F + eps), scaled by sx, as hi + lo, transposed where U is taller than wide.  A CTA
// takes a 64 x 64 tile of U; a warp reads and writes whole rows of it, four elements a lane.
template <int V>
__global__ void __launch_bounds__(kPassThreads, 6)
ns_split_kernel(const NsSource s, int q0, const NsBuffers w, int parts, float eps, float sx, int tiles_c) {
  __shared__ float tile[kTile][kTile + 1];
  __shared__ double red[kPassThreads / 32];
  const int z = blockIdx.y, tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  const bool tall = s.rows > s.cols;
  const int tr = static_cast<int>(blockIdx.x) / tiles_c, tc = static_cast<int>(blockIdx.x) - tr * tiles_c;
  const long long base = matrix_base(q0 + z, s.L, s.replica_stride, s.matrix_stride);
  float u[kTileVecs][4];
#pragma unroll
  for (int k = 0; k < kTileVecs; ++k) {
    const int r = tr * kTile + (tid >> 4) + 16 * k, c = tc * kTile + 4 * (tid & 15);
    const long long i = base + static_cast<long long>(r) * s.row_stride + c;
#pragma unroll
    for (int e = 0; e < 4; e += V) {
      float t[V];
#pragma unroll
      for (int x = 0; x < V; ++x) t[x] = 0.f;
      if (r < s.rows && c + e < s.cols) load_update<V>(s, i + e, t);
#pragma unroll
      for (int x = 0; x < V; ++x) u[k][e + x] = t[x];
    }
  }
  double sum = 0.0;
  for (int k = tid; k < parts; k += kPassThreads) sum += w.part[static_cast<long long>(z) * kNormParts + k];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if ((tid & 31) == 0) red[tid >> 5] = sum;
  if (tall) {
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[4 * (tid & 15) + e][(tid >> 4) + 16 * k] = u[k][e];
  }
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int k = 0; k < kPassThreads / 32; ++k) sum += red[k];
  // fp64: a tiny norm's inverse may pass the range of fp32
  const double scale = static_cast<double>(sx) / (sqrt(sum) + static_cast<double>(eps));
  const long long zoff = z * w.ldx * w.m;
#pragma unroll
  for (int k = 0; k < kTileVecs; ++k) {
    const int ri = (tid >> 4) + 16 * k, cj = 4 * (tid & 15);
    const int i = (tall ? tc : tr) * kTile + ri, j = (tall ? tr : tc) * kTile + cj;      // row and column of X
    if (i >= w.m || j >= w.n) continue;                        // ldx is a multiple of 64: four columns stay in the row
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = static_cast<float>((tall ? tile[ri][cj + e] : u[k][e]) * scale);
    const __half2 h[2] = {__floats2half2_rn(x[0], x[1]), __floats2half2_rn(x[2], x[3])};
    const long long o = zoff + static_cast<long long>(i) * w.ldx + j;
    *reinterpret_cast<uint2*>(w.xh[0] + o) = *reinterpret_cast<const uint2*>(h);
    const float2 f0 = __half22float2(h[0]), f1 = __half22float2(h[1]);
    const __half2 l[2] = {__floats2half2_rn(x[0] - f0.x, x[1] - f0.y), __floats2half2_rn(x[2] - f1.x, x[3] - f1.y)};
    *reinterpret_cast<uint2*>(w.xl[0] + o) = *reinterpret_cast<const uint2*>(l);
  }
}

// O = X / sx back in the caller's orientation: the result, or the parameter update.
template <int V, bool MUON>
__global__ void __launch_bounds__(kPassThreads, MUON ? 5 : 6)
ns_finish_kernel(const NsSource s, const NsTarget t, int q0, const NsBuffers w, int cur, int low, float inv_sx, int tiles_c,
                 const unsigned* flag) {
  __shared__ float tile[kTile][kTile + 1];
  const int z = blockIdx.y, tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  const bool tall = s.rows > s.cols;
  const int tr = static_cast<int>(blockIdx.x) / tiles_c, tc = static_cast<int>(blockIdx.x) - tr * tiles_c;
  const long long zoff = z * w.ldx * w.m;
  const float bad = *flag ? __int_as_float(0x7fc00000) : 0.f;          // a product whose wait ran out: nothing is valid
  // Every load before the first store, which may be to the same place as far as the compiler knows, and few enough
  // registers for five or six CTAs an SM: 32 of 768 x 768 in 34 us (Muon 49), without 51 (56).  (At five the Muon kernel has 48
  // registers and spills 108 bytes a thread, with single elements 16; the times are with that.)
  const long long base = matrix_base(q0 + z, s.L, t.replica_stride, t.matrix_stride);
  float x0[kTileVecs][4];
#pragma unroll
  for (int k = 0; k < kTileVecs; ++k) {
    const int r = tr * kTile + (tid >> 4) + 16 * k, c = tc * kTile + 4 * (tid & 15);
#pragma unroll
    for (int e = 0; e < 4; e += V) {
      float x[V];
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = 0.f;
      if (MUON && r < s.rows && c + e < s.cols) load_f32<V>(t.X + base + static_cast<long long>(r) * t.row_stride + c + e, x);
#pragma unroll
      for (int v = 0; v < V; ++v) x0[k][e + v] = x[v];
    }
  }
  float u[kTileVecs][4];
#pragma unroll
  for (int k = 0; k < kTileVecs; ++k) {
    const int ri = (tid >> 4) + 16 * k, cj = 4 * (tid & 15);
    const int i = (tall ? tc : tr) * kTile + ri, j = (tall ? tr : tc) * kTile + cj;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < w.m && j < w.n) {
      const long long o = zoff + static_cast<long long>(i) * w.ldx + j;
      const uint2 h = *reinterpret_cast<const uint2*>((cur ? w.xh[1] : w.xh[0]) + o), l = *reinterpret_cast<const uint2*>((low ? w.xl[1] : w.xl[0]) + o);
      const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&h.x)), l0 = __half22float2(*reinterpret_cast<const __half2*>(&l.x));
      const float2 h1 = __half22float2(*reinterpret_cast<const __half2*>(&h.y)), l1 = __half22float2(*reinterpret_cast<const __half2*>(&l.y));
      x = make_float4(h0.x + l0.x, h0.y + l0.y, h1.x + l1.x, h1.y + l1.y);
    }
    u[k][0] = x.x * inv_sx + bad;
    u[k][1] = x.y * inv_sx + bad;
    u[k][2] = x.z * inv_sx + bad;
    u[k][3] = x.w * inv_sx + bad;
    if (tall) {
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[cj + e][ri] = u[k][e];
    }
  }
  if (tall) __syncthreads();
#pragma unroll
  for (int k = 0; k < kTileVecs; ++k) {
    const int ri = (tid >> 4) + 16 * k, cj = 4 * (tid & 15);
    const int r = tr * kTile + ri, c = tc * kTile + cj;
    if (r >= s.rows) continue;
    const long long i = base + static_cast<long long>(r) * t.row_stride + c;
    if (tall) {
#pragma unroll
      for (int e = 0; e < 4; ++e) u[k][e] = tile[ri][cj + e];
    }
#pragma unroll
    for (int e = 0; e < 4; e += V) {
      if (c + e >= s.cols) continue;
      float v[V];
#pragma unroll
      for (int x = 0; x < V; ++x) v[x] = u[k][e + x];
      if (MUON) {
#pragma unroll
        for (int x = 0; x < V; ++x) v[x] = fmaf(-t.step, v[x], t.decay * x0[k][e + x]);
        store_f32<V>(t.X + i + e, v);
      } else if (t.dst_bf16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(t.O) + i + e;
        if constexpr (V == 4) {
          __nv_bfloat162 p[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
          *reinterpret_cast<uint2*>(o) = *reinterpret_cast<const uint2*>(p);
        } else {
          *o = __float2bfloat16_rn(v[0]);
        }
      } else {
        store_f32<V>(static_cast<float*>(t.O) + i + e, v);
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------
// Largest |p| on [0, hi] for p(s) = a s + b s^3 + c s^5, and for q(s) = b s^2 + c s^4.
double bound_poly(double a, double b, double c, double hi) {
  auto p = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
  double best = p(hi);
  // p'(s) = a + 3 b t + 5 c t^2 with t = s^2
  const double A = 5.0 * c, B = 3.0 * b;
  double roots[2];
  int n = 0;
  if (A != 0.0) {
    const double disc = B * B - 4.0 * A * a;
    if (disc >= 0.0) {
      roots[n++] = (-B + sqrt(disc)) / (2.0 * A);
      roots[n++] = (-B - sqrt(disc)) / (2.0 * A);
    }
  } else if (B != 0.0) {
    roots[n++] = -a / B;
  }
  for (int k = 0; k < n; ++k)
    if (roots[k] > 0.0 && roots[k] < hi * hi) best = fmax(best, p(sqrt(roots[k])));
  return best;
}
double bound_even(double b, double c, double hi) {
  auto q = [&](double t) { return fabs(t * (b + t * c)); };
  double best = q(hi * hi);
  if (c != 0.0) {
    const double t = -b / (2.0 * c);
    if (t > 0.0 && t < hi * hi) best = fmax(best, q(t));
  }
  return best;
}
// The largest power of two that keeps entries up to `bound` at or below 2^14.
float pow2_scale(double bound) { return static_cast<float>(exp2(floor(log2(16384.0 / fmax(bound, 1e-6))))); }

constexpr double kMaxSingular = 1024.0;

int validate_ns(abs_ctx* ctx, int count, long long rows, long long cols, const abs_ns_cfg* cfg) {
  if (cfg == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "cfg is null");
  if (count < 1 || rows < 1 || cols < 1)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need at least one matrix of at least 1 x 1 (count=%d rows=%lld cols=%lld)",
                     count, rows, cols);
  if (cfg->steps < 1 || cfg->steps > kNsMaxSteps)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "steps must be 1..%d, got %d", kNsMaxSteps, cfg->steps);
  if (cfg->precision != ABS_NS_F16 && cfg->precision != ABS_NS_F32)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown precision %d", cfg->precision);
  if (!(cfg->eps >= 0.f) || !isfinite(cfg->eps) || !isfinite(cfg->a) || !isfinite(cfg->b) || !isfinite(cfg->c))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "coefficients must be finite and eps finite and >= 0");
  if (rows > 65536 || cols > 65536 || count > (1 << 24))
    return set_error(ctx, ABS_ERR_UNSUPPORTED, "matrices are at most 65536 x 65536 and 2^24 in number");
  return ABS_OK;
}

long long align_up(long long v, long long a) { return (v + a - 1) / a * a; }

struct NsPlan {
  int m, n;
  long long ldx, ldm, x_halves, m_halves;    // per matrix
  bool split;
  size_t per_matrix() const {
    return static_cast<size_t>((split ? 4 : 3) * x_halves + (split ? 4 : 2) * m_halves) * 2 + kNormParts * sizeof(double) +
           static_cast<size_t>(3 * ns_row_blocks(m)) * sizeof(unsigned);
  }
};
constexpr size_t kNsFixedBytes = 16 * 1024;       // alignment of the (at most ten) buffers
// Matrices that are worked on together.  More of them hide the waits between products, fewer keep what a step
// reads and writes inside L2 (126 MB).  us with groups of 100, 200, 300 and 600 MB: 96 matrices of 768 x 768 1320, 1303,
// 1310, 1326; 28 of them 450, 394, 394, 420; 16 of 2048 x 2048 2723, 2528, 2624, 2578.
constexpr size_t kGroupBytes = 200ull << 20;

NsPlan plan_ns(long long rows, long long cols, const abs_ns_cfg* cfg) {
  NsPlan p;
  p.m = static_cast<int>(rows < cols ? rows : cols);
  p.n = static_cast<int>(rows < cols ? cols : rows);
  p.ldx = align_up(p.n, 64);      // rows of whole 128-byte lines: 8 of 784 x 1024 44 us a step in pairs, 48 with rows of 8 halves
  p.ldm = align_up(p.m, 64);
  p.x_halves = p.ldx * p.m;
  p.m_halves = p.ldm * p.m;
  // Up to 64 rows the operands are split at either precision: with few rows the roundings of 11 bits do
  // not average out (simulated, worst of 200 Gaussian matrices: 2 x 2 1.8e-2, 4 x 4 6.5e-3, 10 x 1024
  // 2e-3), and a product of one row tile is bound by latency, not by its three tensor-core products.
  // (Most such matrices are small ones, whose operands are always split.)
  p.split = cfg->precision == ABS_NS_F32 || p.m <= 64;
  return p;
}
// Matrices worked on together where `bytes` of scratch hold them: groups of about the same size, so that 36 matrices with room
// for 35 are two groups of 18.
int group_size(const NsPlan& p, int count, size_t bytes) {
  long long z = static_cast<long long>((bytes < kGroupBytes ? bytes : kGroupBytes) / p.per_matrix());
  if (z < 1) z = 1;
  if (z > 65535) z = 65535;
  const long long groups = (count + z - 1) / z;
  return static_cast<int>((count + groups - 1) / groups);
}
// What the call asks for.  One group's size is not monotone in the number of matrices (35 of 768 x 768 207 MB, 36 106 MB),
// so any call takes what it gets from one matrix's up, in smaller groups: scratch for some number serves every smaller one.
size_t scratch_need(const NsPlan& p, int count) {
  const int cluster = ns_small_cluster(count, p.m, p.n);
  // Everything stays in shared memory.  (Larger clusters may have to take the general path.)
  if (cluster > 0 && cluster <= kPortableCluster) return kNsFixedBytes;
  return kNsFixedBytes + group_size(p, count, kGroupBytes) * p.per_matrix();
}

// Whether four consecutive elements of a row can be moved at once everywhere (strides that are not used
// are zero).
bool vectors_of_four(const void* p, int bf16, long long row_stride, long long matrix_stride, long long replica_stride, int cols) {
  return (reinterpret_cast<uintptr_t>(p) & (bf16 ? 7u : 15u)) == 0 &&
         ((row_stride | matrix_stride | replica_stride | static_cast<long long>(cols)) & 3) == 0;
}

int run_ns(abs_ctx* ctx, const NsSource& src, const NsTarget& dst, int count, const abs_ns_cfg* cfg, void* scratch,
           size_t scratch_bytes, cudaStream_t st) {
  const NsPlan p = plan_ns(src.rows, src.cols, cfg);
  const int cluster = ns_small_cluster(count, src.rows, src.cols);
  const bool small = cluster > 0 && ns_small_resident(ctx, cluster);
  const size_t least = kNsFixedBytes + (small ? 0 : p.per_matrix());
  if (scratch == nullptr || scratch_bytes < least)
    return set_error(ctx, ABS_ERR_WORKSPACE, "scratch of %zu bytes is too small: at least %zu needed", scratch_bytes, least);
  const int zmax = group_size(p, count, scratch_bytes - kNsFixedBytes);
  // scales of the stored matrices, from bounds on the singular values step by step
  NsScales sc;
  double hi = 1.0;
  for (int k = 0; k < cfg->steps; ++k) {
    sc.sx[k] = pow2_scale(hi);
    sc.ta[k] = pow2_scale(hi * hi);
    sc.tb[k] = pow2_scale(bound_even(cfg->b, cfg->c, hi));
    hi = bound_poly(cfg->a, cfg->b, cfg->c, hi);
    if (!(hi <= kMaxSingular))
      return set_error(ctx, ABS_ERR_UNSUPPORTED, "the coefficients let singular values grow beyond %g in step %d",
                       kMaxSingular, k + 1);
  }
  sc.sx[cfg->steps] = pow2_scale(hi);

  if (small)
    return launch_ns_small(ctx, src, dst, count, cfg->eps, sc, cfg->steps, cfg->a, cfg->b, cfg->c, st);
  const bool src_vec = vectors_of_four(src.G, src.src_bf16, src.row_stride, src.matrix_stride, src.replica_stride, src.cols) &&
                       vectors_of_four(src.Buf, 0, src.row_stride, src.matrix_stride, src.replica_stride, src.cols);
  const bool dst_vec = vectors_of_four(src.muon ? static_cast<const void*>(dst.X) : dst.O, dst.dst_bf16, dst.row_stride, dst.matrix_stride,
                                       dst.replica_stride, src.cols);
  const int tiles_c = (src.cols + kTile - 1) / kTile, tiles_r = (src.rows + kTile - 1) / kTile;
  for (int q0 = 0; q0 < count; q0 += zmax) {
    NsBuffers w = {};
    w.Z = count - q0 < zmax ? count - q0 : zmax;
    w.m = p.m; w.n = p.n; w.ldx = p.ldx; w.ldm = p.ldm;
    uintptr_t at = reinterpret_cast<uintptr_t>(scratch);
    auto take = [&](size_t bytes) {
      at = (at + 1023) / 1024 * 1024;
      void* r = reinterpret_cast<void*>(at);
      at += bytes;
      return r;
    };
    const size_t xb = static_cast<size_t>(p.x_halves) * zmax * 2, mb = static_cast<size_t>(p.m_halves) * zmax * 2;
    for (int k = 0; k < 2; ++k) {
      w.xh[k] = static_cast<__half*>(take(xb));
      if (p.split || k == 0) w.xl[k] = static_cast<__half*>(take(xb));
    }
    w.ah = static_cast<__half*>(take(mb));
    w.bh = static_cast<__half*>(take(mb));
    if (p.split) {
      w.al = static_cast<__half*>(take(mb));
      w.bl = static_cast<__half*>(take(mb));
    }
    w.part = static_cast<double*>(take(static_cast<size_t>(zmax) * kNormParts * sizeof(double)));
    w.progress = static_cast<unsigned*>(take(static_cast<size_t>(zmax) * 3 * ns_row_blocks(p.m) * sizeof(unsigned)));

    unsigned* flag = ctx->flags + kNsFlagWord;
    // enough CTAs to fill the GPU, at least four groups of elements per thread
    const long long vecs = static_cast<long long>(src.rows) * src.cols / 4;
    long long parts = (static_cast<long long>(ctx->sm_count) * 8 + w.Z - 1) / w.Z;
    if (parts > vecs / (4 * kPassThreads)) parts = vecs / (4 * kPassThreads);
    if (parts < 1) parts = 1;
    if (parts > kNormParts) parts = kNormParts;
    ABS_CUDA_TRY(ctx, launch_dependent(src_vec ? ns_norm_kernel<4> : ns_norm_kernel<1>, dim3(static_cast<unsigned>(parts), w.Z),
                                       dim3(kPassThreads), 0, st, src, q0, w.part, w.progress, 3 * ns_row_blocks(p.m), flag));
    const dim3 tiles(static_cast<unsigned>(tiles_c) * tiles_r, w.Z);
    ABS_CUDA_TRY(ctx, launch_dependent(src_vec ? ns_split_kernel<4> : ns_split_kernel<1>, tiles, dim3(kPassThreads), 0, st, src,
                                       q0, w, static_cast<int>(parts), cfg->eps, sc.sx[0], tiles_c));
    const int rc = launch_ns_steps(ctx, w, cfg->steps, cfg->a, cfg->b, cfg->c, sc, p.split, st);
    if (rc != ABS_OK) return rc;
    const int cur = cfg->steps & 1;
    auto finish = src.muon ? (dst_vec ? ns_finish_kernel<4, true> : ns_finish_kernel<1, true>)
                           : (dst_vec ? ns_finish_kernel<4, false> : ns_finish_kernel<1, false>);
    ABS_CUDA_TRY(ctx, launch_dependent(finish, tiles, dim3(kPassThreads), 0, st, src, dst, q0, w, cur, p.split ? cur : 0,
                                       1.0f / sc.sx[cfg->steps], tiles_c, static_cast<const unsigned*>(flag)));
  }
  return ABS_OK;
}

struct DeviceGuardNs {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuardNs(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuardNs() { if (prev >= 0) cudaSetDevice(prev); }
};

}  // namespace
}  // namespace absk

using namespace absk;

extern "C" int abs_ns_scratch_bytes(int count, long long rows, long long cols, const abs_ns_cfg* cfg, size_t* out) {
  if (out == nullptr) return ABS_ERR_INVALID_ARG;
  *out = 0;
  const int rc = validate_ns(nullptr, count, rows, cols, cfg);
  if (rc != ABS_OK) return rc;
  const NsPlan p = plan_ns(rows, cols, cfg);
  *out = scratch_need(p, count);
  return ABS_OK;
}

extern "C" int abs_orthogonalise(abs_ctx* ctx, const void* G, abs_dtype g_dtype, int count, long long rows, long long cols,
                                 long long g_row_stride, long long g_matrix_stride, void* O, abs_dtype o_dtype,
                                 long long o_row_stride, long long o_matrix_stride, const abs_ns_cfg* cfg, void* scratch,
                                 size_t scratch_bytes, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  const int rc = validate_ns(ctx, count, rows, cols, cfg);
  if (rc != ABS_OK) return rc;
  if (G == nullptr || O == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "G or O is null");
  if ((g_dtype != ABS_F32 && g_dtype != ABS_BF16) || (o_dtype != ABS_F32 && o_dtype != ABS_BF16))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype");
  if (g_row_stride < cols || o_row_stride < cols ||
      (count > 1 && (g_matrix_stride < (rows - 1) * g_row_stride + cols || o_matrix_stride < (rows - 1) * o_row_stride + cols)))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "rows or matrices overlap: check the strides");
  DeviceGuardNs guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  NsSource s = {};
  s.G = G; s.src_bf16 = g_dtype == ABS_BF16; s.L = count; s.matrix_stride = g_matrix_stride;
  s.row_stride = g_row_stride; s.rows = static_cast<int>(rows); s.cols = static_cast<int>(cols);
  NsTarget t = {};
  t.O = O; t.dst_bf16 = o_dtype == ABS_BF16; t.matrix_stride = o_matrix_stride; t.row_stride = o_row_stride;
  return run_ns(ctx, s, t, count, cfg, scratch, scratch_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int local_muon_step(abs_ctx* ctx, float* X, float* Buf, const float* Gb, int M, int matrices, long long rows,
                               long long cols, long long matrix_stride, long long replica_stride, const abs_muon_cfg* cfg,
                               int average_after, void* scratch, size_t scratch_bytes, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (cfg == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "cfg is null");
  if (M < 1 || matrices < 1 || static_cast<long long>(M) * matrices > (1 << 24))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need M >= 1 and matrices >= 1 (M=%d matrices=%d)", M, matrices);
  int rc = validate_ns(ctx, M * matrices, rows, cols, &cfg->ns);
  if (rc != ABS_OK) return rc;
  if (X == nullptr || Buf == nullptr || Gb == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "null tensor pointer");
  if (!(cfg->momentum >= 0.f && cfg->momentum < 1.f) || !isfinite(cfg->lr) || !isfinite(cfg->weight_decay) || !isfinite(cfg->scale))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need momentum in [0, 1) and finite lr, weight_decay and scale");
  const long long size = rows * cols;
  if (matrices > 1 && matrix_stride < size)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "matrix_stride %lld < rows * cols %lld", matrix_stride, size);
  if (M > 1 && replica_stride < (matrices > 1 ? (matrices - 1) * matrix_stride : 0) + size)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "replica_stride %lld overlaps the previous replica", replica_stride);
  DeviceGuardNs guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  NsSource s = {};
  s.G = Gb; s.Buf = Buf; s.momentum = cfg->momentum; s.nesterov = cfg->nesterov ? 1 : 0; s.muon = 1; s.L = matrices;
  s.replica_stride = replica_stride; s.matrix_stride = matrix_stride; s.row_stride = cols;
  s.rows = static_cast<int>(rows); s.cols = static_cast<int>(cols);
  NsTarget t = {};
  t.X = X;
  t.decay = static_cast<float>(1.0 - static_cast<double>(cfg->lr) * cfg->weight_decay);
  t.step = static_cast<float>(static_cast<double>(cfg->lr) * cfg->scale);
  t.replica_stride = replica_stride; t.matrix_stride = matrix_stride; t.row_stride = cols;
  rc = run_ns(ctx, s, t, M * matrices, &cfg->ns, scratch, scratch_bytes, static_cast<cudaStream_t>(stream));
  if (rc != ABS_OK || !average_after || M == 1) return rc;
  if (matrices == 1 || matrix_stride == size) return replica_average(ctx, X, M, size * matrices, replica_stride, stream);
  for (int l = 0; l < matrices; ++l) {
    rc = replica_average(ctx, X + l * matrix_stride, M, size, replica_stride, stream);
    if (rc != ABS_OK) return rc;
  }
  return ABS_OK;
}
