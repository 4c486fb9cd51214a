// Root-mean-square norm with the residual's addition, forward and backward, for the rows of M replicas with weights of their own.
//
//   h = x + r,  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w      (or e4m3 with one scale a row)
//   xh = h rstd,  a = w dy,  dx = dh + rstd (a - xh mean(a xh)),  dw = sum_rows dy xh
//
// Each pass must read its inputs and write its outputs once; the arithmetic (5 and 9 operations an element) is far below
// what the memory rate leaves time for.
#include <cuda_fp8.h>

#include "abs_pipeline.cuh"

namespace absk {
namespace {

constexpr int kRmsThreads = 256;
constexpr float kE4m3Max = 448.f;

struct Rows {
  const void* p;
  long long rs, ws;
};
struct RowsOut {
  void* p;
  long long rs, ws;
};
struct RmsForward {
  Rows x, r;
  RowsOut h, y, q;
  const float* weight;
  long long p_stride;
  float eps;
  float* scales;
  float* rstd;
  int M;
  long long rows;
  int d;
};
// The rows of all segments (samples, or all rows of a replica) are shared out in pieces of `chunk` rows, `chunks` to a
// segment; the sums of a piece over its rows go to part + (segment * chunks + piece) * d, or, with one piece a segment, to `out`.
struct RmsBackward {
  Rows dy, h, dh;
  const float* rstd;
  const float* weight;
  long long p_stride;
  RowsOut dx;
  int M;
  long long samples, tokens;           // segments of a replica and rows of a segment
  int d;
  long long chunk;
  int chunks;
  float* part;
  float* out;                          // segment i of replica m at m * o_ws + i * o_rs
  long long o_rs, o_ws;
};

template <typename T> __device__ __forceinline__ float widen1(T v);
template <> __device__ __forceinline__ float widen1<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen1<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T round1(float v);
template <> __device__ __forceinline__ float round1<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 round1<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  __syncthreads();                       // the previous use of red is over
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kRmsThreads / 32; ++w) s += red[w];
  return s;
}
__device__ __forceinline__ unsigned block_max(unsigned v, float* red) {
  v = __reduce_max_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = __uint_as_float(v);
  __syncthreads();
  unsigned s = 0u;
#pragma unroll
  for (int w = 0; w < kRmsThreads / 32; ++w) s = max(s, __float_as_uint(red[w]));
  return s;
}
// The largest magnitude of a row, as the bits of its absolute value: these order as whole numbers do, an infinity above every
// number and a NaN above that.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(unsigned top) {
  if (top == 0u) return 1.f;
  return top >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : __uint_as_float(top) / kE4m3Max;
}
__device__ __forceinline__ unsigned char e4m3(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// Any width, stride and alignment: one CTA per row, two sweeps over it (three for 8 bits).
template <typename T>
__global__ void __launch_bounds__(kRmsThreads)
rms_forward_any_kernel(const RmsForward a) {
  __shared__ float red[kRmsThreads / 32];
  pdl_wait();
  const long long total = a.rows * a.M;
  for (long long rr = blockIdx.x; rr < total; rr += gridDim.x) {
    const long long m = rr / a.rows, r = rr - m * a.rows;
    const T* x = static_cast<const T*>(a.x.p) + m * a.x.ws + r * a.x.rs;
    const T* res = a.r.p ? static_cast<const T*>(a.r.p) + m * a.r.ws + r * a.r.rs : nullptr;
    T* h = a.h.p ? static_cast<T*>(a.h.p) + m * a.h.ws + r * a.h.rs : nullptr;
    T* y = a.y.p ? static_cast<T*>(a.y.p) + m * a.y.ws + r * a.y.rs : nullptr;
    const float* w = a.weight ? a.weight + m * a.p_stride : nullptr;
    float s = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kRmsThreads) {
      T v = x[j];
      if (res) v = round1<T>(widen1<T>(v) + widen1<T>(res[j]));
      if (h) h[j] = v;
      const float f = widen1<T>(v);
      s = fmaf(f, f, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum(s, red) / static_cast<float>(a.d) + a.eps);
    // an element of the row as this thread read or wrote it
    auto again = [&](int j) {
      if (h) return widen1<T>(h[j]);
      return res ? widen1<T>(round1<T>(widen1<T>(x[j]) + widen1<T>(res[j]))) : widen1<T>(x[j]);
    };
    float scale = 1.f;
    if (a.q.p) {
      unsigned top = 0u;
      for (int j = threadIdx.x; j < a.d; j += kRmsThreads) top = max(top, magnitude(again(j) * rstd * (w ? w[j] : 1.f)));
      scale = scale_of(block_max(top, red));
      unsigned char* q = static_cast<unsigned char*>(a.q.p) + m * a.q.ws + r * a.q.rs;
      for (int j = threadIdx.x; j < a.d; j += kRmsThreads) q[j] = e4m3(again(j) * rstd * (w ? w[j] : 1.f) / scale);
    }
    if (y)
      for (int j = threadIdx.x; j < a.d; j += kRmsThreads) y[j] = round1<T>(again(j) * rstd * (w ? w[j] : 1.f));
    if (threadIdx.x == 0) {
      if (a.rstd) a.rstd[rr] = rstd;
      if (a.q.p) a.scales[rr] = scale;
    }
  }
}

// dx of any width, stride and alignment: one CTA per row, two sweeps.
template <typename T>
__global__ void __launch_bounds__(kRmsThreads)
rms_dx_any_kernel(const RmsBackward a) {
  __shared__ float red[kRmsThreads / 32];
  pdl_wait();
  const long long rows = a.samples * a.tokens, total = rows * a.M;
  for (long long rr = blockIdx.x; rr < total; rr += gridDim.x) {
    const long long m = rr / rows, r = rr - m * rows;
    const T* dy = static_cast<const T*>(a.dy.p) + m * a.dy.ws + r * a.dy.rs;
    const T* h = static_cast<const T*>(a.h.p) + m * a.h.ws + r * a.h.rs;
    const T* dh = a.dh.p ? static_cast<const T*>(a.dh.p) + m * a.dh.ws + r * a.dh.rs : nullptr;
    T* dx = static_cast<T*>(a.dx.p) + m * a.dx.ws + r * a.dx.rs;
    const float* w = a.weight ? a.weight + m * a.p_stride : nullptr;
    const float rstd = a.rstd[rr];
    float s = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kRmsThreads) s = fmaf(widen1<T>(dy[j]) * (w ? w[j] : 1.f), widen1<T>(h[j]) * rstd, s);
    const float c = block_sum(s, red) / static_cast<float>(a.d);
    for (int j = threadIdx.x; j < a.d; j += kRmsThreads) {
      const float g = widen1<T>(dy[j]) * (w ? w[j] : 1.f), xh = widen1<T>(h[j]) * rstd;
      dx[j] = round1<T>(fmaf(rstd, fmaf(-xh, c, g), dh ? widen1<T>(dh[j]) : 0.f));
    }
  }
}

// The sums of dw of any width, stride and alignment: a thread owns a column of one piece of a segment.
template <typename T>
__global__ void __launch_bounds__(kRmsThreads)
rms_weight_any_kernel(const RmsBackward a) {
  pdl_wait();
  const int col_tiles = (a.d + kRmsThreads - 1) / kRmsThreads;
  const long long jobs = static_cast<long long>(a.M) * a.samples * a.chunks;
  for (long long b = blockIdx.x; b < jobs * col_tiles; b += gridDim.x) {
    const long long job = b / col_tiles;
    const int j = static_cast<int>(b - job * col_tiles) * kRmsThreads + threadIdx.x;
    if (j >= a.d) continue;
    const long long seg = job / a.chunks, m = seg / a.samples, first = (job - seg * a.chunks) * a.chunk;
    const long long r0 = (seg - m * a.samples) * a.tokens + first;
    const long long n = a.tokens - first < a.chunk ? a.tokens - first : a.chunk;
    float s = 0.f;
    for (long long r = r0; r < r0 + n; ++r) {
      const float g = widen1<T>(static_cast<const T*>(a.dy.p)[m * a.dy.ws + r * a.dy.rs + j]);
      s = fmaf(g, widen1<T>(static_cast<const T*>(a.h.p)[m * a.h.ws + r * a.h.rs + j]) * a.rstd[m * a.samples * a.tokens + r], s);
    }
    if (a.part) a.part[job * a.d + j] = s;
    else a.out[m * a.o_ws + (seg - m * a.samples) * a.o_rs + j] = s;
  }
}

// Sums of rows: out[m][i] = sum_k in[m][i][k], `n` rows each, in a fixed order; eight lanes share them.
struct RmsSums {
  const float* in;
  long long in_ws, in_group, in_rs;      // replica, group of rows, row
  long long n;
  float* out;
  long long out_ws, out_group;
  int d;
};
__global__ void __launch_bounds__(kRmsThreads)
rms_sum_kernel(const RmsSums a) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const float* p = a.in + blockIdx.y * a.in_ws + blockIdx.z * a.in_group + col;
  pdl_wait();
  float s = 0.f;
  if (col < a.d) {
#pragma unroll 8
    for (long long k = row; k < a.n; k += 8) s += p[k * a.in_rs];
  }
  red[row][lane] = s;
  __syncthreads();
  if (row == 0 && col < a.d) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += red[k][lane];
    a.out[blockIdx.y * a.out_ws + blockIdx.z * a.out_group + col] = s;
  }
}
__global__ void __launch_bounds__(kRmsThreads)
rms_zero_kernel(float* p, long long ws, long long rs, long long n, int d) {
  pdl_wait();
  for (long long i = blockIdx.x; i < n; i += gridDim.x)
    for (int j = threadIdx.x; j < d; j += kRmsThreads) p[blockIdx.y * ws + i * rs + j] = 0.f;
}

struct DeviceGuardRms {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuardRms(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuardRms() { if (prev >= 0) cudaSetDevice(prev); }
};

int validate_rms_rows(abs_ctx* ctx, const char* what, int M, long long rows, long long d, long long rs, long long ws) {
  if (rs < d) return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: row_stride %lld < d %lld", what, rs, d);
  if (M > 1 && rows > 0 && ws < (rows - 1) * rs + d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: worker_stride %lld overlaps the previous worker", what, ws);
  return ABS_OK;
}
int validate_rms_shape(abs_ctx* ctx, abs_dtype dtype, int M, long long rows, long long d) {
  if (dtype != ABS_F32 && dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (M < 1 || rows < 0 || d < 1)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need M >= 1, rows >= 0 and d >= 1 (M=%d rows=%lld d=%lld)", M, rows, d);
  if (M > 65535 || d > (1 << 24) || rows > (1ll << 40))
    return set_error(ctx, ABS_ERR_UNSUPPORTED, "M <= 65535, d <= 2^24 and rows <= 2^40 (M=%d rows=%lld d=%lld)", M, rows, d);
  return ABS_OK;
}
unsigned rms_grid(const abs_ctx* ctx, long long work) {
  const long long most = static_cast<long long>(ctx->sm_count) * 64;
  return static_cast<unsigned>(work < most ? work : most);
}

// How a backward pass shares out its rows: pieces of a segment, as many as fill the GPU a few times and as the workspace has
// places for (none is needed with one piece a segment).
struct RmsPlan {
  long long samples, tokens, chunk;
  int chunks;
  long long groups, per_group;       // of the totals' sum: groups of segments that are summed first, segments of a group
  size_t sums_at;                    // floats in front of the groups' sums
};
RmsPlan plan_rms(int M, long long samples, long long tokens, long long d, bool per_sample, bool totals, long long jobs_wanted,
                 size_t workspace_bytes) {
  RmsPlan p = {};
  if (!per_sample) {
    tokens *= samples;
    samples = 1;
  }
  p.samples = samples;
  p.tokens = tokens;
  const long long room = static_cast<long long>(workspace_bytes / sizeof(float) / d);
  long long chunks = (jobs_wanted + samples * M - 1) / (samples * M);
  if (chunks > (tokens + 7) / 8) chunks = (tokens + 7) / 8;            // eight rows a piece at least
  if (chunks * samples * M > room) chunks = room / (samples * M);
  if (chunks < 1) chunks = 1;
  p.chunk = (tokens + chunks - 1) / chunks;
  if (p.chunk < 1) p.chunk = 1;
  p.chunks = static_cast<int>(tokens > 0 ? (tokens + p.chunk - 1) / p.chunk : 1);
  const long long used = p.chunks > 1 ? p.chunks * samples * M : 0;
  p.sums_at = static_cast<size_t>(used) * d;
  p.groups = 1;
  if (totals && per_sample && samples > 256) {
    p.groups = (samples + 127) / 128;
    if (p.groups > 1024) p.groups = 1024;
    if (p.groups * M > room - used) p.groups = (room - used) / M;
    if (p.groups < 1) p.groups = 1;
  }
  p.per_group = (samples + p.groups - 1) / p.groups;
  if (p.per_group < 1) p.per_group = 1;
  p.groups = samples > 0 ? (samples + p.per_group - 1) / p.per_group : 1;
  return p;
}

template <typename T>
int run_forward(abs_ctx* ctx, const RmsForward& a, cudaStream_t st) {
  ABS_CUDA_TRY(ctx, launch_dependent(rms_forward_any_kernel<T>, dim3(rms_grid(ctx, a.rows * a.M)), dim3(kRmsThreads), 0, st, a));
  return ABS_OK;
}
template <typename T>
int run_backward(abs_ctx* ctx, const RmsBackward& a, bool sums, cudaStream_t st) {
  if (sums) {                      // before dx, which may take the place of dy or h
    const long long work = static_cast<long long>(a.M) * a.samples * a.chunks * ((a.d + kRmsThreads - 1) / kRmsThreads);
    const long long most = 1 << 30;
    ABS_CUDA_TRY(ctx, launch_dependent(rms_weight_any_kernel<T>, dim3(static_cast<unsigned>(work < most ? work : most)), dim3(kRmsThreads), 0, st, a));
  }
  if (a.dx.p)
    ABS_CUDA_TRY(ctx, launch_dependent(rms_dx_any_kernel<T>, dim3(rms_grid(ctx, a.samples * a.tokens * a.M)), dim3(kRmsThreads), 0, st, a));
  return ABS_OK;
}

}  // namespace
}  // namespace absk

using namespace absk;

extern "C" int abs_rms_norm(abs_ctx* ctx, const void* X, abs_dtype dtype, int M, long long rows, long long d, long long x_row_stride,
                            long long x_worker_stride, const void* R, long long r_row_stride, long long r_worker_stride, void* H,
                            long long h_row_stride, long long h_worker_stride, const float* weight, long long param_stride, float eps,
                            void* Y, long long y_row_stride, long long y_worker_stride, void* Q, long long q_row_stride,
                            long long q_worker_stride, float* scales, float* rstd, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  int rc = validate_rms_shape(ctx, dtype, M, rows, d);
  if (rc != ABS_OK) return rc;
  if (!(eps >= 0.f) || eps > 3.0e38f) return set_error(ctx, ABS_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if ((Q == nullptr) != (scales == nullptr)) return set_error(ctx, ABS_ERR_INVALID_ARG, "Q and scales go together");
  if (rows == 0) return ABS_OK;
  if (X == nullptr || (Y == nullptr && Q == nullptr)) return set_error(ctx, ABS_ERR_INVALID_ARG, "X is null, or Y and Q are");
  if ((rc = validate_rms_rows(ctx, "X", M, rows, d, x_row_stride, x_worker_stride)) != ABS_OK) return rc;
  if (R && (rc = validate_rms_rows(ctx, "R", M, rows, d, r_row_stride, r_worker_stride)) != ABS_OK) return rc;
  if (H && (rc = validate_rms_rows(ctx, "H", M, rows, d, h_row_stride, h_worker_stride)) != ABS_OK) return rc;
  if (Y && (rc = validate_rms_rows(ctx, "Y", M, rows, d, y_row_stride, y_worker_stride)) != ABS_OK) return rc;
  if (Q && (rc = validate_rms_rows(ctx, "Q", M, rows, d, q_row_stride, q_worker_stride)) != ABS_OK) return rc;
  if (M > 1 && weight && param_stride != 0 && param_stride < d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "param_stride %lld < d %lld", param_stride, d);
  DeviceGuardRms guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  const RmsForward a{{X, x_row_stride, x_worker_stride}, {R, r_row_stride, r_worker_stride}, {H, h_row_stride, h_worker_stride},
                     {Y, y_row_stride, y_worker_stride}, {Q, q_row_stride, q_worker_stride}, weight, param_stride, eps, scales, rstd, M,
                     rows, static_cast<int>(d)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == ABS_F32 ? run_forward<float>(ctx, a, st) : run_forward<__nv_bfloat16>(ctx, a, st);
}

extern "C" int abs_rms_norm_backward(abs_ctx* ctx, const void* dY, long long dy_row_stride, long long dy_worker_stride, const void* H,
                                     long long h_row_stride, long long h_worker_stride, const void* dH, long long dh_row_stride,
                                     long long dh_worker_stride, abs_dtype dtype, int M, long long samples, long long tokens, long long d,
                                     const float* rstd, const float* weight, long long param_stride, void* dX, long long dx_row_stride,
                                     long long dx_worker_stride, float* dW, long long grad_stride, float* Gw, long long g_row_stride,
                                     long long g_worker_stride, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (samples < 0 || tokens < 0 || (tokens > 0 && samples > (1ll << 40) / tokens))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "samples and tokens must be >= 0 and their product <= 2^40");
  const long long rows = samples * tokens;
  int rc = validate_rms_shape(ctx, dtype, M, rows, d);
  if (rc != ABS_OK) return rc;
  if (rows > 0) {
    if (dY == nullptr || H == nullptr || rstd == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "dY, H or rstd is null");
    if ((rc = validate_rms_rows(ctx, "dY", M, rows, d, dy_row_stride, dy_worker_stride)) != ABS_OK) return rc;
    if ((rc = validate_rms_rows(ctx, "H", M, rows, d, h_row_stride, h_worker_stride)) != ABS_OK) return rc;
    if (dH && (rc = validate_rms_rows(ctx, "dH", M, rows, d, dh_row_stride, dh_worker_stride)) != ABS_OK) return rc;
    if (dX && (rc = validate_rms_rows(ctx, "dX", M, rows, d, dx_row_stride, dx_worker_stride)) != ABS_OK) return rc;
  }
  if (M > 1 && weight && param_stride != 0 && param_stride < d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "param_stride %lld < d %lld", param_stride, d);
  if (M > 1 && dW && grad_stride < d) return set_error(ctx, ABS_ERR_INVALID_ARG, "grad_stride %lld < d %lld", grad_stride, d);
  if (Gw && samples > 0 && (rc = validate_rms_rows(ctx, "Gw", M, samples, d, g_row_stride, g_worker_stride)) != ABS_OK) return rc;
  if (Gw && samples > (1ll << 31) / M) return set_error(ctx, ABS_ERR_UNSUPPORTED, "M * samples <= 2^31 with Gw");
  DeviceGuardRms guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool sums = Gw != nullptr || dW != nullptr;
  const unsigned col_tiles = static_cast<unsigned>((d + 31) / 32);
  if (rows == 0) {
    if (Gw && samples > 0)
      ABS_CUDA_TRY(ctx, launch_dependent(rms_zero_kernel, dim3(rms_grid(ctx, samples), M), dim3(kRmsThreads), 0, st, Gw, g_worker_stride,
                                         g_row_stride, samples, static_cast<int>(d)));
    if (dW)
      ABS_CUDA_TRY(ctx, launch_dependent(rms_zero_kernel, dim3(1, M), dim3(kRmsThreads), 0, st, dW, grad_stride, 0ll, 1ll, static_cast<int>(d)));
    return ABS_OK;
  }
  const RmsPlan p = plan_rms(M, samples, tokens, d, Gw != nullptr, dW != nullptr, ctx->sm_count * 8ll, ctx->workspace_bytes);
  RmsBackward a{{dY, dy_row_stride, dy_worker_stride}, {H, h_row_stride, h_worker_stride}, {dH, dh_row_stride, dh_worker_stride}, rstd,
                weight, param_stride, {dX, dx_row_stride, dx_worker_stride}, M, p.samples, p.tokens, static_cast<int>(d), p.chunk,
                p.chunks, nullptr, Gw ? Gw : dW, Gw ? g_row_stride : 0, Gw ? g_worker_stride : grad_stride};
  float* ws = static_cast<float*>(ctx->workspace);
  if (p.chunks > 1) a.part = ws;
  rc = dtype == ABS_F32 ? run_backward<float>(ctx, a, sums, st) : run_backward<__nv_bfloat16>(ctx, a, sums, st);
  if (rc != ABS_OK || !sums) return rc;
  if (p.chunks > 1) {              // pieces -> segments
    for (long long s0 = 0; s0 < p.samples; s0 += 32768) {
      const unsigned n = static_cast<unsigned>(p.samples - s0 < 32768 ? p.samples - s0 : 32768);
      const RmsSums q{ws + s0 * p.chunks * d, p.samples * p.chunks * d, static_cast<long long>(p.chunks) * d, d, p.chunks, a.out + s0 * a.o_rs,
                      a.o_ws, a.o_rs, static_cast<int>(d)};
      ABS_CUDA_TRY(ctx, launch_dependent(rms_sum_kernel, dim3(col_tiles, M, n), dim3(kRmsThreads), 0, st, q));
    }
  }
  if (Gw && dW) {                  // segments -> replica
    const long long tail = p.samples - (p.groups - 1) * p.per_group;
    if (p.groups == 1) {
      const RmsSums q{Gw, g_worker_stride, 0, g_row_stride, p.samples, dW, grad_stride, 0, static_cast<int>(d)};
      ABS_CUDA_TRY(ctx, launch_dependent(rms_sum_kernel, dim3(col_tiles, M), dim3(kRmsThreads), 0, st, q));
    } else {
      float* to = ws + p.sums_at;
      const RmsSums q{Gw, g_worker_stride, p.per_group * g_row_stride, g_row_stride, p.per_group, to, p.groups * d, d, static_cast<int>(d)};
      ABS_CUDA_TRY(ctx, launch_dependent(rms_sum_kernel, dim3(col_tiles, M, static_cast<unsigned>(p.groups - 1)), dim3(kRmsThreads), 0, st, q));
      const RmsSums t{Gw + (p.groups - 1) * p.per_group * g_row_stride, g_worker_stride, 0, g_row_stride, tail, to + (p.groups - 1) * d,
                      p.groups * d, 0, static_cast<int>(d)};
      ABS_CUDA_TRY(ctx, launch_dependent(rms_sum_kernel, dim3(col_tiles, M), dim3(kRmsThreads), 0, st, t));
      const RmsSums u{to, p.groups * d, 0, d, p.groups, dW, grad_stride, 0, static_cast<int>(d)};
      ABS_CUDA_TRY(ctx, launch_dependent(rms_sum_kernel, dim3(col_tiles, M), dim3(kRmsThreads), 0, st, u));
    }
  }
  return ABS_OK;
}
