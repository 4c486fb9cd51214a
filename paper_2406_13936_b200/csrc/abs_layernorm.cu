// Layer norm, forward and backward, for the rows of M replicas with parameters of their own.
//
//   xh = (x - mean) rstd,   y = xh w + b
//   a = w dy,   dx = rstd (a - mean_j(a) - xh mean_j(a xh)),   dw = sum_rows dy xh,   db = sum_rows dy
//
// Each pass must read its inputs and write its outputs once; the arithmetic (7 and 14 operations an
// element) is far below what the memory rate leaves time for.
#include "abs_pipeline.cuh"

namespace absk {
namespace {

constexpr int kLnThreads = 256;

struct LnForward {
  const void* X;
  long long x_rs, x_ws;
  const float* weight;
  const float* bias;
  long long p_stride;
  float eps;
  void* Y;
  long long y_rs, y_ws;
  float* mean;
  float* rstd;
  int M;
  long long rows;
  int d;
};
struct LnBackward {
  const void* dY;
  long long dy_rs, dy_ws;
  const void* X;
  long long x_rs, x_ws;
  const float* mean;
  const float* rstd;
  const float* weight;
  long long p_stride;
  void* dX;
  long long dx_rs, dx_ws;
  int M;
  long long samples, tokens;   // segments of a replica and rows of a segment
  int d;
  // sums of `rows_per_chunk` rows of a segment: part[((m * samples + i) * chunks + c) * 2d + {0, d} + j]
  float* part;
  int chunks;
  long long rows_per_chunk;
};
struct LnReduce {
  const float* part;
  int M;
  long long samples;
  int chunks, d;
  float* Gw;
  float* Gb;
  long long g_rs, g_ws;
  float* dW;
  float* dB;
  long long grad_stride;
};

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float2 block_sum2(float a, float b, float2* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, off);
    b += __shfl_xor_sync(0xffffffffu, b, off);
  }
  __syncthreads();                       // the previous use of red is over
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kLnThreads / 32; ++w) {
    s.x += red[w].x;
    s.y += red[w].y;
  }
  return s;
}

// Any width, stride and alignment: one CTA per row, three sweeps over it.
template <typename T>
__global__ void __launch_bounds__(kLnThreads)
ln_forward_any_kernel(const LnForward a) {
  __shared__ float2 red[kLnThreads / 32];
  pdl_wait();
  const long long total = a.rows * a.M;
  for (long long rr = blockIdx.x; rr < total; rr += gridDim.x) {
    const long long m = rr / a.rows, r = rr - m * a.rows;
    const T* x = static_cast<const T*>(a.X) + m * a.x_ws + r * a.x_rs;
    T* y = static_cast<T*>(a.Y) + m * a.y_ws + r * a.y_rs;
    const float inv_d = 1.0f / static_cast<float>(a.d);
    float s = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kLnThreads) s += to_f32<T>(x[j]);
    const float mean = block_sum2(s, 0.f, red).x * inv_d;
    float v = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kLnThreads) {
      const float c = to_f32<T>(x[j]) - mean;
      v = fmaf(c, c, v);
    }
    const float rstd = 1.0f / sqrtf(fmaf(block_sum2(v, 0.f, red).x, inv_d, a.eps));
    const float* w = a.weight ? a.weight + m * a.p_stride : nullptr;
    const float* b = a.bias ? a.bias + m * a.p_stride : nullptr;
    for (int j = threadIdx.x; j < a.d; j += kLnThreads) {
      const float xh = (to_f32<T>(x[j]) - mean) * rstd;
      y[j] = from_f32<T>(fmaf(xh, w ? w[j] : 1.f, b ? b[j] : 0.f));
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[rr] = mean;
      if (a.rstd) a.rstd[rr] = rstd;
    }
  }
}

// dx of any width, stride and alignment: one CTA per row, two sweeps.
template <typename T>
__global__ void __launch_bounds__(kLnThreads)
ln_dx_any_kernel(const LnBackward a) {
  __shared__ float2 red[kLnThreads / 32];
  pdl_wait();
  const long long rows = a.samples * a.tokens, total = rows * a.M;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (long long rr = blockIdx.x; rr < total; rr += gridDim.x) {
    const long long m = rr / rows, r = rr - m * rows;
    const T* x = static_cast<const T*>(a.X) + m * a.x_ws + r * a.x_rs;
    const T* dy = static_cast<const T*>(a.dY) + m * a.dy_ws + r * a.dy_rs;
    T* dx = static_cast<T*>(a.dX) + m * a.dx_ws + r * a.dx_rs;
    const float* w = a.weight ? a.weight + m * a.p_stride : nullptr;
    const float mean = a.mean[rr], rstd = a.rstd[rr];
    float s1 = 0.f, s2 = 0.f;
    for (int j = threadIdx.x; j < a.d; j += kLnThreads) {
      const float g = to_f32<T>(dy[j]) * (w ? w[j] : 1.f), xh = (to_f32<T>(x[j]) - mean) * rstd;
      s1 += g;
      s2 = fmaf(g, xh, s2);
    }
    const float2 s = block_sum2(s1, s2, red);
    const float c1 = s.x * inv_d, c2 = s.y * inv_d;
    for (int j = threadIdx.x; j < a.d; j += kLnThreads) {
      const float g = to_f32<T>(dy[j]) * (w ? w[j] : 1.f), xh = (to_f32<T>(x[j]) - mean) * rstd;
      dx[j] = from_f32<T>(rstd * (g - c1 - xh * c2));
    }
  }
}

// Partial sums of dw and db over one chunk of rows: a thread owns a column.
template <typename T>
__global__ void __launch_bounds__(kLnThreads)
ln_params_any_kernel(const LnBackward a) {
  pdl_wait();
  const int col_tiles = (a.d + kLnThreads - 1) / kLnThreads;
  const long long unit = blockIdx.x / col_tiles;                     // (m * samples + i) * chunks + c
  const int j = static_cast<int>(blockIdx.x - unit * col_tiles) * kLnThreads + threadIdx.x;
  const long long seg = unit / a.chunks, chunk = unit - seg * a.chunks;
  const long long m = seg / a.samples, i = seg - m * a.samples;
  const long long t0 = chunk * a.rows_per_chunk;
  const long long t1 = t0 + a.rows_per_chunk < a.tokens ? t0 + a.rows_per_chunk : a.tokens;
  if (j >= a.d) return;
  const long long rows = a.samples * a.tokens;
  float dw = 0.f, db = 0.f;
  for (long long t = t0; t < t1; ++t) {
    const long long r = i * a.tokens + t;
    const float g = to_f32<T>(static_cast<const T*>(a.dY)[m * a.dy_ws + r * a.dy_rs + j]);
    const float xh = (to_f32<T>(static_cast<const T*>(a.X)[m * a.x_ws + r * a.x_rs + j]) - a.mean[m * rows + r]) *
                     a.rstd[m * rows + r];
    dw = fmaf(g, xh, dw);
    db += g;
  }
  float* out = a.part + unit * 2 * a.d;
  out[j] = dw;
  out[a.d + j] = db;
}

// Chunks -> samples -> replica: 32 columns of one replica per CTA, 8 lanes of samples, fixed order.
__global__ void __launch_bounds__(kLnThreads)
ln_reduce_kernel(const LnReduce a) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;                            // column of [dw ; db]
  const long long m = blockIdx.y;
  pdl_wait();
  const bool live = col < 2 * a.d, is_b = col >= a.d;
  const int j = is_b ? col - a.d : col;
  float* G = is_b ? a.Gb : a.Gw;
  float total = 0.f;
  for (long long i = row; i < a.samples; i += 8) {
    const float* p = a.part + (m * a.samples + i) * a.chunks * 2 * a.d + col;
    float s = 0.f;
    if (live)
      for (int c = 0; c < a.chunks; ++c) s += p[static_cast<long long>(c) * 2 * a.d];
    if (live && G) G[m * a.g_ws + i * a.g_rs + j] = s;
    total += s;
  }
  red[row][lane] = total;
  __syncthreads();
  float* out = is_b ? a.dB : a.dW;
  if (row == 0 && live && out) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += red[k][lane];
    out[m * a.grad_stride + j] = s;
  }
}

struct DeviceGuardLn {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuardLn(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuardLn() { if (prev >= 0) cudaSetDevice(prev); }
};

int validate_rows(abs_ctx* ctx, const char* what, int M, long long rows, long long d, long long rs, long long ws) {
  if (rs < d) return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: row_stride %lld < d %lld", what, rs, d);
  if (M > 1 && rows > 0 && ws < (rows - 1) * rs + d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: worker_stride %lld overlaps the previous worker", what, ws);
  return ABS_OK;
}
int validate_shape(abs_ctx* ctx, abs_dtype dtype, int M, long long rows, long long d) {
  if (dtype != ABS_F32 && dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (M < 1 || rows < 0 || d < 1)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need M >= 1, rows >= 0 and d >= 1 (M=%d rows=%lld d=%lld)", M, rows, d);
  if (M > 65535 || d > (1 << 24) || rows > (1ll << 40))
    return set_error(ctx, ABS_ERR_UNSUPPORTED, "M <= 65535, d <= 2^24 and rows <= 2^40 (M=%d rows=%lld d=%lld)", M, rows, d);
  return ABS_OK;
}
unsigned row_grid(const abs_ctx* ctx, long long rows) {
  const long long most = static_cast<long long>(ctx->sm_count) * 64;
  return static_cast<unsigned>(rows < most ? rows : most);
}

}  // namespace
}  // namespace absk

using namespace absk;

extern "C" int abs_layer_norm(abs_ctx* ctx, const void* X, abs_dtype dtype, int M, long long rows, long long d,
                              long long x_row_stride, long long x_worker_stride, const float* weight, const float* bias,
                              long long param_stride, float eps, void* Y, long long y_row_stride,
                              long long y_worker_stride, float* mean, float* rstd, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  int rc = validate_shape(ctx, dtype, M, rows, d);
  if (rc != ABS_OK) return rc;
  if (!(eps >= 0.f) || eps > 3.0e38f) return set_error(ctx, ABS_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (rows == 0) return ABS_OK;
  if (X == nullptr || Y == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "X or Y is null");
  if ((rc = validate_rows(ctx, "X", M, rows, d, x_row_stride, x_worker_stride)) != ABS_OK) return rc;
  if ((rc = validate_rows(ctx, "Y", M, rows, d, y_row_stride, y_worker_stride)) != ABS_OK) return rc;
  if (M > 1 && (weight || bias) && param_stride != 0 && param_stride < d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "param_stride %lld < d %lld", param_stride, d);
  DeviceGuardLn guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  LnForward a{X, x_row_stride, x_worker_stride, weight, bias, param_stride, eps, Y, y_row_stride, y_worker_stride,
              mean, rstd, M, rows, static_cast<int>(d)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 grid(row_grid(ctx, rows * M));
  if (dtype == ABS_F32) ABS_CUDA_TRY(ctx, launch_dependent(ln_forward_any_kernel<float>, grid, dim3(kLnThreads), 0, st, a));
  else ABS_CUDA_TRY(ctx, launch_dependent(ln_forward_any_kernel<__nv_bfloat16>, grid, dim3(kLnThreads), 0, st, a));
  return ABS_OK;
}

extern "C" int abs_layer_norm_backward(abs_ctx* ctx, const void* dY, long long dy_row_stride, long long dy_worker_stride,
                                       const void* X, long long x_row_stride, long long x_worker_stride, abs_dtype dtype,
                                       int M, long long samples, long long tokens, long long d, const float* mean,
                                       const float* rstd, const float* weight, long long param_stride, void* dX,
                                       long long dx_row_stride, long long dx_worker_stride, float* dW, float* dB,
                                       long long grad_stride, float* Gw, float* Gb, long long g_row_stride,
                                       long long g_worker_stride, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (samples < 0 || tokens < 0 || (tokens > 0 && samples > (1ll << 40) / tokens))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "samples and tokens must be >= 0 and their product <= 2^40");
  long long rows = samples * tokens;
  int rc = validate_shape(ctx, dtype, M, rows, d);
  if (rc != ABS_OK) return rc;
  if (rows > 0) {
    if (dY == nullptr || X == nullptr || mean == nullptr || rstd == nullptr)
      return set_error(ctx, ABS_ERR_INVALID_ARG, "dY, X, mean or rstd is null");
    if ((rc = validate_rows(ctx, "dY", M, rows, d, dy_row_stride, dy_worker_stride)) != ABS_OK) return rc;
    if ((rc = validate_rows(ctx, "X", M, rows, d, x_row_stride, x_worker_stride)) != ABS_OK) return rc;
    if (dX && (rc = validate_rows(ctx, "dX", M, rows, d, dx_row_stride, dx_worker_stride)) != ABS_OK) return rc;
  }
  const bool per_sample = Gw != nullptr || Gb != nullptr, totals = dW != nullptr || dB != nullptr;
  if (M > 1 && weight && param_stride != 0 && param_stride < d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "param_stride %lld < d %lld", param_stride, d);
  if (M > 1 && totals && grad_stride < d) return set_error(ctx, ABS_ERR_INVALID_ARG, "grad_stride %lld < d %lld", grad_stride, d);
  if (per_sample && samples > 0 && (rc = validate_rows(ctx, "Gw / Gb", M, samples, d, g_row_stride, g_worker_stride)) != ABS_OK)
    return rc;
  DeviceGuardLn guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!per_sample) {               // only the totals: a replica's rows are one segment
    samples = rows > 0 ? 1 : 0;
    tokens = rows;
  }
  LnBackward a{dY, dy_row_stride, dy_worker_stride, X, x_row_stride, x_worker_stride, mean, rstd, weight, param_stride,
               dX, dx_row_stride, dx_worker_stride, M, samples, tokens, static_cast<int>(d), nullptr, 1, tokens};
  const long long col_tiles = (d + kLnThreads - 1) / kLnThreads;
  long long chunks = 0;
  if (rows > 0 && (per_sample || totals)) {
    const long long segments = samples * M;
    const long long room = static_cast<long long>(ctx->workspace_bytes / (2 * sizeof(float))) / d;     // units
    if (room < segments)
      return set_error(ctx, ABS_ERR_WORKSPACE, "the workspace holds %lld partial sums of %lld needed", room, segments);
    chunks = (static_cast<long long>(ctx->sm_count) * 8 + segments * col_tiles - 1) / (segments * col_tiles);
    const long long by_rows = (tokens + 15) / 16;                    // at least 16 rows per chunk
    if (chunks > by_rows) chunks = by_rows;
    if (chunks > room / segments) chunks = room / segments;
    if (chunks < 1) chunks = 1;
    a.part = static_cast<float*>(ctx->workspace);
    a.rows_per_chunk = (tokens + chunks - 1) / chunks;
    chunks = (tokens + a.rows_per_chunk - 1) / a.rows_per_chunk;
    a.chunks = static_cast<int>(chunks);
    const long long blocks = segments * chunks * col_tiles;
    if (blocks > 0x7fffffffll) return set_error(ctx, ABS_ERR_UNSUPPORTED, "too many samples (%lld) of width %lld", segments, d);
    const dim3 grid(static_cast<unsigned>(blocks));
    if (dtype == ABS_F32) ABS_CUDA_TRY(ctx, launch_dependent(ln_params_any_kernel<float>, grid, dim3(kLnThreads), 0, st, a));
    else ABS_CUDA_TRY(ctx, launch_dependent(ln_params_any_kernel<__nv_bfloat16>, grid, dim3(kLnThreads), 0, st, a));
  }
  // after the sums: dX may take the place of dY or X
  if (dX && rows > 0) {
    const dim3 grid(row_grid(ctx, rows * M));
    if (dtype == ABS_F32) ABS_CUDA_TRY(ctx, launch_dependent(ln_dx_any_kernel<float>, grid, dim3(kLnThreads), 0, st, a));
    else ABS_CUDA_TRY(ctx, launch_dependent(ln_dx_any_kernel<__nv_bfloat16>, grid, dim3(kLnThreads), 0, st, a));
  }
  if (!per_sample && !totals) return ABS_OK;
  LnReduce r{static_cast<const float*>(ctx->workspace), M, samples, static_cast<int>(chunks), static_cast<int>(d), Gw, Gb,
             g_row_stride, g_worker_stride, dW, dB, grad_stride};
  ABS_CUDA_TRY(ctx, launch_dependent(ln_reduce_kernel, dim3(static_cast<unsigned>((2 * d + 31) / 32), M), dim3(kLnThreads), 0,
                                     st, r));
  return ABS_OK;
}
