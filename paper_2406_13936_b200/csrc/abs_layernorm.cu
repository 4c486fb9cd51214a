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
  // The rows of all segments in order, `rows_per_cta` to a CTA; the sums of a CTA over its rows of a segment go to
  // part + part_slot() * 2d, or, where the segment lies within the CTA and both are given, to its rows of Gw and Gb.
  float* part;
  long long rows_per_cta;
  float* Gw;
  float* Gb;
  long long g_rs, g_ws;
};
// Place of CTA c's sums of segment s (counted over all replicas).  direct: only segments that do not lie within a CTA
// have one, at most a CTA's first and last; else along the rows each step raises c or s, so no two share a place.
__device__ __forceinline__ long long part_slot(bool direct, long long c, long long s, long long tokens, long long rows_per_cta) {
  return direct ? 2 * c + (s * tokens > c * rows_per_cta ? 1 : 0) : c + s;
}
struct LnReduce {
  const float* part;
  int M;
  long long samples, tokens, rows_per_cta;
  int d, direct;               // direct: segments within one CTA are in G already
  int whole;                   // ... and all of them lie within one
  long long per_cta;           // samples of a CTA (blockIdx.z)
  float* totals;               // [M][gridDim.z][2 d] where there are several, else NULL
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

// Any width, stride and alignment: one CTA per row, three sweeps over it.  2000 rows of 16384: fp32 92 us (2.9 TB/s of what has to
// move), bf16 54 (2.4): scalar loads.
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

// dx of any width, stride and alignment: one CTA per row, two sweeps; with the sums below x and dy are read from memory
// twice.  Backward on 2000 rows: fp32 of 8192 97 us (2.0 TB/s of what has to move), of 16384 227, bf16 of 9224 93, of 16384 202.
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

// The sums of dw and db of any width, stride and alignment: a thread owns a column of one CTA's rows.
template <typename T>
__global__ void __launch_bounds__(kLnThreads)
ln_params_any_kernel(const LnBackward a) {
  pdl_wait();
  const int col_tiles = (a.d + kLnThreads - 1) / kLnThreads;
  const long long c = blockIdx.x / col_tiles;
  const int j = static_cast<int>(blockIdx.x - c * col_tiles) * kLnThreads + threadIdx.x;
  if (j >= a.d) return;
  const long long rows = a.samples * a.tokens, total = rows * a.M;
  long long r = c * a.rows_per_cta;
  const long long end = r + a.rows_per_cta < total ? r + a.rows_per_cta : total;
  while (r < end) {
    const long long seg = r / a.tokens, m = seg / a.samples;
    const long long stop = (seg + 1) * a.tokens < end ? (seg + 1) * a.tokens : end;
    float dw = 0.f, db = 0.f;
    for (; r < stop; ++r) {
      const long long q = r - m * rows;
      const float g = to_f32<T>(static_cast<const T*>(a.dY)[m * a.dy_ws + q * a.dy_rs + j]);
      const float xh = (to_f32<T>(static_cast<const T*>(a.X)[m * a.x_ws + q * a.x_rs + j]) - a.mean[r]) * a.rstd[r];
      dw = fmaf(g, xh, dw);
      db += g;
    }
    float* out_w = a.part + part_slot(a.Gw != nullptr, c, seg, a.tokens, a.rows_per_cta) * 2 * a.d;
    float* out_b = out_w + a.d;
    if (a.Gw != nullptr && seg * a.tokens >= c * a.rows_per_cta && stop == (seg + 1) * a.tokens) {
      const long long g = m * a.g_ws + (seg - m * a.samples) * a.g_rs;
      out_w = a.Gw + g;
      out_b = a.Gb + g;
    }
    out_w[j] = dw;
    out_b[j] = db;
  }
}

// Partial sums -> samples -> replica, in a fixed order: 32 columns of one replica per CTA.  Eight lanes share the
// samples or, where there are few, the partial sums of each.
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
  const bool by_sample = a.samples >= 8 || a.tokens == 0;
  const long long i0 = blockIdx.z * a.per_cta, i1 = i0 + a.per_cta < a.samples ? i0 + a.per_cta : a.samples;
  if (a.whole) {
    if (live) {
      const float* p = G + m * a.g_ws + j;
#pragma unroll 8
      for (long long i = i0 + row; i < i1; i += 8) total += p[i * a.g_rs];
    }
  } else for (long long i = i0 + (by_sample ? row : 0); i < i1; i += by_sample ? 8 : 1) {
    const long long seg = m * a.samples + i;
    float s = 0.f;
    if (a.tokens > 0) {
      const long long c0 = seg * a.tokens / a.rows_per_cta, c1 = ((seg + 1) * a.tokens - 1) / a.rows_per_cta;
      if (a.direct && c0 == c1) {
        if (live && (by_sample || row == 0)) total += G[m * a.g_ws + i * a.g_rs + j];
        continue;
      }
      if (live) {
#pragma unroll 4
        for (long long c = by_sample ? c0 : c0 + row; c <= c1; c += by_sample ? 1 : 8)
          s += a.part[part_slot(a.direct, c, seg, a.tokens, a.rows_per_cta) * 2 * a.d + col];
      }
    }
    if (!by_sample) {
      __syncthreads();
      red[row][lane] = s;
      __syncthreads();
      s = 0.f;
      if (row == 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s += red[k][lane];
      }
    }
    if (live && (by_sample || row == 0)) {
      if (G) G[m * a.g_ws + i * a.g_rs + j] = s;
      total += s;
    }
  }
  __syncthreads();
  red[row][lane] = total;
  __syncthreads();
  float* out = is_b ? a.dB : a.dW;
  if (row == 0 && live && (out || a.totals)) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += red[k][lane];
    if (a.totals) a.totals[(m * gridDim.z + blockIdx.z) * 2 * a.d + col] = s;
    else out[m * a.grad_stride + j] = s;
  }
}

__global__ void __launch_bounds__(kLnThreads)
ln_total_kernel(const LnReduce a, int n) {
  const int col = blockIdx.x * kLnThreads + threadIdx.x;
  const long long m = blockIdx.y;
  pdl_wait();
  if (col >= 2 * a.d) return;
  const bool is_b = col >= a.d;
  float* out = is_b ? a.dB : a.dW;
  if (out == nullptr) return;
  float s = 0.f;
#pragma unroll 8
  for (int k = 0; k < n; ++k) s += a.totals[(m * n + k) * 2 * a.d + col];
  out[m * a.grad_stride + (is_b ? col - a.d : col)] = s;
}

// ---- rows held in registers -----------------------------------------------------------------------------
// Rows that are not 16-byte aligned, in pieces of one element or, bf16, two.  A group of `tpr` threads (whole warps)
// has a row: thread t holds the pieces t, t + tpr, ... of V elements, NV of them.  The next row's loads are issued before
// this row's arithmetic, weights (and, backward, the sums of dw and db) stay in registers from row to row, and a row is
// read and written once.  Sums over a row: shuffles, and through shared memory with a barrier of the group's own where
// it has several warps.  40000 x 1021, forward and backward: fp32 67 and 121 us (4.9 and 4.1 TB/s; narrow pieces through a ring of
// asynchronous copies, as below, 92 and 170: each copy is an instruction and 4 bytes), bf16 60 and 126 (2.7 and 1.9: 2 bytes a lane).
// The backward kernels of one element a piece spill 8 to 44 bytes a thread.
constexpr int kFastThreads = 384;

template <typename T, int V> struct Piece;       // V elements as one load
template <> struct Piece<float, 1> { typedef uint32_t Raw; };
template <> struct Piece<__nv_bfloat16, 2> { typedef uint32_t Raw; };
template <> struct Piece<__nv_bfloat16, 1> { typedef unsigned short Raw; };

__device__ __forceinline__ uint32_t ld_once(const uint32_t* p) { return __ldcs(p); }
__device__ __forceinline__ unsigned short ld_once(const unsigned short* p) { return __ldcs(p); }
template <typename R> __device__ __forceinline__ void st_once(R* p, const R& v) { __stcs(p, v); }
__device__ __forceinline__ void zero_raw(uint32_t& r) { r = 0u; }
__device__ __forceinline__ void zero_raw(unsigned short& r) { r = 0; }

template <typename T, int V>
__device__ __forceinline__ void unpack(const typename Piece<T, V>::Raw& r, float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
    x[0] = __uint_as_float(r);
  } else {
    x[0] = __uint_as_float(static_cast<uint32_t>(r) << 16);
    if constexpr (V == 2) x[1] = __uint_as_float(r & 0xffff0000u);
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T, int V>
__device__ __forceinline__ typename Piece<T, V>::Raw pack(const float (&x)[V]) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(x[0]);
  else if constexpr (V == 2) return pack_bf16(x[0], x[1]);
  else return __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
}

// Sums over a group's threads, the same in each.  red: [2][32] of the group; the two halves alternate, so one
// barrier a sum is enough.
template <bool ONE_WARP>
__device__ __forceinline__ float2 group_sum2(float a, float b, float2* red, int& flip, int group, int t, int tpr) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, off);
    b += __shfl_xor_sync(0xffffffffu, b, off);
  }
  if constexpr (ONE_WARP) return make_float2(a, b);
  float2* r = red + 32 * flip;
  flip ^= 1;
  if ((t & 31) == 0) r[t >> 5] = make_float2(a, b);
  named_bar_sync(1 + group, tpr);
  float2 s = make_float2(0.f, 0.f);
  for (int w = 0; w < tpr / 32; ++w) {
    s.x += r[w].x;
    s.y += r[w].y;
  }
  return s;
}

template <bool ONE_WARP>
__device__ __forceinline__ float4 group_sum4(float4 v, float4* red, int& flip, int group, int t, int tpr) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, off);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, off);
    v.z += __shfl_xor_sync(0xffffffffu, v.z, off);
    v.w += __shfl_xor_sync(0xffffffffu, v.w, off);
  }
  if constexpr (ONE_WARP) return v;
  float4* r = red + 32 * flip;
  flip ^= 1;
  if ((t & 31) == 0) r[t >> 5] = v;
  named_bar_sync(1 + group, tpr);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = 0; w < tpr / 32; ++w) {
    const float4 q = r[w];
    s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
  }
  return s;
}

template <int NV, int V>
__device__ __forceinline__ void load_params(const float* p, float other, int t, int tpr, int pieces, float (&w)[NV][V]) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + k * tpr;
#pragma unroll
    for (int e = 0; e < V; ++e) w[k][e] = p != nullptr && v < pieces ? __ldg(p + v * V + e) : other;
  }
}

template <typename T, int V, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(kFastThreads)
ln_forward_kernel(const LnForward a, int tpr, long long per_group) {
  typedef typename Piece<T, V>::Raw Raw;
  __shared__ float2 red_mem[12][2][32];
  const int group = static_cast<int>(threadIdx.x) / tpr, t = static_cast<int>(threadIdx.x) - group * tpr;
  const int groups = static_cast<int>(blockDim.x) / tpr, pieces = a.d / V;
  float2* red = &red_mem[ONE_WARP ? 0 : group][0][0];
  int flip = 0;
  const long long total = a.rows * a.M;
  long long rr = (static_cast<long long>(blockIdx.x) * groups + group) * per_group;
  const long long end = rr + per_group < total ? rr + per_group : total;
  long long m = rr / a.rows, r = rr - m * a.rows;
  pdl_wait();
  Raw next[NV];
  auto fetch = [&](long long mm, long long row) {
    const T* x = static_cast<const T*>(a.X) + mm * a.x_ws + row * a.x_rs;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) next[k] = ld_once(reinterpret_cast<const Raw*>(x) + v);
      else zero_raw(next[k]);
    }
  };
  if (rr < end) fetch(m, r);
  float w[NV][V], b[NV][V];
  bool have = false;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (; rr < end; ++rr) {
    if (!have) {
      load_params<NV, V>(a.weight ? a.weight + m * a.p_stride : nullptr, 1.f, t, tpr, pieces, w);
      load_params<NV, V>(a.bias ? a.bias + m * a.p_stride : nullptr, 0.f, t, tpr, pieces, b);
      have = true;
    }
    float x[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      unpack<T, V>(next[k], x[k]);
#pragma unroll
      for (int e = 0; e < V; ++e) s += x[k][e];
    }
    T* y = static_cast<T*>(a.Y) + m * a.y_ws + r * a.y_rs;
    const bool same = r + 1 < a.rows;
    if (same) {
      ++r;
    } else {
      r = 0;
      ++m;
      have = a.p_stride == 0;
    }
    if (rr + 1 < end) fetch(m, r);
    const float mean = group_sum2<ONE_WARP>(s, 0.f, red, flip, group, t, tpr).x * inv_d;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool in = t + k * tpr < pieces;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[k][e] -= mean;
        if (in) q = fmaf(x[k][e], x[k][e], q);
      }
    }
    const float rstd = 1.0f / sqrtf(fmaf(group_sum2<ONE_WARP>(q, 0.f, red, flip, group, t, tpr).x, inv_d, a.eps));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(x[k][e] * rstd, w[k][e], b[k][e]);
        st_once(reinterpret_cast<Raw*>(y) + v, pack<T, V>(o));
      }
    }
    if (t == 0) {
      if (a.mean) a.mean[rr] = mean;
      if (a.rstd) a.rstd[rr] = rstd;
    }
  }
}

// A CTA has rows_per_cta rows in a run; its groups take them in turn.  Where a segment ends, the groups' sums are
// added in order through shared memory and leave.
template <typename T, int V, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(kFastThreads)
ln_backward_kernel(const LnBackward a, int tpr) {
  typedef typename Piece<T, V>::Raw Raw;
  extern __shared__ float sums[];                                     // [groups - 1][2 d]
  __shared__ float2 red_mem[6][2][32];
  const int group = static_cast<int>(threadIdx.x) / tpr, t = static_cast<int>(threadIdx.x) - group * tpr;
  const int groups = static_cast<int>(blockDim.x) / tpr, pieces = a.d / V;
  float2* red = &red_mem[ONE_WARP ? 0 : group][0][0];
  int flip = 0;
  const long long rows = a.samples * a.tokens, total = rows * a.M;    // of a replica, of all
  const long long first = static_cast<long long>(blockIdx.x) * a.rows_per_cta;
  const long long end = first + a.rows_per_cta < total ? first + a.rows_per_cta : total;
  long long row = first + group;                                      // this group's row among all
  long long m = row / rows, r = row - m * rows;                       // ... its replica and place there
  pdl_wait();
  Raw nx[NV], ng[NV];
  float n_mean = 0.f, n_rstd = 0.f;
  auto fetch = [&]() {
    const Raw* x = reinterpret_cast<const Raw*>(static_cast<const T*>(a.X) + m * a.x_ws + r * a.x_rs);
    const Raw* g = reinterpret_cast<const Raw*>(static_cast<const T*>(a.dY) + m * a.dy_ws + r * a.dy_rs);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) {
        nx[k] = ld_once(x + v);
        ng[k] = ld_once(g + v);
      } else {
        zero_raw(nx[k]);
        zero_raw(ng[k]);
      }
    }
    n_mean = __ldg(a.mean + row);
    n_rstd = __ldg(a.rstd + row);
  };
  if (row < end) fetch();
  float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[k][e] = db[k][e] = 0.f;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  long long have = -1;                                                // the replica whose weight is in w
  long long seg = first / a.tokens;
  for (long long at = first; at < end; ++seg) {
    const long long stop = (seg + 1) * a.tokens < end ? (seg + 1) * a.tokens : end;
    const long long sm = seg / a.samples;                             // the segment's replica
    if (sm != have) {
      if (have < 0 || a.p_stride != 0)
        load_params<NV, V>(a.weight ? a.weight + sm * a.p_stride : nullptr, 1.f, t, tpr, pieces, w);
      have = sm;
    }
    while (row < stop) {
      Raw cx[NV], cg[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        cx[k] = nx[k];
        cg[k] = ng[k];
      }
      const float mean = n_mean, rstd = n_rstd;
      Raw* o = reinterpret_cast<Raw*>(static_cast<T*>(a.dX) + m * a.dx_ws + r * a.dx_rs);
      row += groups;
      r += groups;
      while (r >= rows) {
        r -= rows;
        ++m;
      }
      if (row < end) fetch();
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float x[V], g[V];
        unpack<T, V>(cx[k], x);
        unpack<T, V>(cg[k], g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float xh = (x[e] - mean) * rstd, y = g[e] * w[k][e];
          s1 += y;
          s2 = fmaf(y, xh, s2);
          dw[k][e] = fmaf(g[e], xh, dw[k][e]);
          db[k][e] += g[e];
        }
      }
      if (a.dX != nullptr) {
        const float2 s = group_sum2<ONE_WARP>(s1, s2, red, flip, group, t, tpr);
        const float c1 = s.x * inv_d, c2 = s.y * inv_d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = t + k * tpr;
          float x[V], g[V], q[V];
          unpack<T, V>(cx[k], x);
          unpack<T, V>(cg[k], g);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float xh = (x[e] - mean) * rstd;
            q[e] = rstd * (fmaf(g[e], w[k][e], -c1) - xh * c2);
          }
          if (v < pieces) st_once(o + v, pack<T, V>(q));
        }
      }
    }
    if (a.part != nullptr) {
      // pieces past the row have zeros in dy: their sums are zero and not stored
      float* out_w = a.part + part_slot(a.Gw != nullptr, blockIdx.x, seg, a.tokens, a.rows_per_cta) * 2 * a.d;
      float* out_b = out_w + a.d;
      if (a.Gw != nullptr && at == seg * a.tokens && stop == (seg + 1) * a.tokens) {
        const long long g = sm * a.g_ws + (seg - sm * a.samples) * a.g_rs;
        out_w = a.Gw + g;
        out_b = a.Gb + g;
      }
      if (groups > 1) {
        if (group > 0) {
          float* p = sums + static_cast<long long>(group - 1) * 2 * a.d;
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const int v = t + k * tpr;
            if (v < pieces) {
#pragma unroll
              for (int e = 0; e < V; ++e) {
                p[v * V + e] = dw[k][e];
                p[a.d + v * V + e] = db[k][e];
              }
            }
          }
        }
        __syncthreads();
      }
      if (group == 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = t + k * tpr;
          if (v < pieces) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              float sw = dw[k][e], sb = db[k][e];
              for (int o = 0; o < groups - 1; ++o) {
                const float* p = sums + static_cast<long long>(o) * 2 * a.d + v * V + e;
                sw += p[0];
                sb += p[a.d];
              }
              out_w[v * V + e] = sw;
              out_b[v * V + e] = sb;
            }
          }
        }
      }
      if (groups > 1) __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[k][e] = db[k][e] = 0.f;
    }
    at = stop;
  }
}

// ---- rows staged in shared memory ---------------------------------------------------------------------------
// Rows whose pieces of 16 bytes are aligned.  A thread copies its own pieces of the rows ahead into its own places of a
// ring with cp.async, so the bytes under way do not depend on registers and nobody waits for anybody else's copies.
// (8 x 16384 x 768 bf16, forward / backward: with the next row in registers, 12 warps an SM, 95 / 167 us; with bulk
// copies of whole rows and an mbarrier each 78 / 260 us.)  A group works on two rows at a time where it can: their sums
// go through the same shuffles and barriers.  Arithmetic on pairs of elements (fma.rn.f32x2): at 2 bytes an element the
// issue slots are the other limit.
constexpr int kRingThreads = 384;
constexpr int kAhead = 2;                          // rows under way besides the two that are worked on
constexpr int kRing = kAhead + 2;

__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float sum2(uint64_t v) {
  const float2 f = unpair(v);
  return f.x + f.y;
}
// A piece of 16 bytes as pairs of fp32: 2 (fp32) or 4 (bf16).
template <typename T>
__device__ __forceinline__ void read_piece(uint32_t addr, uint64_t (&x)[8 / sizeof(T)]) {
  const uint4 r = lds128(addr);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (sizeof(T) == 4) {
    x[0] = pair(__uint_as_float(w[0]), __uint_as_float(w[1]));
    x[1] = pair(__uint_as_float(w[2]), __uint_as_float(w[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pair(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
  }
}
template <typename T>
__device__ __forceinline__ void write_piece(void* p, const uint64_t (&x)[8 / sizeof(T)]) {
  uint32_t w[4];
  if constexpr (sizeof(T) == 4) {
    const float2 a = unpair(x[0]), b = unpair(x[1]);
    w[0] = __float_as_uint(a.x); w[1] = __float_as_uint(a.y); w[2] = __float_as_uint(b.x); w[3] = __float_as_uint(b.y);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = unpair(x[e]);
      w[e] = pack_bf16(f.x, f.y);
    }
  }
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ void copy_ahead(uint32_t dst, const char* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// ... until all but the last kAhead rows' copies are done
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory"); }

// A replica's weight (or bias) into shared memory: element j of piece v = j / 2P lies in the piece's quarter q, [Q][pieces]
// of 16 bytes, so that a warp's reads of one quarter are contiguous.
template <typename T>
__device__ __forceinline__ void stage_params(float* to, const float* from, float other, int d) {
  constexpr int E = 16 / sizeof(T);
  const int pieces = d / E;
  for (int j = threadIdx.x; j < d; j += blockDim.x) {
    const int v = j / E, q = (j - v * E) / 4;
    to[(q * pieces + v) * 4 + (j & 3)] = from ? __ldg(from + j) : other;
  }
}
__device__ __forceinline__ void read_params(uint32_t addr, uint64_t& a, uint64_t& b) {
  const uint4 v = lds128(addr);
  a = pair(__uint_as_float(v.x), __uint_as_float(v.y));
  b = pair(__uint_as_float(v.z), __uint_as_float(v.w));
}
// Pairs of sums to consecutive floats; `wide`: p is 16-byte aligned.
template <int P>
__device__ __forceinline__ void store_sums(float* p, const uint64_t (&x)[P], bool wide) {
#pragma unroll
  for (int e = 0; e < P; e += 2) {
    const float2 a = unpair(x[e]), b = unpair(x[e + 1]);
    if (wide) {
      *reinterpret_cast<float4*>(p + 2 * e) = make_float4(a.x, a.y, b.x, b.y);
    } else {
      p[2 * e] = a.x; p[2 * e + 1] = a.y; p[2 * e + 2] = b.x; p[2 * e + 3] = b.y;
    }
  }
}

// A place in the ring of rows that a thread walks.
struct Place {
  uint32_t at, begin, end, step;
  __device__ __forceinline__ void forward() {
    at += step;
    if (at == end) at = begin;
  }
};

// A CTA has rows_per_cta rows in a run, its groups take them in turn; weight and bias of the replica lie in shared
// memory.
template <typename T, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(kRingThreads, 1)
ln_forward_ring_kernel(const LnForward a, int tpr, long long rows_per_cta) {
  constexpr int P = 8 / sizeof(T), Q = P / 2;                          // a piece's weights are Q times 16 bytes
  constexpr long long es = sizeof(T);
  extern __shared__ __align__(128) unsigned char ring_mem[];           // [kRing][NV][threads] pieces, weight, bias [Q][pieces]
  __shared__ float2 red_mem[ONE_WARP ? 1 : kRingThreads / 64][2][32];
  const int group = static_cast<int>(threadIdx.x) / tpr, t = static_cast<int>(threadIdx.x) - group * tpr;
  const int groups = static_cast<int>(blockDim.x) / tpr, pieces = a.d / (2 * P);
  const uint32_t piece_step = blockDim.x * 16u, row_bytes = NV * piece_step;
  const uint32_t mine = smem_u32(ring_mem) + threadIdx.x * 16u;
  float* params = reinterpret_cast<float*>(ring_mem + static_cast<size_t>(kRing) * row_bytes);
  const uint32_t w_at = smem_u32(params) + 16u * t, b_at = w_at + Q * pieces * 16u;
  float2* red = &red_mem[ONE_WARP ? 0 : group][0][0];
  int flip = 0;
  const long long total = a.rows * a.M;
  const long long first = static_cast<long long>(blockIdx.x) * rows_per_cta;
  const int run = static_cast<int>(total - first < rows_per_cta ? total - first : rows_per_cta);      // this CTA's rows
  const int count = run > group ? (run - group + groups - 1) / groups : 0;                            // ... this group's
  // the row that is copied next: its number in the group's run, its address, the rows of its replica from it on
  int copied = 0;
  long long c_m = (first + group) / a.rows, c_left = a.rows - (first + group - c_m * a.rows);
  const char* c_x = static_cast<const char*>(a.X) + (c_m * a.x_ws + (a.rows - c_left) * a.x_rs) * es + t * 16;
  const long long x_step = groups * a.x_rs * es, y_step = groups * a.y_rs * es;
  Place c_at = {mine, mine, mine + kRing * row_bytes, row_bytes}, x_at = c_at;
  pdl_wait();
  auto copy_until = [&](int n) {                                       // rows up to the n-th; past the run nothing
    for (; copied < n; ++copied) {
      if (copied < count) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (t + k * tpr < pieces) copy_ahead(c_at.at + k * piece_step, c_x + k * tpr * 16);
        c_x += x_step;
        c_left -= groups;
        if (c_left <= 0) {
          while (c_left <= 0) {
            c_left += a.rows;
            ++c_m;
          }
          c_x = static_cast<const char*>(a.X) + (c_m * a.x_ws + (a.rows - c_left) * a.x_rs) * es + t * 16;
        }
      }
      copies_commit();
      c_at.forward();
    }
  };
  copy_until(kAhead);
  const float inv_d = 1.0f / static_cast<float>(a.d);
  long long m = first / a.rows;
  int next = group, done = 0;                                          // this group's next row in the run, rows done
  for (int at = 0; at < run; ++m) {                                    // the run's rows of replica m
    const long long m_end = (m + 1) * a.rows - first;
    const int stop = m_end < run ? static_cast<int>(m_end) : run;
    if (at == 0 || a.p_stride != 0) {
      if (at > 0) __syncthreads();
      stage_params<T>(params, a.weight ? a.weight + m * a.p_stride : nullptr, 1.f, a.d);
      stage_params<T>(params + a.d, a.bias ? a.bias + m * a.p_stride : nullptr, 0.f, a.d);
      __syncthreads();
    }
    const long long row = first + next;                                // of all
    char* y = static_cast<char*>(a.Y) + (m * a.y_ws + (row - m * a.rows) * a.y_rs) * es + 16 * t;
    float* mean_out = a.mean ? a.mean + row : nullptr;
    float* rstd_out = a.rstd ? a.rstd + row : nullptr;
    while (next < stop) {
      copy_until(done + kRing);                                        // into the places of the rows before
      const bool two = next + groups < stop;                           // this group's next two rows
      copies_wait();
      uint64_t x[2][NV][P], sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (q == 0 || two) {
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            if (t + k * tpr < pieces) {
              read_piece<T>(x_at.at + k * piece_step, x[q][k]);
#pragma unroll
              for (int e = 0; e < P; ++e) sum[q] = add2(sum[q], x[q][k][e]);
            }
          }
          x_at.forward();
        }
      }
      const float2 s = group_sum2<ONE_WARP>(sum2(sum[0]), sum2(sum[1]), red, flip, group, t, tpr);
      const float mean[2] = {s.x * inv_d, s.y * inv_d};
      uint64_t sq[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint64_t shift = pair(-mean[q], -mean[q]);
        if (q == 0 || two) {
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            if (t + k * tpr < pieces) {
#pragma unroll
              for (int e = 0; e < P; ++e) {
                x[q][k][e] = add2(x[q][k][e], shift);
                sq[q] = fma2(x[q][k][e], x[q][k][e], sq[q]);
              }
            }
          }
        }
      }
      const float2 v = group_sum2<ONE_WARP>(sum2(sq[0]), sum2(sq[1]), red, flip, group, t, tpr);
      const float rstd[2] = {rsqrtf(fmaf(v.x, inv_d, a.eps)), rsqrtf(fmaf(v.y, inv_d, a.eps))};      // (within 2 ulp)
      const uint64_t scale[2] = {pair(rstd[0], rstd[0]), pair(rstd[1], rstd[1])};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * tpr < pieces) {
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            uint64_t w0, w1, b0, b1;
            read_params(w_at + (q * pieces + k * tpr) * 16u, w0, w1);
            read_params(b_at + (q * pieces + k * tpr) * 16u, b0, b1);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              x[r][k][2 * q] = fma2(mul2(x[r][k][2 * q], scale[r]), w0, b0);
              x[r][k][2 * q + 1] = fma2(mul2(x[r][k][2 * q + 1], scale[r]), w1, b1);
            }
          }
          write_piece<T>(y + k * tpr * 16, x[0][k]);
          if (two) write_piece<T>(y + y_step + k * tpr * 16, x[1][k]);
        }
      }
      if (t == 0) {
        if (mean_out) {
          mean_out[0] = mean[0];
          if (two) mean_out[groups] = mean[1];
        }
        if (rstd_out) {
          rstd_out[0] = rstd[0];
          if (two) rstd_out[groups] = rstd[1];
        }
      }
      const int n = two ? 2 : 1;
      done += n;
      next += n * groups;
      y += n * y_step;
      if (mean_out) mean_out += n * groups;
      if (rstd_out) rstd_out += n * groups;
    }
    at = stop;
  }
}

// A CTA has rows_per_cta rows in a run; its groups take them in turn.  Where a segment ends, the groups' sums are
// added in order through shared memory (`slots` of them at a time) and leave.
template <typename T, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(kRingThreads, 1)
ln_backward_ring_kernel(const LnBackward a, int tpr, int slots) {
  constexpr int P = 8 / sizeof(T), Q = P / 2;                          // a piece's weights are Q times 16 bytes
  constexpr long long es = sizeof(T);
  extern __shared__ __align__(128) unsigned char ring_mem[];           // [kRing][x, dy][NV][threads] pieces, weight, [slots][2 d] sums
  __shared__ float4 red_mem[ONE_WARP ? 1 : kRingThreads / 64][2][32];
  const int group = static_cast<int>(threadIdx.x) / tpr, t = static_cast<int>(threadIdx.x) - group * tpr;
  const int groups = static_cast<int>(blockDim.x) / tpr, pieces = a.d / (2 * P);
  const uint32_t piece_step = blockDim.x * 16u, half_bytes = NV * piece_step, row_bytes = 2u * half_bytes;
  const uint32_t mine = smem_u32(ring_mem) + threadIdx.x * 16u;
  float* params = reinterpret_cast<float*>(ring_mem + static_cast<size_t>(kRing) * row_bytes);
  float* sums = params + a.d;
  const uint32_t w_at = smem_u32(params) + 16u * t;
  float4* red = &red_mem[ONE_WARP ? 0 : group][0][0];
  int flip = 0;
  const long long rows = a.samples * a.tokens, total = rows * a.M;     // of a replica, of all
  const long long first = static_cast<long long>(blockIdx.x) * a.rows_per_cta;
  const int run = static_cast<int>(total - first < a.rows_per_cta ? total - first : a.rows_per_cta);      // this CTA's rows
  const int count = run > group ? (run - group + groups - 1) / groups : 0;                                // ... this group's
  // the row that is copied next: its number in the group's run, its address, the rows of its replica from it on
  int copied = 0;
  long long c_m = (first + group) / rows, c_left = rows - (first + group - c_m * rows);
  const char *c_x, *c_g;
  auto find = [&]() {
    const long long r = rows - c_left;
    c_x = static_cast<const char*>(a.X) + (c_m * a.x_ws + r * a.x_rs) * es + t * 16;
    c_g = static_cast<const char*>(a.dY) + (c_m * a.dy_ws + r * a.dy_rs) * es + t * 16;
  };
  find();
  const long long x_step = groups * a.x_rs * es, g_step = groups * a.dy_rs * es, o_step = groups * a.dx_rs * es;
  Place c_at = {mine, mine, mine + kRing * row_bytes, row_bytes}, x_at = c_at;
  pdl_wait();
  auto copy_row = [&]() {
    if (copied < count) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * tpr < pieces) {
          copy_ahead(c_at.at + k * piece_step, c_x + k * tpr * 16);
          copy_ahead(c_at.at + half_bytes + k * piece_step, c_g + k * tpr * 16);
        }
      }
      ++copied;
      c_x += x_step;
      c_g += g_step;
      c_left -= groups;
      if (c_left <= 0) {
        while (c_left <= 0) {
          c_left += rows;
          ++c_m;
        }
        find();
      }
    }
    copies_commit();
    c_at.forward();
  };
  for (int s = 0; s < kAhead; ++s) copy_row();
  const float *mean_in = a.mean + first + group, *rstd_in = a.rstd + first + group;      // of this group's next row
  // of its next two rows, asked for an iteration early
  float n_mean[2] = {0.f, 0.f}, n_rstd[2] = {0.f, 0.f};
  int done = 0;                                                        // rows of this group that are done
  auto next_statistics = [&]() {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (done + q < count) {
        n_mean[q] = __ldg(mean_in + q * groups);
        n_rstd[q] = __ldg(rstd_in + q * groups);
      }
    }
  };
  next_statistics();
  uint64_t dw[NV][P], db[NV][P];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < P; ++e) dw[k][e] = db[k][e] = pair(0.f, 0.f);
  const float inv_d = 1.0f / static_cast<float>(a.d);
  long long have = -1;                                                 // the replica whose weight is in shared memory
  long long seg = first / a.tokens;
  int next = group;                                                    // this group's next row in the run
  for (int at = 0; at < run; ++seg) {
    const long long seg_end = (seg + 1) * a.tokens - first;
    const int stop = seg_end < run ? static_cast<int>(seg_end) : run;
    const long long sm = seg / a.samples;                              // the segment's replica
    if (sm != have) {
      if (have < 0 || a.p_stride != 0) {
        if (have >= 0) __syncthreads();
        stage_params<T>(params, a.weight ? a.weight + sm * a.p_stride : nullptr, 1.f, a.d);
        __syncthreads();
      }
      have = sm;
    }
    char* o = static_cast<char*>(a.dX) + (sm * a.dx_ws + (first + next - sm * rows) * a.dx_rs) * es + 16 * t;
    while (next < stop) {
      const bool two = next + groups < stop;                           // this group's next two rows, of one segment
      copy_row();                                                      // into the places of the rows before
      if (two) copy_row();
      const float mean[2] = {n_mean[0], n_mean[1]}, rstd[2] = {n_rstd[0], n_rstd[1]};
      const int n = two ? 2 : 1;
      done += n;
      mean_in += n * groups;
      rstd_in += n * groups;
      next_statistics();
      copies_wait();
      const uint32_t xp0 = x_at.at;
      x_at.forward();
      const uint32_t xp1 = x_at.at;
      if (two) x_at.forward();
      const uint64_t r2[2] = {pair(rstd[0], rstd[0]), pair(rstd[1], rstd[1])};
      const uint64_t shift[2] = {pair(-mean[0], -mean[0]), pair(-mean[1], -mean[1])};
      uint64_t s1[2] = {pair(0.f, 0.f), pair(0.f, 0.f)}, s2[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * tpr < pieces) {
          uint64_t w[P];
#pragma unroll
          for (int e = 0; e < Q; ++e) read_params(w_at + (e * pieces + k * tpr) * 16u, w[2 * e], w[2 * e + 1]);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            if (q == 0 || two) {
              const uint32_t xp = q == 0 ? xp0 : xp1;
              uint64_t x[P], g[P];
              read_piece<T>(xp + k * piece_step, x);
              read_piece<T>(xp + half_bytes + k * piece_step, g);
#pragma unroll
              for (int e = 0; e < P; ++e) {
                const uint64_t xh = mul2(add2(x[e], shift[q]), r2[q]), y = mul2(g[e], w[e]);
                s1[q] = add2(s1[q], y);
                s2[q] = fma2(y, xh, s2[q]);
                dw[k][e] = fma2(g[e], xh, dw[k][e]);
                db[k][e] = add2(db[k][e], g[e]);
              }
            }
          }
        }
      }
      if (a.dX != nullptr) {
        float4 c = make_float4(sum2(s1[0]), sum2(s2[0]), sum2(s1[1]), sum2(s2[1]));
        c = group_sum4<ONE_WARP>(c, red, flip, group, t, tpr);
        const uint64_t nc1[2] = {pair(-c.x * inv_d, -c.x * inv_d), pair(-c.z * inv_d, -c.z * inv_d)};
        const uint64_t nc2[2] = {pair(-c.y * inv_d, -c.y * inv_d), pair(-c.w * inv_d, -c.w * inv_d)};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          if (t + k * tpr < pieces) {
            uint64_t w[P];
#pragma unroll
            for (int e = 0; e < Q; ++e) read_params(w_at + (e * pieces + k * tpr) * 16u, w[2 * e], w[2 * e + 1]);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              if (q == 0 || two) {
                const uint32_t xp = q == 0 ? xp0 : xp1;
                uint64_t x[P], g[P];
                read_piece<T>(xp + k * piece_step, x);
                read_piece<T>(xp + half_bytes + k * piece_step, g);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                  const uint64_t xh = mul2(add2(x[e], shift[q]), r2[q]);
                  x[e] = mul2(r2[q], fma2(xh, nc2[q], fma2(g[e], w[e], nc1[q])));
                }
                write_piece<T>(o + q * o_step + k * tpr * 16, x);
              }
            }
          }
        }
      }
      next += n * groups;
      o += n * o_step;
    }
    if (a.part != nullptr) {
      float* out_w = a.part + part_slot(a.Gw != nullptr, blockIdx.x, seg, a.tokens, a.rows_per_cta) * 2 * a.d;
      float* out_b = out_w + a.d;
      if (a.Gw != nullptr && first + at == seg * a.tokens && first + stop == (seg + 1) * a.tokens) {
        const long long g = sm * a.g_ws + (seg - sm * a.samples) * a.g_rs;
        out_w = a.Gw + g;
        out_b = a.Gb + g;
      }
      for (int base = 1; base < groups; base += slots) {               // groups base .. base + slots - 1 hand theirs to group 0
        if (group >= base && group < base + slots) {
          float2* p = reinterpret_cast<float2*>(sums + static_cast<size_t>(group - base) * 2 * a.d);
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const int v = t + k * tpr;
            if (v < pieces) {
#pragma unroll
              for (int e = 0; e < P; ++e) {
                p[v * P + e] = unpair(dw[k][e]);
                p[a.d / 2 + v * P + e] = unpair(db[k][e]);
              }
            }
          }
        }
        __syncthreads();
        if (group == 0) {
          const int n = groups - base < slots ? groups - base : slots;
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const int v = t + k * tpr;
            if (v < pieces) {
              for (int g = 0; g < n; ++g) {
                const float2* p = reinterpret_cast<const float2*>(sums + static_cast<size_t>(g) * 2 * a.d);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                  const float2 fw = p[v * P + e], fb = p[a.d / 2 + v * P + e];
                  dw[k][e] = add2(dw[k][e], pair(fw.x, fw.y));
                  db[k][e] = add2(db[k][e], pair(fb.x, fb.y));
                }
              }
            }
          }
        }
        __syncthreads();
      }
      if (group == 0) {
        const bool wide = ((reinterpret_cast<uintptr_t>(out_w) | reinterpret_cast<uintptr_t>(out_b)) & 15u) == 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = t + k * tpr;
          if (v < pieces) {
            store_sums<P>(out_w + v * 2 * P, dw[k], wide);
            store_sums<P>(out_b + v * 2 * P, db[k], wide);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < P; ++e) dw[k][e] = db[k][e] = pair(0.f, 0.f);
    }
    at = stop;
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


// How a row of d elements is laid out over threads, or tpr = 0 where it does not fit: the fewest threads (a divisor of
// the CTA's) that hold it in at most NV pieces each; few, because what a row costs a warp besides its elements is half
// of the instructions.  Pieces are of 16 bytes (NV up to most_wide: forward 6, where two rows' elements are in
// registers; backward 4 of fp32 or 3 of bf16, where each element has two running sums), or, where the alignment does not allow them, of
// one element or two bf16 (one variant each, 16 elements a thread).  The widest rows are 9216 fp32 and, by the shared memory, 12800 bf16
// forward, 6144 and 9216 backward, 6144 in narrow pieces.
struct RowPlan {
  bool wide;
  int V, NV, tpr;
};
constexpr size_t kRingBytes = 220 * 1024;          // dynamic shared memory of the ring kernels, at most
size_t ring_smem(int NV, int threads, int tensors) { return static_cast<size_t>(kRing) * tensors * NV * threads * 16; }
RowPlan plan_row(abs_dtype dtype, long long d, unsigned long long align_bits, int most_wide, int tensors) {
  const int es = dtype == ABS_F32 ? 4 : 2;
  RowPlan p = {false, 1, 0, 0};
  align_bits |= static_cast<unsigned long long>(d) * es;
  p.wide = (align_bits & 15u) == 0;
  if (p.wide) p.V = 16 / es;
  else if (es == 2 && (align_bits & 3u) == 0) p.V = 2;
  const long long pieces = d / p.V;
  const int most = p.wide ? most_wide : 16 / p.V;
  const int tprs[6] = {32, 64, 96, 128, 192, 384};
  for (int k = 0; k < 6; ++k) {
    if (pieces > static_cast<long long>(tprs[k]) * most) continue;
    const int NV = p.wide ? static_cast<int>((pieces + tprs[k] - 1) / tprs[k]) : most;
    // the ring, the parameters (two vectors forward, one backward) and, backward, one group's sums
    const size_t vectors = tensors == 1 ? 2 : tprs[k] < kRingThreads ? 3 : 1;
    if (p.wide && ring_smem(NV, kRingThreads, tensors) + vectors * static_cast<size_t>(d) * sizeof(float) > kRingBytes) continue;
    p.tpr = tprs[k];
    p.NV = NV;
    break;
  }
  return p;
}

template <typename T, int V, int NV>
cudaError_t run_forward(abs_ctx* ctx, const LnForward& a, int tpr, cudaStream_t st) {
  const int groups = kFastThreads / tpr;
  const long long total = a.rows * a.M;
  const long long most = static_cast<long long>(ctx->sm_count) * groups;
  const long long per = (total + most - 1) / most;
  const long long used = (total + per - 1) / per;
  const unsigned grid = static_cast<unsigned>((used + groups - 1) / groups);
  auto kern = tpr == 32 ? ln_forward_kernel<T, V, NV, true> : ln_forward_kernel<T, V, NV, false>;
  return launch_dependent(kern, dim3(grid), dim3(kFastThreads), 0, st, a, tpr, per);
}
template <typename T, int NV>
cudaError_t run_forward_ring(abs_ctx* ctx, const LnForward& a, int tpr, cudaStream_t st) {
  const long long total = a.rows * a.M;
  const int groups = kRingThreads / tpr;
  const size_t smem = ring_smem(NV, kRingThreads, 1) + 2 * static_cast<size_t>(a.d) * sizeof(float);
  const long long most = static_cast<long long>(ctx->sm_count);
  long long per = (total + most - 1) / most;
  if (per < groups) per = groups < total ? groups : total;             // a row for every group before a second CTA
  if (per > (1ll << 30)) per = 1ll << 30;                              // a CTA counts its rows in 32 bits
  const unsigned grid = static_cast<unsigned>((total + per - 1) / per);
  auto kern = tpr == 32 ? ln_forward_ring_kernel<T, NV, true> : ln_forward_ring_kernel<T, NV, false>;
  const cudaError_t e = ensure_dynamic_smem(ctx, kern, smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kern, dim3(grid), dim3(kRingThreads), smem, st, a, tpr, per);
}
cudaError_t dispatch_forward(abs_ctx* ctx, const LnForward& a, abs_dtype dtype, const RowPlan& p, cudaStream_t st) {
  const bool f = dtype == ABS_F32;
  if (!p.wide) {
    if (f) return run_forward<float, 1, 16>(ctx, a, p.tpr, st);
    return p.V == 2 ? run_forward<__nv_bfloat16, 2, 8>(ctx, a, p.tpr, st) : run_forward<__nv_bfloat16, 1, 16>(ctx, a, p.tpr, st);
  }
  switch (p.NV) {
    case 1: return f ? run_forward_ring<float, 1>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 1>(ctx, a, p.tpr, st);
    case 2: return f ? run_forward_ring<float, 2>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 2>(ctx, a, p.tpr, st);
    case 3: return f ? run_forward_ring<float, 3>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 3>(ctx, a, p.tpr, st);
    case 4: return f ? run_forward_ring<float, 4>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 4>(ctx, a, p.tpr, st);
    case 5: return f ? run_forward_ring<float, 5>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 5>(ctx, a, p.tpr, st);
    default: return f ? run_forward_ring<float, 6>(ctx, a, p.tpr, st) : run_forward_ring<__nv_bfloat16, 6>(ctx, a, p.tpr, st);
  }
}

template <typename T, int V, int NV>
cudaError_t run_backward(abs_ctx* ctx, const LnBackward& a, int tpr, int groups, unsigned grid, cudaStream_t st) {
  const size_t smem = a.part != nullptr ? static_cast<size_t>(groups - 1) * 2 * a.d * sizeof(float) : 0;
  auto kern = tpr == 32 ? ln_backward_kernel<T, V, NV, true> : ln_backward_kernel<T, V, NV, false>;
  if (smem > 40 * 1024) {
    const cudaError_t e = ensure_dynamic_smem(ctx, kern, smem);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kern, dim3(grid), dim3(tpr * groups), smem, st, a, tpr);
}
template <typename T, int NV>
cudaError_t run_backward_ring(abs_ctx* ctx, const LnBackward& a, int tpr, int groups, unsigned grid, cudaStream_t st) {
  const size_t sum = 2 * static_cast<size_t>(a.d) * sizeof(float);
  int slots = 0;
  const size_t ring = ring_smem(NV, tpr * groups, 2) + static_cast<size_t>(a.d) * sizeof(float);
  if (a.part != nullptr && groups > 1) {             // sums of as many groups at a time as there is room for, up to 48 KB
    const size_t room = kRingBytes - ring;
    slots = static_cast<int>((room < 48 * 1024 ? room : 48 * 1024) / sum);
    if (slots > groups - 1) slots = groups - 1;
    if (slots < 1) slots = 1;
  }
  const size_t smem = ring + slots * sum;
  auto kern = tpr == 32 ? ln_backward_ring_kernel<T, NV, true> : ln_backward_ring_kernel<T, NV, false>;
  const cudaError_t e = ensure_dynamic_smem(ctx, kern, smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kern, dim3(grid), dim3(tpr * groups), smem, st, a, tpr, slots);
}
cudaError_t dispatch_backward(abs_ctx* ctx, const LnBackward& a, abs_dtype dtype, const RowPlan& p, int groups, unsigned grid,
                              cudaStream_t st) {
  const bool f = dtype == ABS_F32;
  if (!p.wide) {
    if (f) return run_backward<float, 1, 16>(ctx, a, p.tpr, groups, grid, st);
    return p.V == 2 ? run_backward<__nv_bfloat16, 2, 8>(ctx, a, p.tpr, groups, grid, st)
                    : run_backward<__nv_bfloat16, 1, 16>(ctx, a, p.tpr, groups, grid, st);
  }
  switch (p.NV) {
    case 1: return f ? run_backward_ring<float, 1>(ctx, a, p.tpr, groups, grid, st) : run_backward_ring<__nv_bfloat16, 1>(ctx, a, p.tpr, groups, grid, st);
    case 2: return f ? run_backward_ring<float, 2>(ctx, a, p.tpr, groups, grid, st) : run_backward_ring<__nv_bfloat16, 2>(ctx, a, p.tpr, groups, grid, st);
    case 3: return f ? run_backward_ring<float, 3>(ctx, a, p.tpr, groups, grid, st) : run_backward_ring<__nv_bfloat16, 3>(ctx, a, p.tpr, groups, grid, st);
    default: return run_backward_ring<float, 4>(ctx, a, p.tpr, groups, grid, st);
  }
}

unsigned long long row_bits(const void* p, abs_dtype dtype, int M, long long rs, long long ws) {
  const unsigned long long es = dtype == ABS_F32 ? 4 : 2;
  return reinterpret_cast<uintptr_t>(p) | static_cast<unsigned long long>(rs) * es | (M > 1 ? static_cast<unsigned long long>(ws) * es : 0);
}

// How a backward pass shares out its rows and what it keeps in the workspace, counted in partial sums of 2 d floats: those of
// the CTAs at part_slot(), `used` places, then the totals of ln_reduce_kernel's CTAs.  Host arithmetic alone.
struct BackwardPlan {
  RowPlan row;
  bool sums, direct, whole;
  int groups;
  long long samples, tokens;             // segments of a replica and rows of one
  long long ctas, rows_per_cta;
  long long room, needed, used;          // places of the workspace, those that the pass cannot do without, those of the CTAs
  long long parts, per_cta;              // CTAs that share a column's samples, samples of one
};
BackwardPlan plan_backward(abs_dtype dtype, int M, long long samples, long long tokens, long long d, unsigned long long align_bits,
                           bool with_gw, bool with_gb, bool totals, int sm_count, size_t workspace_bytes) {
  BackwardPlan p = {};
  const bool per_sample = with_gw || with_gb;
  const long long rows = samples * tokens;
  if (!per_sample) {               // only the totals: a replica's rows are one segment
    samples = rows > 0 ? 1 : 0;
    tokens = rows;
  }
  p.row = plan_row(dtype, d, align_bits, dtype == ABS_F32 ? 4 : 3, 2);
  p.sums = per_sample || totals;
  p.samples = samples;
  p.tokens = tokens;
  p.groups = 1;
  p.rows_per_cta = 1;
  p.parts = 1;
  p.per_cta = samples > 0 ? samples : 1;
  p.room = static_cast<long long>(workspace_bytes / (2 * sizeof(float))) / d;
  if (rows == 0) return p;
  const bool fast = p.row.tpr > 0;
  const long long total = rows * M, segments = samples * M;
  // Groups of a CTA share segments; short ones (up to two rows a group) are better off with CTAs of one group.
  if (fast) {
    const int full = kRingThreads / p.row.tpr;
    if (tokens >= 2 * full || !p.sums) p.groups = full;
    p.ctas = static_cast<long long>(sm_count) * (full / p.groups);
  } else {
    p.ctas = static_cast<long long>(sm_count) * 8 * kLnThreads / (d < kLnThreads ? kLnThreads : d);
    if (p.ctas < sm_count) p.ctas = sm_count;
  }
  const long long worth = (total + 2 * p.groups - 1) / (2 * p.groups);         // at least two rows a group
  if (p.ctas > worth) p.ctas = worth;
  const long long fewest = (total >> 30) + 1;                                  // a CTA counts its rows in 32 bits
  if (p.ctas < fewest) p.ctas = fewest;
  if (p.sums) {
    p.direct = with_gw && with_gb;
    p.needed = p.direct ? 2 * fewest : segments + fewest;
    if (p.room < p.needed) return p;
    const long long most = p.direct ? p.room / 2 : p.room - segments;          // (never below fewest)
    if (p.ctas > most) p.ctas = most;
  }
  p.rows_per_cta = (total + p.ctas - 1) / p.ctas;
  if (p.groups == 1 && p.sums && p.rows_per_cta > tokens) {
    // Whole segments.  Rounded down they take more CTAs, whose places the workspace has to have (direct: none is used then);
    // rounded up they never do.
    const long long down = p.rows_per_cta / tokens * tokens;
    const bool fits = p.direct || (total + down - 1) / down + segments <= p.room;
    p.rows_per_cta = fits || down == p.rows_per_cta ? down : down + tokens;
  }
  p.ctas = (total + p.rows_per_cta - 1) / p.rows_per_cta;
  p.whole = p.direct && p.rows_per_cta % tokens == 0;
  if (p.sums) p.used = p.whole ? 0 : p.direct ? 2 * p.ctas : p.ctas + segments;
  // 32 samples a CTA, where that fills the GPU no further than needed
  if (per_sample) {
    p.parts = (samples + 31) / 32;
    const long long most = 1 + 16ll * sm_count * 32 / (2 * d * M), fit = totals ? (p.room - p.used) / M : p.parts;
    if (p.parts > most) p.parts = most;
    if (p.parts > fit) p.parts = fit;
    if (p.parts < 1) p.parts = 1;
    p.per_cta = (samples + p.parts - 1) / p.parts;
    p.parts = (samples + p.per_cta - 1) / p.per_cta;
  }
  return p;
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
  const RowPlan plan = plan_row(dtype, d, row_bits(X, dtype, M, x_row_stride, x_worker_stride) |
                                              row_bits(Y, dtype, M, y_row_stride, y_worker_stride), 6, 1);
  if (plan.tpr > 0) {
    ABS_CUDA_TRY(ctx, dispatch_forward(ctx, a, dtype, plan, st));
    return ABS_OK;
  }
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
  const unsigned long long align_bits = row_bits(dY, dtype, M, dy_row_stride, dy_worker_stride) |
                                        row_bits(X, dtype, M, x_row_stride, x_worker_stride) |
                                        (dX ? row_bits(dX, dtype, M, dx_row_stride, dx_worker_stride) : 0);
  const BackwardPlan p = plan_backward(dtype, M, samples, tokens, d, align_bits, Gw != nullptr, Gb != nullptr, totals, ctx->sm_count,
                                       ctx->workspace_bytes);
  if (p.room < p.needed)
    return set_error(ctx, ABS_ERR_WORKSPACE, "the workspace holds %lld partial sums of %lld needed", p.room, p.needed);
  LnBackward a{dY, dy_row_stride, dy_worker_stride, X, x_row_stride, x_worker_stride, mean, rstd, weight, param_stride,
               dX, dx_row_stride, dx_worker_stride, M, p.samples, p.tokens, static_cast<int>(d), nullptr, p.rows_per_cta, nullptr,
               nullptr, 0, 0};
  LnReduce red{static_cast<const float*>(ctx->workspace), M, p.samples, p.tokens, p.rows_per_cta, static_cast<int>(d), p.direct,
               p.whole, p.per_cta, nullptr, Gw, Gb, g_row_stride, g_worker_stride, dW, dB, grad_stride};
  if (rows > 0) {
    if (p.sums) a.part = static_cast<float*>(ctx->workspace);
    if (p.direct) {
      a.Gw = Gw; a.Gb = Gb; a.g_rs = g_row_stride; a.g_ws = g_worker_stride;
    }
    if (p.parts > 1 && totals) red.totals = static_cast<float*>(ctx->workspace) + p.used * 2 * d;
    if (p.row.tpr > 0) {
      ABS_CUDA_TRY(ctx, dispatch_backward(ctx, a, dtype, p.row, p.groups, static_cast<unsigned>(p.ctas), st));
    } else {
      if (p.sums) {
        const dim3 grid(static_cast<unsigned>(p.ctas * ((d + kLnThreads - 1) / kLnThreads)));
        if (dtype == ABS_F32) ABS_CUDA_TRY(ctx, launch_dependent(ln_params_any_kernel<float>, grid, dim3(kLnThreads), 0, st, a));
        else ABS_CUDA_TRY(ctx, launch_dependent(ln_params_any_kernel<__nv_bfloat16>, grid, dim3(kLnThreads), 0, st, a));
      }
      if (dX) {                    // after the sums: dX may take the place of dY or X
        const dim3 grid(row_grid(ctx, rows * M));
        if (dtype == ABS_F32) ABS_CUDA_TRY(ctx, launch_dependent(ln_dx_any_kernel<float>, grid, dim3(kLnThreads), 0, st, a));
        else ABS_CUDA_TRY(ctx, launch_dependent(ln_dx_any_kernel<__nv_bfloat16>, grid, dim3(kLnThreads), 0, st, a));
      }
    }
  }
  if (!p.sums || (p.whole && !totals)) return ABS_OK;
  ABS_CUDA_TRY(ctx, launch_dependent(ln_reduce_kernel, dim3(static_cast<unsigned>((2 * d + 31) / 32), M, static_cast<unsigned>(p.parts)),
                                     dim3(kLnThreads), 0, st, red));
  if (red.totals)
    ABS_CUDA_TRY(ctx, launch_dependent(ln_total_kernel, dim3(static_cast<unsigned>((2 * d + kLnThreads - 1) / kLnThreads), M),
                                       dim3(kLnThreads), 0, st, red, static_cast<int>(p.parts)));
  return ABS_OK;
}

extern "C" int abs_plan_layer_norm_backward(abs_dtype dtype, int M, long long samples, long long tokens, long long d, int aligned,
                                            int with_gw, int with_gb, int with_totals, int sm_count, size_t workspace_bytes,
                                            abs_ln_backward_plan* out) {
  if (out == nullptr || M < 1 || samples < 0 || tokens < 0 || d < 1 || sm_count < 1 || (dtype != ABS_F32 && dtype != ABS_BF16) ||
      d > (1 << 24) || M > 65535 || (tokens > 0 && samples > (1ll << 40) / tokens))
    return ABS_ERR_INVALID_ARG;
  const BackwardPlan p = plan_backward(dtype, M, samples, tokens, d, aligned ? 0u : (dtype == ABS_F32 ? 4u : 2u), with_gw != 0,
                                       with_gb != 0, with_totals != 0, sm_count, workspace_bytes);
  memset(out, 0, sizeof(*out));
  out->route = p.row.tpr == 0 ? 2 : p.row.wide ? 0 : 1;
  out->groups = p.groups;
  out->samples = p.samples;
  out->tokens = p.tokens;
  out->ctas = p.ctas;
  out->rows_per_cta = p.rows_per_cta;
  out->direct = p.direct;
  out->parts = static_cast<int>(p.parts);
  out->room = p.room;
  out->needed = p.needed;
  out->used = p.used;
  return p.room < p.needed ? ABS_ERR_WORKSPACE : ABS_OK;
}
