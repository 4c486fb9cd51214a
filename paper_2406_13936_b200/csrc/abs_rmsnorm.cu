// Root-mean-square norm with the residual's addition, forward and backward, for the rows of M replicas with weights of their own.
//
//   h = x + r,  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w      (or e4m3 with one scale a row)
//   xh = h rstd,  a = w dy,  dx = dh + rstd (a - xh mean(a xh)),  dw = sum_rows dy xh
//
// Each pass must read its inputs and write its outputs once; the arithmetic (5 and 9 operations an element) is far below
// what the memory rate leaves time for.  8 x 16384 x 768 bf16 with the residual: 128 us forward, 131 backward, 6.3 and 6.2 TB/s; fp32 239 and
// 327; 4099 x 4096 bf16 to 8 bits 18 us.  Through the kernels for any width 471, 596 and 70 (bf16).
#include <cuda_fp8.h>

#include "abs_tc.cuh"

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
// (never zero for a row that is not: the quotient of a subnormal number may round to it)
__device__ __forceinline__ float scale_of(unsigned top) {
  if (top == 0u) return 1.f;
  return top >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : fmaxf(__uint_as_float(top) / kE4m3Max, __uint_as_float(1u));
}
// y / scale: the product with the reciprocal and a correction by its remainder, which is exact (Markstein's method): the quotient's own rounding
// is all that is left, where the product alone rounds twice and takes an element at a border to the next step.  Scales below 2^-60 and their
// rows are taken 2^100 times (exact), so that neither the reciprocal overflows nor a remainder that matters underflows.  (4099 x 4096 bf16:
// 18.1 us; the product alone 17.3, a division an element 22.3.)
struct DivideBy {
  float up, scale, inv;
  __device__ __forceinline__ explicit DivideBy(float s) : up(s < 0x1p-60f ? 0x1p100f : 1.f), scale(s * up), inv(1.f / scale) {}
  __device__ __forceinline__ float operator()(float y) const {
    y *= up;
    const float q = y * inv;
    return fmaf(fmaf(-q, scale, y), inv, q);
  }
  // in pairs: what issues is what bounds a row in registers
  template <int V>
  __device__ __forceinline__ void all(float (&y)[V]) const {
    if constexpr (V == 1) {
      y[0] = (*this)(y[0]);
    } else {
      const uint64_t up2 = pack2f(up, up), less2 = pack2f(-scale, -scale), inv2 = pack2f(inv, inv);
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const uint64_t v = mul2f(pack2f(y[e], y[e + 1]), up2), q = mul2f(v, inv2);
        const float2 f = unpack2f(fma2f(fma2f(q, less2, v), inv2, q));
        y[e] = f.x;
        y[e + 1] = f.y;
      }
    }
  }
};
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
      const DivideBy by(scale);
      unsigned char* q = static_cast<unsigned char*>(a.q.p) + m * a.q.ws + r * a.q.rs;
      for (int j = threadIdx.x; j < a.d; j += kRmsThreads) q[j] = e4m3(by(again(j) * rstd * (w ? w[j] : 1.f)));
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

// Pieces -> segments -> replica, in a fixed order: 32 columns of one replica and `per` of its segments a CTA.  Eight lanes share the
// segments or, where there are few, the pieces of each.
struct RmsJoin {
  const float* part;                   // [M][samples][chunks][d], or NULL: the segments are in G
  int chunks;
  float* G;                            // segment i of replica m at m * g_ws + i * g_rs, or NULL (one segment)
  long long g_rs, g_ws;
  long long samples, per;
  float* total;                        // sums over segments at m * t_ws + blockIdx.z * d, or NULL
  long long t_ws;
  int d;
};
__global__ void __launch_bounds__(kRmsThreads)
rms_join_kernel(const RmsJoin a) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const long long m = blockIdx.y, i0 = blockIdx.z * a.per, i1 = i0 + a.per < a.samples ? i0 + a.per : a.samples;
  const bool in = col < a.d, by_segment = i1 - i0 >= 8 || a.part == nullptr;
  pdl_wait();
  float total = 0.f;
  if (a.part == nullptr) {
    if (in) {
      const float* p = a.G + m * a.g_ws + col;
#pragma unroll 8
      for (long long i = i0 + row; i < i1; i += 8) total += p[i * a.g_rs];
    }
  } else {
    for (long long i = by_segment ? i0 + row : i0; i < i1; i += by_segment ? 8 : 1) {
      const float* p = a.part + (m * a.samples + i) * a.chunks * a.d + col;
      float s = 0.f;
      if (in) {
#pragma unroll 8
        for (int c = by_segment ? 0 : row; c < a.chunks; c += by_segment ? 1 : 8) s += p[static_cast<long long>(c) * a.d];
      }
      if (!by_segment) {
        __syncthreads();
        red[row][lane] = s;
        __syncthreads();
        s = 0.f;
        if (row == 0) {
#pragma unroll
          for (int k = 0; k < 8; ++k) s += red[k][lane];
        }
      }
      if (in && (by_segment || row == 0)) {
        if (a.G) a.G[m * a.g_ws + i * a.g_rs + col] = s;
        total += s;
      }
    }
  }
  if (a.total == nullptr) return;
  __syncthreads();
  red[row][lane] = total;
  __syncthreads();
  if (row == 0 && in) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += red[k][lane];
    a.total[m * a.t_ws + static_cast<long long>(blockIdx.z) * a.d + col] = s;
  }
}
__global__ void __launch_bounds__(kRmsThreads)
rms_zero_kernel(float* p, long long ws, long long rs, long long n, int d) {
  pdl_wait();
  for (long long i = blockIdx.x; i < n; i += gridDim.x)
    for (int j = threadIdx.x; j < d; j += kRmsThreads) p[blockIdx.y * ws + i * rs + j] = 0.f;
}

// ---- rows in registers ------------------------------------------------------------------------------------
// A group of `tpr` threads has a row: thread t its pieces t, t + tpr, ... of V elements, at most NV of them.  Pieces are of 16 bytes
// where all rows are aligned to that, else of 8 or 4, or of one element.
constexpr int kMostRow = 512;                        // threads of a row
template <typename T, int V> struct RmsPiece;
template <> struct RmsPiece<float, 4> { typedef uint4 Raw; };
template <> struct RmsPiece<float, 2> { typedef uint2 Raw; };
template <> struct RmsPiece<float, 1> { typedef uint32_t Raw; };
template <> struct RmsPiece<__nv_bfloat16, 8> { typedef uint4 Raw; };
template <> struct RmsPiece<__nv_bfloat16, 4> { typedef uint2 Raw; };
template <> struct RmsPiece<__nv_bfloat16, 2> { typedef uint32_t Raw; };
template <> struct RmsPiece<__nv_bfloat16, 1> { typedef unsigned short Raw; };
__device__ __forceinline__ void open_two(uint32_t r, float& a, float& b) {
  a = __uint_as_float(r << 16);
  b = __uint_as_float(r & 0xffff0000u);
}
template <typename T, int V>
__device__ __forceinline__ void open_piece(const typename RmsPiece<T, V>::Raw& r, float (&x)[V]) {
  if constexpr (V * sizeof(T) == 16) {
    Vec<T>::unpack(r, x);
  } else if constexpr (sizeof(T) == 4) {
    if constexpr (V == 2) {
      x[0] = __uint_as_float(r.x);
      x[1] = __uint_as_float(r.y);
    } else {
      x[0] = __uint_as_float(r);
    }
  } else if constexpr (V == 4) {
    open_two(r.x, x[0], x[1]);
    open_two(r.y, x[2], x[3]);
  } else if constexpr (V == 2) {
    open_two(r, x[0], x[1]);
  } else {
    x[0] = __uint_as_float(static_cast<uint32_t>(r) << 16);
  }
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T, int V>
__device__ __forceinline__ typename RmsPiece<T, V>::Raw close_piece(const float (&x)[V]) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(x[0]);
    else return __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
  } else if constexpr (V == 2) {
    if constexpr (sizeof(T) == 4) return make_uint2(__float_as_uint(x[0]), __float_as_uint(x[1]));
    else return two_bf16(x[0], x[1]);
  } else if constexpr (V * sizeof(T) == 8) {
    return make_uint2(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]));
  } else if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    return make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
  }
}
template <int V>
__device__ __forceinline__ void weights_of(const float* w, int at, float (&x)[V]) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = 1.f;
  } else if constexpr (V < 4) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = __ldg(w + at + e);
  } else if ((reinterpret_cast<uintptr_t>(w) & 15u) == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(w + at + e));
      x[e] = f.x; x[e + 1] = f.y; x[e + 2] = f.z; x[e + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = __ldg(w + at + e);
  }
}
template <int V>
__device__ __forceinline__ void store_e4m3(unsigned char* q, const float (&x)[V]) {
  if constexpr (V == 1) {
    *q = e4m3(x[0]);
  } else if constexpr (V == 2) {
    *reinterpret_cast<unsigned short*>(q) = __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3);
  } else {
    uint32_t w[V / 4];
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[e], x[e + 1]), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[e + 2], x[e + 3]), __NV_SATFINITE, __NV_E4M3);
      w[e / 4] = lo | (hi << 16);
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
  }
}
// Sum (or largest) over a group's threads, the same in each.  red: 32 words of the group, used by one of these at a time.
template <bool ONE_WARP>
__device__ __forceinline__ float group_sum(float v, float* red, int group, int t, int tpr) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  if constexpr (ONE_WARP) return v;
  if ((t & 31) == 0) red[t >> 5] = v;
  named_bar_sync(1 + group, tpr);
  v = 0.f;
  for (int w = 0; w < tpr / 32; ++w) v += red[w];
  return v;
}
template <bool ONE_WARP>
__device__ __forceinline__ unsigned group_max(unsigned v, float* red, int group, int t, int tpr) {
  v = __reduce_max_sync(0xffffffffu, v);
  if constexpr (ONE_WARP) return v;
  if ((t & 31) == 0) red[t >> 5] = __uint_as_float(v);
  named_bar_sync(1 + group, tpr);
  for (int w = 0; w < tpr / 32; ++w) v = max(v, __float_as_uint(red[w]));
  return v;
}

// A row a group, one each; the bytes under way come from the number of groups on an SM, so at most 64 registers a thread.  (A group that
// loads its next row ahead needs 100 and more: 4099 x 4096 bf16 27 us for 23.)
template <typename T, int V, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(ONE_WARP ? 256 : kMostRow, ONE_WARP ? 4 : 2)
rms_forward_kernel(const RmsForward a, int tpr, int pieces) {
  typedef typename RmsPiece<T, V>::Raw Raw;
  __shared__ float red_mem[2][4][32];
  const int group = threadIdx.x / tpr, t = threadIdx.x - group * tpr, groups = blockDim.x / tpr;
  const unsigned rows = static_cast<unsigned>(a.rows), rr = blockIdx.x * groups + group;      // (at most 2^31 of all replicas)
  pdl_wait();
  if (rr >= rows * a.M) return;                      // (a whole group: its barriers are its own)
  const long long m = rr / rows, r = rr - m * rows;
  const Raw* x = reinterpret_cast<const Raw*>(static_cast<const T*>(a.x.p) + m * a.x.ws + r * a.x.rs);
  const Raw* res = reinterpret_cast<const Raw*>(static_cast<const T*>(a.r.p) + m * a.r.ws + r * a.r.rs);
  Raw rx[NV], rr_[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + k * tpr;
    if (v < pieces) {
      rx[k] = __ldcs(x + v);
      if (a.r.p) rr_[k] = __ldcs(res + v);
    }
  }
  float h[NV][V];
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + k * tpr;
    if (v < pieces) {
      open_piece<T, V>(rx[k], h[k]);
      if (a.r.p) {
        float o[V];
        open_piece<T, V>(rr_[k], o);
#pragma unroll
        for (int e = 0; e < V; ++e) h[k][e] += o[e];
        const Raw sum = close_piece<T, V>(h[k]);
        open_piece<T, V>(sum, h[k]);
        if (a.h.p) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.h.p) + m * a.h.ws + r * a.h.rs) + v, sum);
      } else if (a.h.p) {
        __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.h.p) + m * a.h.ws + r * a.h.rs) + v, rx[k]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) s = fmaf(h[k][e], h[k][e], s);
    }
  }
  s = group_sum<ONE_WARP>(s, red_mem[0][ONE_WARP ? 0 : group], group, t, tpr);
  const float rstd = 1.0f / sqrtf(s / static_cast<float>(a.d) + a.eps);
  const float* weight = a.weight ? a.weight + m * a.p_stride : nullptr;
  unsigned top = 0u;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + k * tpr;
    if (v < pieces) {
      float w[V];
      weights_of<V>(weight, v * V, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        h[k][e] = h[k][e] * rstd * w[e];
        top = max(top, magnitude(h[k][e]));
      }
      if (a.y.p) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.y.p) + m * a.y.ws + r * a.y.rs) + v, close_piece<T, V>(h[k]));
    }
  }
  if (a.q.p) {
    const float scale = scale_of(group_max<ONE_WARP>(top, red_mem[1][ONE_WARP ? 0 : group], group, t, tpr));
    const DivideBy by(scale);
    unsigned char* q = static_cast<unsigned char*>(a.q.p) + m * a.q.ws + r * a.q.rs;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) {
        by.all<V>(h[k]);
        store_e4m3<V>(q + v * V, h[k]);
      }
    }
    if (t == 0) a.scales[rr] = scale;
  }
  if (t == 0 && a.rstd) a.rstd[rr] = rstd;
}

// ---- rows through a ring in shared memory ------------------------------------------------------------------------
// Backward, rows of whole 16-byte pieces up to 4096 fp32 or 8192 bf16 columns (200 KB of ring); all others go through the kernels for any
// width, which read them twice or thrice in single elements (16384 x 1020 bf16 91 us, 1024 columns 42; 2000 x 8192 fp32 130 us, the memory
// rate allows 30).  A thread copies its own pieces of the rows ahead into its own places of a ring (cp.async), so what is
// under way does not depend on registers and nobody waits for anybody else's copies.  A CTA has a piece of a segment and its groups take
// the rows in turn, the sums of dw staying in registers; or (by_group) every group has a segment of its own.
constexpr int kDeep = 4;                             // rows of a group's ring
__device__ __forceinline__ void ring_copy(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <typename T, int NV, bool ONE_WARP>
__global__ void __launch_bounds__(ONE_WARP ? 128 : kMostRow)
rms_backward_ring_kernel(const RmsBackward a, int tpr, int pieces, int by_group) {
  constexpr int V = 16 / sizeof(T);
  extern __shared__ __align__(16) unsigned char ring_mem[];          // [kDeep][3][NV][threads] pieces; the groups' sums afterwards
  __shared__ float red_mem[2][4][32];
  const int group = threadIdx.x / tpr, t = threadIdx.x - group * tpr, groups = blockDim.x / tpr;
  const uint32_t step = blockDim.x * 16u, mine = smem_u32(ring_mem) + threadIdx.x * 16u;
  const long long job = by_group ? static_cast<long long>(blockIdx.x) * groups + group : blockIdx.x;
  const long long segments = static_cast<long long>(a.M) * a.samples;
  const long long seg = by_group ? job : job / a.chunks;
  const bool live = seg < segments;
  const long long m = live ? seg / a.samples : 0;
  const long long first = by_group || !live ? 0 : (job - seg * a.chunks) * a.chunk;
  const long long n = !live ? 0 : by_group ? a.tokens : (a.tokens - first < a.chunk ? a.tokens - first : a.chunk);
  const int stride = by_group ? 1 : groups, off = by_group ? 0 : group;
  const int count = n > off ? static_cast<int>((n - off + stride - 1) / stride) : 0;                 // this group's rows
  long long row = live ? (seg - m * a.samples) * a.tokens + first + off : 0;                         // of the replica
  const bool with_dh = a.dh.p != nullptr;
  const char* c_dy = reinterpret_cast<const char*>(static_cast<const T*>(a.dy.p) + m * a.dy.ws + row * a.dy.rs) + t * 16;
  const char* c_h = reinterpret_cast<const char*>(static_cast<const T*>(a.h.p) + m * a.h.ws + row * a.h.rs) + t * 16;
  const char* c_dh = reinterpret_cast<const char*>(static_cast<const T*>(a.dh.p) + m * a.dh.ws + row * a.dh.rs) + t * 16;
  const float* rstd_in = a.rstd + m * a.samples * a.tokens + row;
  pdl_wait();
  int copied = 0;
  uint32_t c_at = 0;
  auto copy_row = [&]() {
    if (copied < count) {
      const uint32_t to = mine + c_at * (3u * NV) * step;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * tpr < pieces) {
          ring_copy(to + k * step, c_dy + k * tpr * 16);
          ring_copy(to + (NV + k) * step, c_h + k * tpr * 16);
          if (with_dh) ring_copy(to + (2 * NV + k) * step, c_dh + k * tpr * 16);
        }
      }
      ++copied;
      c_dy += stride * a.dy.rs * sizeof(T);
      c_h += stride * a.h.rs * sizeof(T);
      c_dh += stride * a.dh.rs * sizeof(T);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    c_at = c_at + 1 == kDeep ? 0 : c_at + 1;
  };
#pragma unroll
  for (int k = 0; k < kDeep - 1; ++k) copy_row();
  float next = count > 0 ? __ldg(rstd_in) : 0.f;
  const float* weight = a.weight ? a.weight + m * a.p_stride : nullptr;
  float dw[NV][V], kept[ONE_WARP ? NV : 1][V];       // (a row of one warp leaves registers for the weight)
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int e = 0; e < V; ++e) dw[k][e] = 0.f;
    if (ONE_WARP && t + k * tpr < pieces) weights_of<V>(weight, (t + k * tpr) * V, kept[k]);
  }
  const float inv_d = 1.0f / static_cast<float>(a.d);
  uint32_t at = 0;
  int flip = 0;
  for (int i = 0; i < count; ++i) {
    copy_row();
    const float rstd = next;
    rstd_in += stride;
    if (i + 1 < count) next = __ldg(rstd_in);
    asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 1) : "memory");
    const uint32_t from = mine + at * (3u * NV) * step;
    at = at + 1 == kDeep ? 0 : at + 1;
    float g[NV][V], xh[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) {
        float w[V];
        Vec<T>::unpack(lds128(from + k * step), g[k]);
        Vec<T>::unpack(lds128(from + (NV + k) * step), xh[k]);
        if constexpr (!ONE_WARP) weights_of<V>(weight, v * V, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if constexpr (ONE_WARP) w[e] = kept[k][e];
          xh[k][e] *= rstd;
          dw[k][e] = fmaf(g[k][e], xh[k][e], dw[k][e]);
          g[k][e] *= w[e];
          s = fmaf(g[k][e], xh[k][e], s);
        }
      }
    }
    if (a.dx.p != nullptr) {
      const float c = group_sum<ONE_WARP>(s, red_mem[flip][ONE_WARP ? 0 : group], group, t, tpr) * inv_d;
      flip ^= 1;
      char* dx = reinterpret_cast<char*>(static_cast<T*>(a.dx.p) + m * a.dx.ws + row * a.dx.rs);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int v = t + k * tpr;
        if (v < pieces) {
          float o[V];
          if (with_dh) {
            Vec<T>::unpack(lds128(from + (2 * NV + k) * step), o);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = fmaf(rstd, fmaf(-xh[k][e], c, g[k][e]), o[e]);
          __stcs(reinterpret_cast<uint4*>(dx) + v, close_piece<T, V>(o));
        }
      }
    }
    row += stride;
  }
  if (a.out == nullptr) return;
  float* out = a.part ? a.part + job * a.d : a.out + m * a.o_ws + (seg - m * a.samples) * a.o_rs;
  if (!by_group && groups > 1) {                     // the groups' sums, in order, through the ring's place
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float* sums = reinterpret_cast<float*>(ring_mem);
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int v = t + k * tpr;
        if (v < pieces) {
#pragma unroll
          for (int e = 0; e < V; e += 4)
            *reinterpret_cast<float4*>(sums + static_cast<size_t>(group - 1) * a.d + v * V + e) = make_float4(dw[k][e], dw[k][e + 1], dw[k][e + 2], dw[k][e + 3]);
        }
      }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = t + k * tpr;
      if (v < pieces) {
        for (int o = 0; o < groups - 1; ++o) {
#pragma unroll
          for (int e = 0; e < V; e += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sums + static_cast<size_t>(o) * a.d + v * V + e);
            dw[k][e] += f.x; dw[k][e + 1] += f.y; dw[k][e + 2] += f.z; dw[k][e + 3] += f.w;
          }
        }
      }
    }
  }
  if (!live) return;
  const bool wide = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = t + k * tpr;
    if (v < pieces) {
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        if (wide) {
          *reinterpret_cast<float4*>(out + v * V + e) = make_float4(dw[k][e], dw[k][e + 1], dw[k][e + 2], dw[k][e + 3]);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) out[v * V + e + q] = dw[k][e + q];
        }
      }
    }
  }
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
  long long groups, per_group;       // CTAs that share a column's segments, segments of one
  size_t sums_at;                    // floats in front of those CTAs' totals
};
RmsPlan plan_rms(int M, long long samples, long long tokens, long long d, bool per_sample, bool totals, long long jobs_wanted,
                 bool by_group, int sm_count, size_t workspace_bytes) {
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
  if (chunks < 1 || by_group) chunks = 1;
  p.chunk = (tokens + chunks - 1) / chunks;
  if (p.chunk < 1) p.chunk = 1;
  p.chunks = static_cast<int>(tokens > 0 ? (tokens + p.chunk - 1) / p.chunk : 1);
  const long long used = p.chunks > 1 ? p.chunks * samples * M : 0;
  p.sums_at = static_cast<size_t>(used) * d;
  // segments of a CTA of rms_join_kernel: as many CTAs as fill the GPU twice, eight segments at least
  const long long wide = (d + 31) / 32 * M;
  p.groups = (2 * sm_count + wide - 1) / wide;
  if (p.groups > (samples + 7) / 8) p.groups = (samples + 7) / 8;
  if (totals && p.groups > 1 && p.groups * M > room - used) p.groups = (room - used) / M;
  if (p.groups < 1) p.groups = 1;
  p.per_group = (samples + p.groups - 1) / p.groups;
  p.groups = (samples + p.per_group - 1) / p.per_group;
  return p;
}

unsigned long long rms_bits(const void* p, int es, int M, long long rs, long long ws) {
  return p == nullptr ? 0 : reinterpret_cast<uintptr_t>(p) | static_cast<unsigned long long>(rs) * es | (M > 1 ? static_cast<unsigned long long>(ws) * es : 0);
}
// Threads of a row of `pieces`, at most `most` pieces each; 0: too wide.
int threads_of(long long pieces, int most) {
  for (int tpr = 32; tpr <= kMostRow; tpr *= 2)
    if (pieces <= static_cast<long long>(tpr) * most) return tpr;
  return 0;
}
template <typename T, int V, int NV>
int launch_forward(abs_ctx* ctx, const RmsForward& a, int tpr, cudaStream_t st) {
  const int groups = tpr < 256 ? 256 / tpr : 1;
  const long long grid = (a.rows * a.M + groups - 1) / groups;
  auto kern = tpr == 32 ? rms_forward_kernel<T, V, NV, true> : rms_forward_kernel<T, V, NV, false>;
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(static_cast<unsigned>(grid)), dim3(tpr * groups), 0, st, a, tpr, a.d / V));
  return ABS_OK;
}
// 32 elements a thread at most, 16 single ones.  Row, residual and sum are all held: bf16 pieces of 16 and 8 bytes fit 64 registers; rows of
// 32 fp32 elements a thread, in pieces of 16 and 8 bytes, spill 100 to 148 bytes, the other full rows up to 56 (16384 x 4096 fp32 122 us, 210 with
// the residual, of 82 and 164 that the memory rate allows).  Rows of 16384 x 1020, 1022 and 1021 bf16, pieces of 8, 4 and 2 bytes: 18, 31, 53 us
// for 15 at 1024.
template <typename T, int V>
int run_pieces(abs_ctx* ctx, const RmsForward& a, cudaStream_t st) {
  const int tpr = threads_of(a.d / V, 32 / V > 16 ? 16 : 32 / V), nv = (a.d / V + tpr - 1) / tpr;
  if constexpr (V == 8) {
    switch (nv) {
      case 1: return launch_forward<T, V, 1>(ctx, a, tpr, st);
      case 2: return launch_forward<T, V, 2>(ctx, a, tpr, st);
      case 3: return launch_forward<T, V, 3>(ctx, a, tpr, st);
      default: return launch_forward<T, V, 4>(ctx, a, tpr, st);
    }
  } else if constexpr (V == 4) {
    return nv <= 2 ? launch_forward<T, V, 2>(ctx, a, tpr, st) : nv <= 4 ? launch_forward<T, V, 4>(ctx, a, tpr, st)
         : nv <= 6 ? launch_forward<T, V, 6>(ctx, a, tpr, st) : launch_forward<T, V, 8>(ctx, a, tpr, st);
  } else {
    return nv <= 4 ? launch_forward<T, V, 4>(ctx, a, tpr, st) : nv <= 8 ? launch_forward<T, V, 8>(ctx, a, tpr, st) : launch_forward<T, V, 16>(ctx, a, tpr, st);
  }
}
template <typename T>
int run_forward(abs_ctx* ctx, const RmsForward& a, cudaStream_t st) {
  constexpr int es = sizeof(T);
  const unsigned long long bits = rms_bits(a.x.p, es, a.M, a.x.rs, a.x.ws) | rms_bits(a.r.p, es, a.M, a.r.rs, a.r.ws) |
                                  rms_bits(a.h.p, es, a.M, a.h.rs, a.h.ws) | rms_bits(a.y.p, es, a.M, a.y.rs, a.y.ws) |
                                  static_cast<unsigned long long>(a.d) * es;
  const unsigned long long q_bits = rms_bits(a.q.p, 1, a.M, a.q.rs, a.q.ws);
  auto takes = [&](int V) { return (bits & (V * es - 1)) == 0 && (q_bits & (V - 1)) == 0 && threads_of(a.d / V, 32 / V > 16 ? 16 : 32 / V) > 0; };
  if (a.rows <= (1ll << 31) / a.M) {
    if constexpr (es == 2) {
      if (takes(8)) return run_pieces<T, 8>(ctx, a, st);
    }
    if (takes(4)) return run_pieces<T, 4>(ctx, a, st);
    if (takes(2)) return run_pieces<T, 2>(ctx, a, st);
    if (takes(1)) return run_pieces<T, 1>(ctx, a, st);
  }
  ABS_CUDA_TRY(ctx, launch_dependent(rms_forward_any_kernel<T>, dim3(rms_grid(ctx, a.rows * a.M)), dim3(kRmsThreads), 0, st, a));
  return ABS_OK;
}

// How a backward pass runs: rows in rings (threads of a row, pieces of a thread, threads of a CTA), or tpr = 0.
struct RmsRows {
  int tpr, NV, threads, by_group;
};
template <typename T>
RmsRows plan_rows(const RmsBackward& a, long long tokens) {
  constexpr int V = 16 / sizeof(T), es = sizeof(T);
  const unsigned long long bits = rms_bits(a.dy.p, es, a.M, a.dy.rs, a.dy.ws) | rms_bits(a.h.p, es, a.M, a.h.rs, a.h.ws) |
                                  rms_bits(a.dh.p, es, a.M, a.dh.rs, a.dh.ws) | rms_bits(a.dx.p, es, a.M, a.dx.rs, a.dx.ws) |
                                  static_cast<unsigned long long>(a.d) * es;
  RmsRows r = {0, 0, 0, 0};
  if ((bits & 15u) != 0) return r;
  r.tpr = threads_of(a.d / V, 4);
  if (r.tpr == 0) return r;
  r.NV = (a.d / V + r.tpr - 1) / r.tpr;
  r.threads = r.tpr < 128 ? 128 : r.tpr;
  if (static_cast<size_t>(kDeep) * 3 * r.NV * r.threads * 16 > 200 * 1024) r.tpr = 0;
  r.by_group = tokens < r.threads / (r.tpr ? r.tpr : 1);
  return r;
}
template <typename T, int NV>
int launch_backward(abs_ctx* ctx, const RmsBackward& a, const RmsRows& r, cudaStream_t st) {
  const int groups = r.threads / r.tpr;
  const size_t smem = static_cast<size_t>(kDeep) * 3 * NV * r.threads * 16;       // (three times what the groups' sums take, or more)
  const long long jobs = r.by_group ? (static_cast<long long>(a.M) * a.samples + groups - 1) / groups : static_cast<long long>(a.M) * a.samples * a.chunks;
  auto kern = r.tpr == 32 ? rms_backward_ring_kernel<T, NV, true> : rms_backward_ring_kernel<T, NV, false>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(static_cast<unsigned>(jobs)), dim3(r.threads), smem, st, a, r.tpr,
                                     static_cast<int>(a.d * sizeof(T) / 16), r.by_group));
  return ABS_OK;
}
template <typename T>
int run_backward(abs_ctx* ctx, const RmsBackward& a, bool sums, const RmsRows& r, cudaStream_t st) {
  if (r.tpr > 0) {
    switch (r.NV) {
      case 1: return launch_backward<T, 1>(ctx, a, r, st);
      case 2: return launch_backward<T, 2>(ctx, a, r, st);
      case 3: return launch_backward<T, 3>(ctx, a, r, st);
      default: return launch_backward<T, 4>(ctx, a, r, st);
    }
  }
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
  RmsBackward a{{dY, dy_row_stride, dy_worker_stride}, {H, h_row_stride, h_worker_stride}, {dH, dh_row_stride, dh_worker_stride}, rstd,
                weight, param_stride, {dX, dx_row_stride, dx_worker_stride}, M, samples, tokens, static_cast<int>(d), 0, 1, nullptr, nullptr,
                0, 0};
  // (without Gw a replica's rows are one segment)
  const RmsRows r = dtype == ABS_F32 ? plan_rows<float>(a, Gw ? tokens : rows) : plan_rows<__nv_bfloat16>(a, Gw ? tokens : rows);
  const RmsPlan p = plan_rms(M, samples, tokens, d, Gw != nullptr, dW != nullptr, ctx->sm_count * 8ll, r.by_group != 0, ctx->sm_count, ctx->workspace_bytes);
  a.samples = p.samples;
  a.tokens = p.tokens;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  a.out = Gw ? Gw : dW;
  a.o_rs = Gw ? g_row_stride : 0;
  a.o_ws = Gw ? g_worker_stride : grad_stride;
  float* ws = static_cast<float*>(ctx->workspace);
  if (p.chunks > 1) a.part = ws;
  rc = dtype == ABS_F32 ? run_backward<float>(ctx, a, sums, r, st) : run_backward<__nv_bfloat16>(ctx, a, sums, r, st);
  if (rc != ABS_OK || !sums) return rc;
  if (p.chunks == 1 && !(Gw && dW)) return ABS_OK;          // in place already
  const bool two = dW != nullptr && p.groups > 1;
  const RmsJoin j{a.part, p.chunks, Gw, g_row_stride, g_worker_stride, p.samples, p.per_group, two ? ws + p.sums_at : dW,
                  two ? p.groups * d : grad_stride, static_cast<int>(d)};
  ABS_CUDA_TRY(ctx, launch_dependent(rms_join_kernel, dim3(col_tiles, M, static_cast<unsigned>(p.groups)), dim3(kRmsThreads), 0, st, j));
  if (two) {
    const RmsJoin k{nullptr, 1, ws + p.sums_at, d, p.groups * d, p.groups, p.groups, dW, grad_stride, static_cast<int>(d)};
    ABS_CUDA_TRY(ctx, launch_dependent(rms_join_kernel, dim3(col_tiles, M), dim3(kRmsThreads), 0, st, k));
  }
  return ABS_OK;
}
