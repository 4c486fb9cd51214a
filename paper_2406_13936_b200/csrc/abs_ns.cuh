// Newton-Schulz orthogonalisation: what the elementwise passes (abs_muon.cu) and the tensor-core
// products (abs_ns_gemm.cu) share.
//
// One matrix is held with its short side as rows, X [m][n], m <= n (a tall matrix is transposed when
// it is read and again when the result is written), as two fp16 matrices, values and remainders (22
// bits).  A step is
//   A = X X',   B = b A + c A A,   X <- a X + B X,
// three products whose operands are the values; the a X term takes the remainders too, so what 11
// bits of an operand lose is always in proportion to B X and never fills directions that the
// gradient does not have (see abs_muon.cu).  With split operands A and B have remainders as well and
// a product is three tensor-core products.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "abs_internal.cuh"

namespace absk {

constexpr int kNsMaxSteps = 32;

// Powers of two by which a step's matrices are stored, so that fp16 neither overflows nor wastes its
// range (largest possible entry at most 2^14).
struct NsScales {
  float sx[kNsMaxSteps + 1];   // X before step k (and after the last one)
  float ta[kNsMaxSteps];       // A
  float tb[kNsMaxSteps];       // B
};

// Device buffers of one group of Z matrices.  Step k reads the X of k & 1 and writes the other.
struct NsBuffers {
  int Z, m, n;
  long long ldx, ldm;              // leading dimensions in elements, multiples of 64
  __half* xh[2];
  __half* xl[2];                   // remainders; without split operands only [0], changed in place
  __half* ah;
  __half* bh;
  __half* al;                      // split operands only
  __half* bl;
  double* part;                    // [Z][kNormParts] partial sums of squares
  unsigned* progress;              // [Z][3][kNsRowBlocks(m)] finished tiles of X, A, B, zero before the products
};
constexpr int kNormParts = 1184;
constexpr int kNsFlagWord = 8;     // word of abs_ctx::flags that a product whose wait ran out sets (cleared by every call)
inline int ns_row_blocks(int m) { return (m + 127) / 128; }

// Where the matrices of a call live: matrix q is worker q / L, layer q % L.
struct NsSource {
  const void* G;          // orthogonalise: the input; Muon: the gradients
  int src_bf16;
  float* Buf;             // Muon: momentum buffers
  float momentum;
  int nesterov;
  int muon;
  int L;
  long long replica_stride, matrix_stride, row_stride;
  int rows, cols;
};
struct NsTarget {
  void* O;                // orthogonalise: the result
  int dst_bf16;
  float* X;               // Muon: the parameters
  float decay, step;      // x <- decay x - step o
  long long replica_stride, matrix_stride, row_stride;
};

struct NsCoef {
  float in, acc;              // result of a product = in * (what it is added to) + acc * accumulator
};
inline void ns_coefs(NsCoef (&out)[3], float a, float b, float c, const NsScales& sc, int step) {
  const float sx = sc.sx[step], ta = sc.ta[step], tb = sc.tb[step], next = sc.sx[step + 1];
  out[0] = {0.f, ta / (sx * sx)};                  // A = X X'
  out[1] = {b * (tb / ta), c * (tb / (ta * ta))};  // B = b A + c A A
  out[2] = {a * (next / sx), next / (tb * sx)};    // X <- a X + B X
}

#ifdef __CUDACC__
__device__ __forceinline__ long long matrix_base(int q, int L, long long replica_stride, long long matrix_stride) {
  const int m = q / L;
  return m * replica_stride + static_cast<long long>(q - m * L) * matrix_stride;
}
template <int V>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[V]) {
  if constexpr (V == 4) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    v[0] = *p;
  }
}
template <int V>
__device__ __forceinline__ void store_f32(float* p, const float (&v)[V]) {
  if constexpr (V == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else *p = v[0];
}
// V consecutive elements at index i of the source, fp32 or bf16.
template <int V>
__device__ __forceinline__ void load_src(const NsSource& s, long long i, float (&v)[V]) {
  if (s.src_bf16) {
    const unsigned short* p = static_cast<const unsigned short*>(s.G) + i;
    if constexpr (V == 4) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      v[0] = __uint_as_float(u.x << 16);
      v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16);
      v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      v[0] = __uint_as_float(static_cast<uint32_t>(*p) << 16);
    }
  } else {
    load_f32<V>(static_cast<const float*>(s.G) + i, v);
  }
}
// The matrix to orthogonalise, after ns_norm_kernel has updated the momentum buffer.
template <int V>
__device__ __forceinline__ void load_update(const NsSource& s, long long i, float (&u)[V]) {
  if (!s.muon) {
    load_src<V>(s, i, u);
    return;
  }
  load_f32<V>(s.Buf + i, u);
  if (s.nesterov) {
    float g[V];
    load_src<V>(s, i, g);
#pragma unroll
    for (int e = 0; e < V; ++e) u[e] = fmaf(s.momentum, u[e], g[e]);
  }
}
#endif

// The whole call for matrices with a side of at most 128 in one launch (one cluster per matrix, everything in
// shared memory), or ABS_ERR_UNSUPPORTED where they do not fit.
int launch_ns_small(abs_ctx* ctx, const NsSource& s, const NsTarget& t, int count, float eps, const NsScales& sc, int steps,
                    float a, float b, float c, cudaStream_t st);
// CTAs of its clusters, 0 where the matrices do not fit; clusters beyond kPortableCluster are the device's to hold or not.
int ns_small_cluster(int count, long long rows, long long cols);
constexpr int kPortableCluster = 8;
bool ns_small_resident(abs_ctx* ctx, int cluster);

// All steps of a group in one launch.
int launch_ns_steps(abs_ctx* ctx, const NsBuffers& w, int steps, float a, float b, float c, const NsScales& sc, bool split,
                    cudaStream_t st);

}  // namespace absk
