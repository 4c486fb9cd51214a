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
  long long ldx, ldm;              // leading dimensions in elements, multiples of 8
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

// All steps of a group in one launch.
int launch_ns_steps(abs_ctx* ctx, const NsBuffers& w, int steps, float a, float b, float c, const NsScales& sc, bool split,
                    cudaStream_t st);

}  // namespace absk
