/*
 * abs.h -- C ABI of the adaptive-batch-size test and the fused local-optimiser
 * kernels for NVIDIA B200 (sm_100a).
 *
 * The library implements the per-round batch-size test of the adaptive local
 * batch size method for local gradient methods and the parameter updates around
 * it, for M simulated workers held as replicas on ONE GPU:
 *
 *   abs_test_stats     mean gradient, norm-test variance, inner-product and
 *                      orthogonality variances of per-sample gradients
 *                      (Eq. batch_grad, Eq. def_var, Eq. approx_norm_local)
 *   abs_next_batch     the ceilings T^m, max{T, b}, the maximum over workers and
 *                      the cap (Eq. norm_test, Eq. test_stat, Algorithm 1)
 *   local_sgd_step     x^m <- x^m - alpha g^m           (Eq. local_sgd_alt, line 1)
 *   local_adamw_step   AdamW inner optimiser             (Section 4.2, Appendix C.2)
 *   local_shb_step     momentum-SGD inner optimiser      (Section 6.1)
 *   replica_average    x^m <- (1/M) sum_m x^m            (Eq. local_sgd_alt, line 2)
 *   local_muon_step    orthogonalised-momentum (Muon) inner optimiser for matrices
 *   abs_layer_norm, abs_layer_norm_backward
 *                      layer norm; its backward pass also gives per-sample gradient
 *                      rows of weight and bias for the test
 *   abs_rms_norm, abs_rms_norm_backward
 *                      root-mean-square norm with the residual's addition
 *   abs_attention, abs_attention_backward
 *                      causal attention with grouped heads over packed sequences
 *   abs_embedding, abs_embedding_backward
 *                      token embedding of the replicas
 *
 * Conventions
 *   - Every function returns an int: ABS_OK (0) or a negative ABS_ERR_* code.
 *     Nothing throws across this boundary.  abs_last_error() gives a message.
 *   - Unless a parameter says "host", every tensor pointer is a DEVICE pointer
 *     owned by the caller, on the device the context was created for.
 *   - Calls only enqueue work on `stream` (a cudaStream_t passed as void*; NULL
 *     is the legacy default stream).  They do not synchronise; results are
 *     valid in stream order.  The *_host variants are the exception: they copy,
 *     run and synchronise before returning.
 *   - A context owns a workspace for per-CTA partial sums.  Calls that use the
 *     same context must be issued in stream order on one stream at a time.
 *   - Data-dependent conditions (non-finite input, zero mean gradient, a
 *     copy that never completed) are reported in abs_stats.status on the
 *     device; they never trap.
 *   - Strides are in ELEMENTS of the tensor's type.  All index arithmetic is
 *     64-bit.
 */
#ifndef ABS_H_
#define ABS_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- error codes ---------------------------------------------------------- */
#define ABS_OK                0
#define ABS_ERR_INVALID_ARG  -1   /* null pointer, b < 2, d < 1, stride < extent, ...        */
#define ABS_ERR_UNSUPPORTED  -2   /* shape outside what the kernels cover (stated per call)  */
#define ABS_ERR_WORKSPACE    -3   /* the context's workspace is too small for this call      */
#define ABS_ERR_CUDA         -4   /* a CUDA runtime / driver call failed                     */
#define ABS_ERR_NO_DEVICE    -5   /* no usable sm_100 device; there is no CPU fallback       */

/* ---- status bits written to abs_stats.status ------------------------------ */
#define ABS_STATUS_NONFINITE  1u  /* an input or an accumulator was not finite (or overflowed) */
#define ABS_STATUS_ZERO_MEAN  2u  /* ||gbar||^2 == 0: the test ratios are undefined            */
#define ABS_STATUS_NORM_ONLY  8u  /* a record merged from sub-batches: only gbar_sq, var_norm,
                                     sum_sq and rows are meaningful (abs_stats_merge)          */
#define ABS_STATUS_TIMEOUT    4u  /* an asynchronous tile copy did not arrive in time; the
                                     numbers in this record are not valid                      */

typedef struct abs_ctx abs_ctx;   /* opaque */

/* Creates a context bound to CUDA device `device` (must be compute capability
 * 10.x; otherwise ABS_ERR_NO_DEVICE).  workspace_bytes = 0 selects the default
 * (64 MiB), enough for b <= 4096 rows and M <= 64 workers.  The context owns
 * its device allocations until abs_destroy. */
int abs_create(abs_ctx** out, int device, size_t workspace_bytes);
int abs_destroy(abs_ctx* ctx);

/* Message of the last failing call on this context (host string, owned by the
 * context, valid until the next call).  ctx may be NULL: then the message of the
 * last failing abs_create on this thread. */
const char* abs_last_error(const abs_ctx* ctx);

/* Optional tuning of the statistics kernels; 0 restores the automatic
 * choice.  key: "stats_stages" (2..8 tile buffers), "stats_ctas_per_worker",
 * "stats_force_generic" (1 = always use the alignment-free kernel),
 * "stats_flush_every" (tiles between fp64 flushes of the per-row sums; for the
 * tcgen05 kernel: tiles added up in its fp32 accumulators before the fold into
 * fp64, at most 64),
 * "stats_stage_kb" (upper bound on one tile buffer, 4..200 KiB),
 * "stats_timeout_cycles" (SM clock cycles a wait for a tile copy may last before
 * the record is flagged ABS_STATUS_TIMEOUT; default about two seconds),
 * "stats_fault_drop_loads" (fault injection for tests: the loaders of the tiled,
 * cluster and tcgen05 kernels issue no copies, abs_logreg_rounds_fused sends no
 * partial gradients and the tensor-core products of the MLP producer fill no
 * operand tile, so every wait runs out and the records come back flagged
 * ABS_STATUS_TIMEOUT; the Newton-Schulz products and the tensor-core attention kernels
 * load nothing and their results are NaN; nothing traps or hangs),
 * "attention_fault_stop_after" (fault injection for tests: in every other CTA of the
 * tensor-core attention kernels the loads stop after so many steps, so that waits run out
 * in the middle of a tile and in CTAs that depend on it; 0 = never),
 * "stats_cluster_rows" (target rows per CTA of the cluster kernel, 16..512),
 * "stats_no_cluster" (1 = do not split the rows of a batch over a thread-block
 * cluster when b > 256),
 * "mlp_no_tensor_cores" (1 = the matrix products of the MLP producer run on the
 * CUDA cores in fp32 with fp64 folding instead of on the tensor cores),
 * "stats_no_secondary" (1 = the cluster kernel leaves the SMs idle that its
 * clusters cannot occupy instead of giving them a second launch of two-CTA
 * clusters), "stats_secondary_pct" (the speed of an SM of that second launch in
 * per cent of an SM of the first, which sets its share of the columns; 0 = 95, or 80 for rows
 * more than 64 MB apart),
 * "stats_no_gram" (1 = do not use the tensor-core Gram kernels for bf16, b <= 256),
 * "stats_no_recheck" (1 = keep a Gram kernel's record even when its sums are
 * ill-conditioned, i.e. never recompute it with the tiled kernel),
 * "ns_pair_tiles" (tiles of the Newton-Schulz products with fp16 operands: 1 =
 * 128 x 128 on single CTAs, 2 = 256 x 256 on pairs of CTAs),
 * "ns_max_cluster" (8..16: matrices with a side up to 128 use no larger thread-block clusters, as on a
 * device that cannot hold them, and take the general path instead),
 * "stats_ctas_per_sm" (1: one CTA per SM, 64 KiB buffers, up to 16 rows per
 * thread; 2: two CTAs per SM, 32 KiB buffers, up to 8 rows per thread).
 * Unknown key or out-of-range value: ABS_ERR_INVALID_ARG. */
int abs_set_tuning(abs_ctx* ctx, const char* key, long long value);

typedef enum { ABS_F32 = 0, ABS_BF16 = 1 } abs_dtype;

/* One record per worker, written by abs_test_stats.  With rows g_1..g_b of one
 * worker, gbar = (1/b) sum_i g_i (Eq. batch_grad), N = ||gbar||^2,
 * c_i = <g_i, gbar>:                                                           */
typedef struct {
  double gbar_sq;     /* N                                                       */
  double var_norm;    /* 1/(b-1) sum_i ||g_i - gbar||^2          (Eq. def_var)   */
  double var_ip;      /* 1/(b-1) sum_i (c_i - mean_i c_i)^2      (Eq. def_var of c_i) */
  double var_orth;    /* 1/(b-1) sum_i ||o_i - mean o||^2, o_i = g_i - (c_i/N) gbar;
                         evaluated as var_norm - var_ip / N (equal by orthogonality);
                         equals var_norm when N == 0                              */
  double sum_sq;      /* sum_i ||g_i||^2 = (b-1) var_norm + b N                  */
  long long rows;     /* b                                                       */
  unsigned status;    /* ABS_STATUS_* bits                                       */
  unsigned recomputed;/* 1: the tensor-core Gram kernel's sums were too ill-conditioned
                         (rows dominated by a common vector) and the record comes
                         from a second, centred pass over G; else 0              */
} abs_stats;          /* 56 bytes */

/* Batch-size test statistics of M workers (Eq. def_var applied per worker,
 * Eq. approx_norm_local; Algorithm 1, variance step).
 *   G            [M][b][d] per-sample (or per-micro-batch) gradients, dtype fp32
 *                or bf16; element (m,i,j) at G[m*worker_stride + i*row_stride + j]
 *   M >= 1, b >= 2 (the variance divides by b-1), d >= 1,
 *   row_stride >= d, worker_stride >= (b-1)*row_stride + d (ignored if M == 1)
 *   gbar_out     optional [M][d] fp32 (contiguous, worker m at gbar_out + m*d):
 *                receives the batch gradients; may be NULL
 *   stats_out    [M] records
 * G is read exactly once from HBM when its base address and both strides are
 * multiples of 16 bytes and b <= 4096 (bf16 input with b <= 256 goes through
 * tensor-core Gram-matrix kernels, other input with b > 256 through a kernel
 * that splits the rows over a thread-block cluster, everything else through the
 * tiled kernel); otherwise an alignment-free kernel that reads it twice is used.
 * The result does not depend on which kernel ran beyond floating-point rounding.
 * Accumulation: fp32 within a tile (the Gram kernels: exact bf16 products added
 * in fp32 over at most 8192 columns), fp64 across tiles; the reduction order is
 * fixed, so repeated calls give bit-identical records.
 * The Gram kernels only see uncentred products, so their variance is a difference
 * of two sums of size sum_i ||g_i||^2: when b N exceeds a few tens (tcgen05) or a
 * few thousand (mma.sync) times (b-1) var_norm -- rows dominated by a common
 * vector -- or N exceeds about 2e5 sqrt(var_ip), the finalisation flags the
 * result on the device and the tiled kernel, which accumulates centred values,
 * recomputes it in a second pass (abs_stats.recomputed = 1).  The two guarded
 * launches are always enqueued and return at once when not needed, so the call
 * stays free of host synchronisation.
 * Errors: ABS_ERR_INVALID_ARG, ABS_ERR_WORKSPACE, ABS_ERR_CUDA.               */
int abs_test_stats(abs_ctx* ctx, const void* G, abs_dtype dtype, int M, long long b, long long d,
                   long long row_stride, long long worker_stride,
                   float* gbar_out, abs_stats* stats_out, void* stream);

/* What abs_test_stats would launch for a shape: the host-side planning of the
 * statistics kernels, exposed for inspection and for tests that need no GPU.
 * aligned != 0 means base address and strides are multiples of 16 bytes.          */
typedef struct {
  int route;              /* 0 Gram (bf16, 7 <= b <= 32), 1 cluster, 2 tiled, 3 generic two-sweep,
                             4 Gram on tcgen05 (bf16, 32 < b <= 256)                          */
  int lanes_per_row;      /* 16-byte vectors per tile row: a tile row has 16*lanes_per_row bytes */
  int warps_per_box;      /* consumer warps that share one box of rows                        */
  int boxes_per_stage;
  int stages;             /* tile buffers in the ring                                         */
  int box_rows;           /* rows of one TMA box (<= 256)                                     */
  int row_boxes;          /* boxes stacked to cover the rows of a tile                        */
  int rows_per_thread;
  int keep_in_registers;  /* the tile stays in registers between the two sweeps               */
  int full;               /* every thread owns exactly rows_per_thread rows                   */
  int cluster_size;       /* CTAs per cluster (1 outside the cluster route)                   */
  int rows_per_cta;
  unsigned stage_bytes;
  unsigned reserved;
  size_t smem_bytes;      /* dynamic shared memory per CTA                                    */
} abs_stats_plan;
int abs_plan_stats(abs_dtype dtype, long long b, int aligned, int sm_count, size_t smem_optin,
                   abs_stats_plan* out);

/* Same computation for HOST buffers: G_host is copied to a device buffer owned
 * by the context (grown on demand), the statistics are computed and copied back
 * to stats_host [M] and, if not NULL, gbar_host [M][d]; the call returns after
 * everything has completed.  G_host is contiguous ([M][b][d], row_stride = d).
 * Pinned host memory makes the copies faster but is not required.
 * stats_dev / gbar_dev are optional DEVICE buffers ([M] records, [M][d] fp32) that
 * receive the same results on the device, for a following abs_next_batch /
 * local_*_step that should not wait for another host-to-device copy.            */
int abs_test_stats_host(abs_ctx* ctx, const void* G_host, abs_dtype dtype, int M, long long b,
                        long long d, float* gbar_host, abs_stats* stats_host,
                        float* gbar_dev, abs_stats* stats_dev, void* stream);

/* Statistics without any allocation.  (The paper has no counterpart: this entry
 * point exists for the sake of the calling program, not of the method.)
 *
 * abs_create allocates a device workspace, and cudaMalloc / cudaFree synchronise the
 * device.  Some callers cannot accept that: programs whose device memory is handed
 * out entirely by their own pool, plug-ins that run under a fixed memory budget,
 * latency-critical sections that must not hit an implicit device synchronisation.
 * For them this call computes the same statistics as abs_test_stats (the same
 * records up to floating-point rounding: it only uses the tiled kernel and the
 * alignment-free kernel, so bf16 input with b <= 256 and any input with b > 256
 * take another, slower kernel than in the context call), takes no
 * context, and keeps its scratch (per-CTA partial sums and a status word) in a
 * fixed array of ABS_NOALLOC_SCRATCH_BYTES + 256 bytes that is part of the library
 * image: every GPU on which the library is loaded holds that array until the
 * process exits, used or not.
 *   - Arguments and results as for abs_test_stats; the device used is the CURRENT
 *     CUDA device of the calling thread, and all pointers must belong to it.
 *   - Limits: b <= ABS_NOALLOC_MAX_ROWS and M <= ABS_NOALLOC_MAX_WORKERS; larger
 *     problems are refused with ABS_ERR_UNSUPPORTED (message from
 *     abs_noalloc_last_error) and need abs_test_stats with a context.
 *   - The first call on each device looks up the device address of the array and a
 *     few device attributes (no allocation by this library; a CUDA runtime that
 *     loads modules lazily places the array on the GPU at this moment).  Make that
 *     first call during start-up, outside any stream capture.
 *   - All calls on one device share the one array.  It still holds the previous
 *     call's partial sums; the call clears what has to start at zero itself.  Two
 *     calls that can run on the GPU at the same time (different streams, different
 *     host threads) would overwrite each other's partial sums: issue them in one
 *     stream, or order them with events.
 *   - Calls no cudaMalloc, cudaFree or other allocating routine.                    */
#define ABS_NOALLOC_SCRATCH_BYTES (8u << 20)
#define ABS_NOALLOC_MAX_ROWS      2048
#define ABS_NOALLOC_MAX_WORKERS   64
int abs_test_stats_noalloc(const void* G, abs_dtype dtype, int M, long long b, long long d,
                           long long row_stride, long long worker_stride,
                           float* gbar_out, abs_stats* stats_out, void* stream);
/* Message of the last failing abs_test_stats_noalloc call on this thread. */
const char* abs_noalloc_last_error(void);

typedef enum {
  ABS_TEST_NORM = 0,               /* norm test on the rows of G (Eq. approx_norm_local)               */
  ABS_TEST_AUG_INNER_PRODUCT = 1,  /* augmented inner-product test on the rows of G                    */
  ABS_TEST_NORM_WORKERS = 2        /* Algorithm 2 ("actual implementation"): the norm test on the M
                                      workers' BATCH gradients (Eq. test_stat_actual).  For
                                      abs_next_batch it is the norm test (the caller sets row_weight =
                                      local batch size and divisor = M); the per-round drivers
                                      abs_logreg_round / abs_mlp_round form the statistics themselves
                                      from the batch gradients of the round's last local step          */
} abs_test_kind;

typedef struct {
  int kind;             /* abs_test_kind                                              */
  int reserved;         /* zero                                                       */
  double eta;           /* norm test constant (Eq. approx_norm)                       */
  double theta;         /* inner-product test constant                                */
  double nu;            /* orthogonality test constant                                */
  long long b_max;      /* maximum local batch size (cap), >= 1                       */
  double row_weight;    /* samples one row stands for: 1 for per-sample gradients, the
                           micro-batch size for micro-batch gradients, the local batch
                           size when rows are workers' batch gradients (Section 4.3)   */
  double divisor;       /* 1, or M for Eq. test_stat_actual / Algorithm 2              */
} abs_test_cfg;

/* Next local batch size (Eq. norm_test, Eq. test_stat, Algorithm 1: b <- max{T, b};
 * display below Eq. test_stat: maximum over workers).  Per worker m, in fp64,
 *   norm test        T^m = ceil( s/D * var_norm / (eta^2 N) )
 *   augmented ip     T^m = max( ceil( s/D * var_ip / (theta^2 N^2) ),
 *                               ceil( s/D * var_orth / (nu^2 N) ) )
 * with s = row_weight, D = divisor; 0/x counts as 0 (also 0/0), x/0 as +infinity;
 * ceilings saturate at 2^62; a record flagged NONFINITE or TIMEOUT gives T^m = 0.
 *   b_next = min( b_max, max( b_cur, max_m T^m ) ).
 *   stats   [M] device records;  cfg  HOST pointer (copied by value at the call)
 *   b_cur   device, 1 value;  T_out device [M] or NULL;  b_next device, 1 value
 *           (may alias b_cur).  M <= 1024.                                          */
int abs_next_batch(abs_ctx* ctx, const abs_stats* stats, int M, const abs_test_cfg* cfg,
                   const long long* b_cur, long long* T_out, long long* b_next, void* stream);

/* Per-worker next local batch sizes (Eq. test_stat before the practical maximum
 * over workers; Algorithm 1: b^m <- max{T^m, b^m}), with one norm-test constant
 * per worker (eta_m of Eq. approx_norm_local):
 *   b_next[m] = min( b_max, max( b_cur[m], T^m ) ),  T^m as in abs_next_batch.
 * eta_m: DEVICE array [M] of constants, or NULL to use cfg->eta for every worker
 * (ignored by the augmented inner-product test).  b_cur, b_next, T_out: device [M]
 * (b_next may alias b_cur; T_out may be NULL).  cfg is a HOST pointer.            */
int abs_next_batch_local(abs_ctx* ctx, const abs_stats* stats, int M, const abs_test_cfg* cfg,
                         const double* eta_m, const long long* b_cur, long long* T_out,
                         long long* b_next, void* stream);

/* Norm-test statistics of a batch that arrives in sub-batches (gradient
 * accumulation over micro-batches, Section 6): folds sub-batch b into the running
 * pair a.  Per worker m, with n = rows, S = (n-1) var_norm (Eq. def_var):
 *   mean_a <- (n_a mean_a + n_b mean_b) / (n_a + n_b)                  (in place)
 *   S      <- S_a + S_b + ||mean_a - mean_b||^2 n_a n_b / (n_a + n_b)
 * rec_a [M] receives rows, var_norm, gbar_sq = ||mean||^2, sum_sq and the status
 * bit ABS_STATUS_NORM_ONLY (var_ip / var_orth cannot be merged: they are set to 0
 * and abs_next_batch gives T = 0 for the augmented test on such a record).
 * mean_a, mean_b: [M][d] fp32 batch gradients as written by abs_test_stats
 * (gbar_out); rec_a, rec_b: the matching records.  All device pointers.           */
int abs_stats_merge(abs_ctx* ctx, float* mean_a, const float* mean_b, int M, long long d,
                    abs_stats* rec_a, const abs_stats* rec_b, void* stream);

/* Local SGD step for all replicas (Eq. local_sgd_alt): X[m] <- X[m] - lr * Gb[m],
 * m < M, in fp32.  X, Gb: [M][d] fp32 with replica m at + m*replica_stride
 * (>= d).  average_after != 0 fuses the model averaging of the round's last step:
 * every replica receives (1/M) sum_m (X[m] - lr*Gb[m]) at no extra memory traffic.
 * X is updated in place.                                                        */
int local_sgd_step(abs_ctx* ctx, float* X, const float* Gb, int M, long long d,
                   long long replica_stride, float lr, int average_after, void* stream);

typedef struct {
  float lr, beta1, beta2, eps, weight_decay;
  int reserved;       /* zero */
  long long step;     /* t >= 1, shared by all replicas, keeps counting across rounds */
} abs_adamw_cfg;

/* Local AdamW step for all replicas (inner optimiser of Section 4.2 / Appendix
 * C.2; rule of the cited optimiser, decoupled weight decay):
 *   m <- beta1 m + (1-beta1) g ;  v <- beta2 v + (1-beta2) g^2
 *   x <- x (1 - lr wd) - lr (m / (1-beta1^t)) / ( sqrt(v / (1-beta2^t)) + eps )
 * X, Mom1, Mom2, Gb: [M][d] fp32, same replica_stride; all but Gb updated in place.
 * average_after != 0: X[m] <- mean over replicas of the updated X; the moments
 * stay local.  cfg is a HOST pointer.                                           */
int local_adamw_step(abs_ctx* ctx, float* X, float* Mom1, float* Mom2, const float* Gb, int M,
                     long long d, long long replica_stride, const abs_adamw_cfg* cfg,
                     int average_after, void* stream);

/* Local stochastic-heavy-ball (momentum SGD) step, the inner optimiser of the
 * paper's image experiments (Section 6.1):
 *   g <- g + wd x ;  u <- momentum u + g ;  x <- x - lr u
 * X, Buf (the momentum buffer u), Gb: [M][d] fp32.                              */
int local_shb_step(abs_ctx* ctx, float* X, float* Buf, const float* Gb, int M, long long d,
                   long long replica_stride, float lr, float momentum, float weight_decay,
                   int average_after, void* stream);

/* ---- orthogonalisation and the Muon step ---------------------------------------------------
 * Newton-Schulz iteration towards the orthogonal polar factor of a matrix: from
 *   X_0 = G / ( ||G||_F + eps )
 * each step applies, with A = X X' (X' X for a matrix taller than wide),
 *   X <- a X + (b A + c A^2) X,
 * i.e. p(s) = a s + b s^3 + c s^5 to every singular value.  (3.4445, -4.7750, 2.0315)
 * with 5 steps is the choice users of Muon make; (1.5, -0.5, 0) is the classical cubic.  */
typedef enum {
  ABS_NS_F16 = 0,       /* operands of the products rounded to 11 bits (fp16), X carried with 22 bits:
                           result within about 2e-3 (normwise) of the exact iteration; a Muon step's
                           parameters are off by that times the step's share of them                    */
  ABS_NS_F32 = 1        /* operands of 22 bits, three products each: fp32-grade (0.8e-6 to 1.8e-6 of the norm
                           on full-rank matrices where plain fp32 products have 0.8e-6 to 2.4e-6)       */
} abs_ns_precision;

typedef struct {
  float a, b, c;        /* finite; ABS_ERR_UNSUPPORTED if they let singular values pass 1024            */
  float eps;            /* >= 0; a zero matrix gives a zero result for eps > 0, NaN for eps = 0          */
  int steps;            /* 1..32                                                                         */
  int precision;        /* abs_ns_precision                                                              */
} abs_ns_cfg;           /* 24 bytes */

/* Bytes of device scratch for abs_orthogonalise (count matrices) or local_muon_step (count = M *
 * matrices).  Matrices are worked on in groups, so past about 200 MB (or one matrix, if that is more) it stops
 * growing with their number; there it also falls, as groups are of equal size.  Both calls take less than this, down to
 * what one matrix needs, in smaller groups (more launches): scratch for some number of matrices serves every
 * smaller one.  cfg is a HOST pointer; needs no context.                                           */
int abs_ns_scratch_bytes(int count, long long rows, long long cols, const abs_ns_cfg* cfg, size_t* out);

/* O[q] = the iterate after cfg->steps steps from G[q], q < count.  Element (q, r, c) of G at
 * G[q*g_matrix_stride + r*g_row_stride + c], row strides >= cols, matrices disjoint (strides of
 * count == 1 are ignored).  fp32 or bf16 in and out.  O may be G (same type and strides).
 * rows, cols <= 65536.  A non-finite entry makes its matrix NaN, no other.  If a wait inside a
 * product runs out (the "stats_timeout_cycles" key), the results are NaN.                         */
int abs_orthogonalise(abs_ctx* ctx, const void* G, abs_dtype g_dtype, int count, long long rows, long long cols,
                      long long g_row_stride, long long g_matrix_stride, void* O, abs_dtype o_dtype,
                      long long o_row_stride, long long o_matrix_stride, const abs_ns_cfg* cfg, void* scratch,
                      size_t scratch_bytes, void* stream);

typedef struct {
  float lr, momentum, weight_decay;
  float scale;          /* factor on the orthogonalised update: sqrt(max(1, rows/cols)), or
                           0.2 sqrt(max(rows, cols)) to match the update size of AdamW                  */
  int nesterov;
  int reserved;         /* zero */
  abs_ns_cfg ns;
} abs_muon_cfg;         /* 48 bytes */

/* Local Muon step for all replicas of `matrices` equal-shaped parameter matrices:
 *   u <- momentum u + g ;  v = nesterov ? g + momentum u : u
 *   x <- x (1 - lr wd) - lr scale O(v),  O as in abs_orthogonalise, matrix by matrix
 * Matrix l of replica m is [rows][cols], contiguous, at + m*replica_stride + l*matrix_stride in X,
 * Buf (the momentum u) and Gb, all fp32 (so the matrices may lie inside flat parameter vectors).
 * average_after != 0: X[m] <- mean over replicas of the updated X; the momentum stays local.
 * cfg is a HOST pointer.  The result of a step whose products ran out of time is NaN.            */
int local_muon_step(abs_ctx* ctx, float* X, float* Buf, const float* Gb, int M, int matrices, long long rows,
                    long long cols, long long matrix_stride, long long replica_stride, const abs_muon_cfg* cfg,
                    int average_after, void* scratch, size_t scratch_bytes, void* stream);

/* Model averaging (Eq. local_sgd_alt, second line; Algorithm 1 "update the
 * global model"): every replica receives (1/M) sum_m X[m], in place.            */
int replica_average(abs_ctx* ctx, float* X, int M, long long d, long long replica_stride,
                    void* stream);

/* ---- the outer loop: sample counter, stop rule, cadence of the test ---------------------- */

/* The counters of Algorithm 1 / Algorithm 2, kept on the DEVICE so that rounds can follow one
 * another without a host read-back: B (samples processed), k (rounds completed) and the N of
 * "while B < N".  The caller allocates it in device memory, initialises it and may copy it back
 * at any time.  The drivers add, per round, sum_m sum_h b^m_{k,h} (Algorithm 1) -- which is
 * H M b_k when the size is shared and constant over a round (Algorithm 2) -- and 1 to k.
 * abs_logreg_rounds_fused_opts also obeys the stop rule on the device: it runs no round once
 * samples >= n_stop (n_stop <= 0: no stop).  The enqueue-only per-round drivers cannot skip
 * launches that are already enqueued; their caller reads the block back with the batch size. */
typedef struct {
  long long samples;    /* B                                                          */
  long long rounds;     /* k                                                          */
  long long n_stop;     /* N; <= 0: never stop                                        */
  long long reserved;   /* zero                                                       */
} abs_round_ctl;

/* Cadence and ownership of the batch size (HOST struct, copied at the call).         */
typedef struct {
  int test_every_step;  /* 0: the test once per round, on the last local step's gradients
                           (Section 4.3, last paragraph); 1: after every local step, the
                           next step already using the new size (Algorithm 1)          */
  int per_worker;       /* 1: b^m <- max{T^m, b^m} per worker (Eq. test_stat, Algorithm 1);
                           0: every worker continues with the maximum over the workers
                           (display below Eq. test_stat)                               */
  const double* eta_m;  /* DEVICE [M] norm-test constants eta_m (Eq. approx_norm_local), or
                           NULL: cfg->eta for every worker                             */
  abs_round_ctl* ctl;   /* DEVICE counter block, or NULL                               */
} abs_round_opts;

/* samples += times * (sizes[0] + ... + sizes[n-1]);  rounds += add_rounds  -- one tiny launch.
 * ctl, sizes: device.                                                                */
int abs_round_count(abs_ctx* ctx, abs_round_ctl* ctl, const long long* sizes, int n, long long times,
                    long long add_rounds, void* stream);

/* ---- producers and round drivers for the synthetic end-to-end problems ------------------ */

/* Per-sample gradients of the logistic loss (Algorithm 1, per-sample gradient
 * step): row i of worker m is (sigmoid(a^T x^m) - y) a with a = A[idx[m][i]].
 *   A [n][d] fp32 features, y [n] fp32 labels in {0,1}, idx [M][idx_stride] int32
 *   sample indices (the first b of each row are used), X [M][d] parameters,
 *   G [M][b][d] output (contiguous).                                              */
int abs_logreg_grads(abs_ctx* ctx, const float* A, const float* y, long long n, long long d,
                     const int* idx, long long idx_stride, const float* X, int M, long long b,
                     float* G, void* stream);

/* One communication round of local SGD on the logistic problem (Algorithm 2's
 * structure, Algorithm 1's per-sample statistic evaluated once per round, Section
 * 4.3): for h < H: per-sample gradients of batch idx[h] -> statistics and batch
 * gradient -> local SGD step (the last one fused with the model averaging); then
 * the batch-size update from the statistics of the last local step.
 *   idx [H][M][idx_stride] int32;  b the current batch size (host value, equal to
 *   *b_dev);  G_scratch [M][b][d], Gb_scratch [M][d], stats [M], T_out [M] or NULL;
 *   b_dev device int64: holds b on entry and the next batch size afterwards.
 *   ctl device counter block or NULL: B += H M b (Algorithm 2's counter), k += 1.
 * cfg->kind == ABS_TEST_NORM_WORKERS runs Algorithm 2 as printed: no per-sample test; after
 * the averaging the M batch gradients of the last local step (rows of Gb_scratch) give
 * Var = b/(M-1) sum_m ||g^m - gbar||^2 and T = ceil(Var / (M eta^2 ||gbar||^2)); needs M >= 2;
 * stats[0] receives that record (rows = M), T_out[0] the T, the other entries are unspecified.
 * Only enqueues; read b_dev (and ctl) back before sizing the next round.          */
int abs_logreg_round(abs_ctx* ctx, const float* A, const float* y, long long n, long long d,
                     const int* idx, long long idx_stride, float* X, int M, int H, long long b,
                     float lr, const abs_test_cfg* cfg, float* G_scratch, float* Gb_scratch,
                     abs_stats* stats, long long* T_out, long long* b_dev, abs_round_ctl* ctl,
                     void* stream);

/* The same round with the test after every local step (Algorithm 1 as printed): at step h
 * worker m draws b^m_{k,h} samples, its statistics give T^m_{k,h}, and step h + 1 runs with
 * b^m_{k,h+1} = min(b_max, max{T^m, b^m}) -- per worker, or the maximum over the workers
 * for all of them (opts->per_worker).  opts may be NULL (shared size, cfg->eta, no counter).
 *   b_host  HOST array [M]: the sizes the round starts with; on return the sizes after it
 *   b_dev   device [M] scratch that holds the same values
 *   idx [H][M][idx_stride] with idx_stride >= cfg->b_max;  G_scratch room for M * b_max rows
 *   of d floats;  stats [H][M] and T_out [H][M] (or NULL): the records and T of every step.
 * The grids of step h + 1 depend on sizes decided on the device in step h, so this call
 * WAITS for the stream once per local step to read M integers back (the one driver of the
 * library that synchronises; abs_logreg_rounds_fused_opts does the same work without).   */
int abs_logreg_round_per_step(abs_ctx* ctx, const float* A, const float* y, long long n, long long d,
                              const int* idx, long long idx_stride, float* X, int M, int H,
                              long long* b_host, float lr, const abs_test_cfg* cfg,
                              const abs_round_opts* opts, float* G_scratch, float* Gb_scratch,
                              abs_stats* stats, long long* T_out, long long* b_dev, void* stream);

/* `rounds` communication rounds of the same method in ONE cooperative launch
 * (Algorithm 2's structure, Algorithm 1's per-sample statistic once per round,
 * Section 4.3; b <- min(b_max, max{b, max_m T_m})): the parameters stay in shared
 * memory, the batch size stays on the device from round to round, the per-sample
 * gradient matrix is never written, and there is one grid-wide barrier per round
 * (none inside a local step).  For small problems, where abs_logreg_round is bound by launch latency.
 *   idx [rounds][H][M][idx_stride] int32 with idx_stride >= cfg->b_max (indices
 *   outside [0, n) are clamped);  X [M][d] in place (replica stride d);
 *   stats [rounds][M] records of each round's test;  T_out [rounds][M] or NULL;
 *   b_hist [rounds + 1] or NULL: the batch size each round ran with, then the last
 *   update;  b_dev: the starting size on entry (raised to 2, capped at b_max), the
 *   size after the last round on exit.
 * Needs d <= 1024, d % 4 == 0, M <= 64 and 16-byte aligned A and X, else
 * ABS_ERR_UNSUPPORTED; scratch comes from the context's workspace
 * (ABS_ERR_WORKSPACE if it is too small).  Each worker is one thread-block cluster
 * and the launch is cooperative (all CTAs resident); ABS_ERR_UNSUPPORTED if the
 * device cannot hold M clusters at once, ABS_ERR_CUDA if it refuses the launch.
 * The CTAs of a cluster wait for one another's partial gradients with the limit of
 * the "stats_timeout_cycles" tuning key; a wait that runs out never hangs the
 * launch: the records of that round and of the following ones carry
 * ABS_STATUS_TIMEOUT, which gives T = 0, and the parameters are then not to be
 * used.  Only enqueues.                                                            */
int abs_logreg_rounds_fused(abs_ctx* ctx, const float* A, const float* y, long long n, long long d,
                            const int* idx, long long idx_stride, int rounds, float* X, int M, int H,
                            float lr, const abs_test_cfg* cfg, abs_stats* stats, long long* T_out,
                            long long* b_hist, long long* b_dev, void* stream);

/* The same launch with the cadence, the ownership of the batch size, per-worker constants
 * and the counters of Algorithm 1 / Algorithm 2 chosen by `opts` (HOST pointer; NULL gives
 * abs_logreg_rounds_fused).  With opts:
 *   b_dev   device [M]: every worker's size on entry and after the last round that ran
 *   test once per round:   stats, T_out [rounds][M];  b_hist [rounds][M] (or NULL): the size
 *                          each round ran with
 *   test_every_step:       stats, T_out, b_hist [rounds][H][M]: record, T and the size of
 *                          every local step (Algorithm 1); one cluster-wide barrier per step
 *                          more, and a grid-wide one per step when the size is shared
 *   cfg->kind == ABS_TEST_NORM_WORKERS (with or without opts; not with test_every_step or
 *                          per_worker; M >= 2): Algorithm 2 as printed -- no per-sample
 *                          statistics, the norm test on the M batch gradients of the round's
 *                          last local step after the averaging; per round stats[.][0] holds that
 *                          record (rows = M, flagged ABS_STATUS_NORM_ONLY) and T_out[.][0] the T
 *   opts->ctl              B and k are read at the start and written back at the end; no
 *                          round starts once B >= n_stop (entries of rounds that did not
 *                          run are left untouched); X holds x_{K,0} of the last round run.  */
int abs_logreg_rounds_fused_opts(abs_ctx* ctx, const float* A, const float* y, long long n, long long d,
                                 const int* idx, long long idx_stride, int rounds, float* X, int M,
                                 int H, float lr, const abs_test_cfg* cfg, const abs_round_opts* opts,
                                 abs_stats* stats, long long* T_out, long long* b_hist,
                                 long long* b_dev, void* stream);

/* ---- layer norm ---------------------------------------------------------------------------
 * Rows of d features, fp32 or bf16, for M replicas with parameters of their own (fp32):
 *   mean = (1/d) sum_j x_j,  rstd = 1 / sqrt( (1/d) sum_j (x_j - mean)^2 + eps ),
 *   y_j = (x_j - mean) rstd weight_j + bias_j
 *   X, Y        row r of replica m at + m*worker_stride + r*row_stride (>= d; replicas disjoint;
 *               the worker strides are ignored for M == 1).  Y may be X (same strides).
 *   weight, bias  replica m at + m*param_stride (0: all replicas share them), or NULL (ones / zeros)
 *   mean, rstd  [M][rows] fp32 for the backward pass, or NULL
 *   rows may be 0.  Statistics are fp32 from values held in registers or read twice: the
 *   variance is that of centred values, and y is rounded once.                              */
int abs_layer_norm(abs_ctx* ctx, const void* X, abs_dtype dtype, int M, long long rows, long long d,
                   long long x_row_stride, long long x_worker_stride, const float* weight, const float* bias,
                   long long param_stride, float eps, void* Y, long long y_row_stride, long long y_worker_stride,
                   float* mean, float* rstd, void* stream);

/* Its backward pass.  A replica's rows are `samples` samples of `tokens` consecutive rows.  With
 * xh = (x - mean) rstd and a = weight dy:
 *   dx = rstd ( a - (1/d) sum_j a_j - xh (1/d) sum_j a_j xh_j )
 *   per-sample gradients (Algorithm 1, per-sample gradient step), sums over the sample's rows:
 *     Gw[i] = sum_t dy xh,  Gb[i] = sum_t dy     at + m*g_worker_stride + i*g_row_stride
 *   and their sums over the samples, dW, dB, at + m*grad_stride.
 * dX, dW, dB, Gw, Gb may each be NULL.  Gw and Gb may be two parts of one row, as abs_test_stats
 * takes them.  dX may be dY or X (same strides).  samples and tokens may be 0 (sums of nothing
 * are zero).  mean, rstd: [M][samples*tokens] as the forward pass wrote them.  All sums are fp32
 * in a fixed order: repeated calls give the same bits.
 * ABS_ERR_WORKSPACE if the context's workspace cannot hold two partial sums of 2d floats (one
 * per replica, or per sample where only one of Gw and Gb is given, and one more); past 2^30 rows
 * of all replicas twice (or one more) for every 2^30.                                         */
int abs_layer_norm_backward(abs_ctx* ctx, const void* dY, long long dy_row_stride, long long dy_worker_stride,
                            const void* X, long long x_row_stride, long long x_worker_stride, abs_dtype dtype, int M,
                            long long samples, long long tokens, long long d, const float* mean, const float* rstd,
                            const float* weight, long long param_stride, void* dX, long long dx_row_stride,
                            long long dx_worker_stride, float* dW, float* dB, long long grad_stride, float* Gw,
                            float* Gb, long long g_row_stride, long long g_worker_stride, void* stream);

/* How abs_layer_norm_backward would share out its rows and its workspace for a shape: the host-side
 * planning, exposed for inspection and for tests that need no GPU.  aligned != 0 means base addresses and
 * strides are multiples of 16 bytes (else of one element).  The M*samples segments of `tokens` rows (without
 * Gw and Gb: one a replica) lie one after the other; CTA c has rows c*rows_per_cta and on.  Its sums of
 * segment s go to the workspace's place c + s, or, direct: to Gw and Gb themselves where the CTA has the whole
 * segment, else to place 2c (its first) or 2c + 1.  M*parts places from `used` on follow where parts > 1 and
 * the totals are asked for.  ABS_ERR_WORKSPACE: room < needed, and ctas to used are not set.              */
typedef struct {
  int route;              /* 0 rows staged in shared memory, 1 rows in registers, 2 any width          */
  int groups;             /* groups of threads of a CTA, each with rows of its own                     */
  long long samples;      /* segments of a replica                                                     */
  long long tokens;       /* rows of a segment                                                         */
  long long ctas;
  long long rows_per_cta;
  int direct;
  int parts;              /* CTAs that add up a column's segments                                      */
  long long room;         /* places of 2d floats in the workspace                                      */
  long long needed;
  long long used;
} abs_ln_backward_plan;   /* 72 bytes */
int abs_plan_layer_norm_backward(abs_dtype dtype, int M, long long samples, long long tokens, long long d, int aligned,
                                 int with_gw, int with_gb, int with_totals, int sm_count, size_t workspace_bytes,
                                 abs_ln_backward_plan* out);

/* ---- root-mean-square norm -----------------------------------------------------------------
 * Rows of d features, fp32 or bf16, for M replicas with a weight of their own (fp32):
 *   h_j = x_j + r_j (rounded to the type once; h = x without R),
 *   rstd = 1 / sqrt( (1/d) sum_j h_j^2 + eps ),   y_j = h_j rstd weight_j
 *   X, R, H, Y  row r of replica m at + m*worker_stride + r*row_stride (>= d; replicas disjoint; the
 *               worker strides are ignored for M == 1).  R (the residual stream) and H (its new
 *               value) are NULL or of X's type.  H may be R or X, Y may be X (same strides each).
 *   Q, scales   NULL, or the rows in 8 bits (e4m3, one byte an element, strides in bytes) and
 *               [M][rows] fp32: scales = max_j |y_j| / 448 (1 for a row of zeros, for any other no
 *               less than 2^-149), Q = y / scales rounded to nearest, at most 448 in magnitude (a
 *               subnormal scale is a whole number of steps of 2^-149 and may be too small for its
 *               row).  y is the value before its rounding to Y's type.  Y may be NULL then.  A row
 *               with a NaN or an infinity among its y gives NaN scales and NaN in Q.
 *   weight      replica m at + m*param_stride (0: all replicas share it), or NULL (ones)
 *   rstd        [M][rows] fp32 for the backward pass, or NULL
 *   rows may be 0.  Sums and y are fp32; y is rounded once.  A row of zeros with eps = 0 is 0 / 0: NaN. */
int abs_rms_norm(abs_ctx* ctx, const void* X, abs_dtype dtype, int M, long long rows, long long d,
                 long long x_row_stride, long long x_worker_stride, const void* R, long long r_row_stride,
                 long long r_worker_stride, void* H, long long h_row_stride, long long h_worker_stride,
                 const float* weight, long long param_stride, float eps, void* Y, long long y_row_stride,
                 long long y_worker_stride, void* Q, long long q_row_stride, long long q_worker_stride, float* scales,
                 float* rstd, void* stream);

/* Its backward pass.  A replica's rows are `samples` samples of `tokens` consecutive rows.  With
 * xh = h rstd and a = weight dy:
 *   dx = dh + rstd ( a - xh (1/d) sum_j a_j xh_j )      (the gradient of X and of R alike)
 *   per-sample gradients:  Gw[i] = sum_t dy xh          at + m*g_worker_stride + i*g_row_stride
 *   and their sum over the samples, dW, at + m*grad_stride.
 * dH: the gradient that reaches the residual stream behind the norm, or NULL (zero).  dX, dW and Gw may each
 * be NULL.  dX may be dY, H or dH (same strides).  samples and tokens may be 0 (sums of nothing are
 * zero).  H: what was normalised; rstd as the forward pass wrote it.  All sums are fp32 in a fixed order:
 * repeated calls give the same bits.  Uses the context's workspace as far as it goes.              */
int abs_rms_norm_backward(abs_ctx* ctx, const void* dY, long long dy_row_stride, long long dy_worker_stride,
                          const void* H, long long h_row_stride, long long h_worker_stride, const void* dH,
                          long long dh_row_stride, long long dh_worker_stride, abs_dtype dtype, int M, long long samples,
                          long long tokens, long long d, const float* rstd, const float* weight,
                          long long param_stride, void* dX, long long dx_row_stride, long long dx_worker_stride,
                          float* dW, long long grad_stride, float* Gw, long long g_row_stride,
                          long long g_worker_stride, void* stream);

/* ---- attention -------------------------------------------------------------------------------
 * Causal attention with grouped heads over packed sequences, fp32 or bf16.  The tokens of all sequences (of all
 * replicas, where there are several) are rows of one tensor, total of them; sequence i has the rows offsets[i] to
 * offsets[i+1] - 1.  Row t of a sequence sees the rows of that sequence up to its own; query head h reads the
 * keys and values of head h / (q_heads / kv_heads):
 *   s_tj = scale <q_t, k_j>,  lse_t = log sum_j exp(s_tj),  o_t = sum_j exp(s_tj - lse_t) v_j
 * Rows outside all sequences (in front of the first, behind the last) are neither computed nor written, and nothing in
 * them reaches a result; neither do the rows of one sequence reach another's.  Inside a sequence an infinity or a NaN in V
 * (backward: in Q, K, V, dO) may reach earlier rows than its own.
 * Sequences may be empty.  head_dim <= 128.
 *
 * A tensor is a HOST struct: token t, head h at data + t*row_stride + h*head_stride, head_dim contiguous elements, no two
 * of these overlapping.  Views of a fused [total][(q_heads + 2 kv_heads) head_dim] tensor are such tensors.
 * bf16 runs on the tensor cores where every tensor's base and strides are multiples of 16 bytes, head_dim is one of 8
 * elements and (forward) scale > 0; other calls and fp32 run on the CUDA cores, 17 to 20 times slower.  The tensor cores' products
 * are 64 or 128 columns wide, whatever head_dim is.
 *
 * Precision: sums, lse and exponents are fp32.  The tensor-core kernels round the weights exp(s_tj - lse_t), and backward the ds
 * too, to bf16 as operands of their products with V, dO, Q and K: against 64 bits o is off by 2.0e-3 and the gradients are by
 * 2.4e-3 (relative 2-norm), where rounding the results alone would give 1.6e-3 and 1.7e-3.  On the CUDA cores only results are rounded.
 * A weight is also off by a few 2^-24 |s_tj|, the rounding of its exponent: scores of 2^20 and more have no meaningful weights, and of
 * 2^28 and more the results may be anything.                                                       */
typedef struct {
  void* data;
  long long row_stride;
  long long head_stride;
} abs_heads;   /* 24 bytes */

/* The plan of a batch: the tiles of its sequences in the order in which they are worked off.  Made once a batch, read by
 * the calls of every layer.  offsets: DEVICE int32 [sequences + 1]; values outside [0, total] are clamped and one
 * below its predecessor is raised to it, which sets the plan's third int32 to 1 (else 0).  plan: device memory of
 * abs_attention_plan_bytes, 16-byte aligned.  A plan for other offsets of as many sequences and the same total may be written over it, also
 * between replays of a graph that captured the calls that read it.
 * A call with a plan of another number of sequences or another total gives NaN in all rows of its outputs.
 * sequences <= 2^24, total <= 2^30.                                                                  */
int abs_attention_plan_bytes(int sequences, long long total, size_t* out);
int abs_attention_plan(abs_ctx* ctx, const int* offsets, int sequences, long long total, void* plan, size_t plan_bytes,
                       void* stream);

/* lse: fp32 [q_heads][total], or NULL.  O overlaps no input.  |scale| < 2e38.  q_heads <= 4096, total * q_heads <= 2^32 and
 * sequences * q_heads <= 2^28.  The tensor-core kernels' waits are bounded ("stats_timeout_cycles"): rows whose tile a wait
 * that ran out left unfinished are NaN.                                                              */
int abs_attention(abs_ctx* ctx, const abs_heads* Q, const abs_heads* K, const abs_heads* V, abs_dtype dtype, const void* plan,
                  int sequences, long long total, int q_heads, int kv_heads, int head_dim, float scale, const abs_heads* O,
                  float* lse, void* stream);

/* Its backward pass.  O, lse: as the forward pass wrote them.  With p_tj = exp(s_tj - lse_t):
 *   ds_tj = p_tj (<do_t, v_j> - <do_t, o_t>)
 *   dv_j = sum_t p_tj do_t,   dk_j = scale sum_t ds_tj q_t,   dq_t = scale sum_j ds_tj k_j
 * with the sums over t of dk and dv running over all query heads of the group.  Sums are fp32 in a fixed order:
 * repeated calls give the same bits.  The outputs overlap no input and not one another.
 * scratch: device memory of abs_attention_scratch_bytes, 256-byte aligned; calls that may overlap have scratch of their own.  */
int abs_attention_scratch_bytes(long long total, int q_heads, int kv_heads, int head_dim, int sequences, size_t* out);
int abs_attention_backward(abs_ctx* ctx, const abs_heads* dO, const abs_heads* Q, const abs_heads* K, const abs_heads* V,
                           const abs_heads* O, const float* lse, abs_dtype dtype, const void* plan, int sequences,
                           long long total, int q_heads, int kv_heads, int head_dim, float scale, const abs_heads* dQ,
                           const abs_heads* dK, const abs_heads* dV, void* scratch, size_t scratch_bytes, void* stream);

/* ---- token embedding -------------------------------------------------------------------------
 * y_t = scale E[token_t], rounded once to Y's type (fp32 or bf16).
 *   E       [M] fp32 tables of vocab rows of d: row v of replica m at + m*e_worker_stride + v*e_row_stride
 *           (>= d).  e_worker_stride 0: all replicas share one table.
 *   tokens  int32, token t of replica m at + m*tokens_stride + t (0: all replicas share them).  A token outside
 *           [0, vocab) gives a row of zeros and no gradient.
 *   Y       row t of replica m at + m*y_worker_stride + t*y_row_stride
 * Worker strides are ignored for M == 1.  rows may be 0.                                            */
int abs_embedding(abs_ctx* ctx, const float* E, int M, long long vocab, long long d, long long e_row_stride,
                  long long e_worker_stride, const int* tokens, long long tokens_stride, long long rows, float scale, void* Y,
                  abs_dtype y_dtype, long long y_row_stride, long long y_worker_stride, void* stream);

/* Its backward pass: dE[v] = scale sum_{t: token_t = v} dy_t for every row v of every replica's table, zeros for
 * tokens that do not occur; accumulate != 0: added to what dE holds (rows of other tokens are not touched).
 * The tokens are sorted on the way; sums are fp32 in a fixed order: repeated calls give the same bits.
 * dE: fp32, replica m at + m*e_worker_stride (replicas disjoint).  scratch: device memory of
 * abs_embedding_scratch_bytes, 256-byte aligned; calls that may overlap have scratch of their own.
 * vocab < 2^24, d <= 2^24, rows <= 2^28, M <= 65535, M * rows <= 2^31, M * vocab <= 2^36 (of the forward pass too).  */
int abs_embedding_scratch_bytes(int M, long long rows, long long vocab, long long d, size_t* out);
int abs_embedding_backward(abs_ctx* ctx, const void* dY, abs_dtype dtype, int M, long long rows, long long d,
                           long long dy_row_stride, long long dy_worker_stride, const int* tokens, long long tokens_stride,
                           long long vocab, float scale, float* dE, long long e_row_stride, long long e_worker_stride,
                           int accumulate, void* scratch, size_t scratch_bytes, void* stream);

/* Three-layer ReLU MLP with softmax cross-entropy (the second synthetic problem).
 * dims = {n0, n1, n2, n3} layer widths.  One replica's parameters are a flat fp32
 * vector W1 [n1][n0], b1 [n1], W2 [n2][n1], b2 [n2], W3 [n3][n2], b3 [n3] (each W
 * row-major [out][in]); abs_mlp_param_count gives its length d.                    */
int abs_mlp_param_count(const int* dims, long long* out);
/* Bytes of scratch abs_mlp_grads needs for M workers and batch size b. */
int abs_mlp_scratch_bytes(int M, long long b, const int* dims, size_t* out);

/* Forward and backward pass of all M workers on their batches (Algorithm 2,
 * local batch gradient step): writes the batch gradients Gb [M][d] and
 * leaves activations and deltas in `scratch` (device, caller-owned) for
 * abs_mlp_per_sample.  inputs [n][n0] fp32, labels [n] int32, idx [M][idx_stride]
 * int32 sample indices (first b used), X [M][d] parameters (replica stride d).     */
int abs_mlp_grads(abs_ctx* ctx, const float* inputs, const int* labels, long long n, const int* dims,
                  const int* idx, long long idx_stride, const float* X, int M, long long b,
                  float* Gb, void* scratch, size_t scratch_bytes, void* stream);

/* Per-sample gradients of one worker as rows G [b][row_stride] (row_stride >= d; a
 * multiple of 4 keeps the rows 16-byte aligned for the fast statistics kernels),
 * from the scratch a preceding abs_mlp_grads call with the same b filled
 * (Algorithm 1, per-sample gradient step).  b <= 65535.                       */
int abs_mlp_per_sample(abs_ctx* ctx, const int* dims, long long b, int worker, const void* scratch,
                       float* G, long long row_stride, void* stream);

/* The statistics of all M workers without forming the per-sample gradient matrix
 * (a per-sample gradient of a layer is the outer product delta_i (x) h_i, so
 * ||g_i||^2 = sum_l ||delta_l,i||^2 (||h_{l-1},i||^2 + 1) and
 * <g_i, gbar> = sum_l delta_l,i^T (dW_l h_{l-1},i + db_l); Eq. def_var expanded):
 * reads the activations and deltas a preceding abs_mlp_grads call with the same b
 * and M left in `scratch` and the batch gradients Gb [M][d] it wrote; writes
 * stats [M].  The expansion sum_i ||g_i||^2 - b N loses accuracy only when the
 * variance is far below b N, i.e. when the test is satisfied by a wide margin.      */
int abs_mlp_fused_stats(abs_ctx* ctx, const int* dims, long long b, int M, void* scratch,
                        size_t scratch_bytes, const float* Gb, abs_stats* stats, void* stream);

/* One communication round of local SGD on the MLP problem, as abs_logreg_round.  At
 * the last local step the statistics come either from per-sample gradients
 * materialised for one worker at a time in G_scratch [b][g_row_stride], or, when
 * G_scratch is NULL, from abs_mlp_fused_stats.  Gb_scratch [M][d].                  */
int abs_mlp_round(abs_ctx* ctx, const float* inputs, const int* labels, long long n, const int* dims,
                  const int* idx, long long idx_stride, float* X, int M, int H, long long b, float lr,
                  const abs_test_cfg* cfg, void* scratch, size_t scratch_bytes, float* G_scratch,
                  long long g_row_stride, float* Gb_scratch, abs_stats* stats, long long* T_out,
                  long long* b_dev, abs_round_ctl* ctl, void* stream);

/* The MLP round with the test after every local step, as abs_logreg_round_per_step; the
 * statistics of every step come from abs_mlp_fused_stats.  scratch must hold M workers at
 * b_max (abs_mlp_scratch_bytes).  Waits for the stream once per local step.              */
int abs_mlp_round_per_step(abs_ctx* ctx, const float* inputs, const int* labels, long long n,
                           const int* dims, const int* idx, long long idx_stride, float* X, int M,
                           int H, long long* b_host, float lr, const abs_test_cfg* cfg,
                           const abs_round_opts* opts, void* scratch, size_t scratch_bytes,
                           float* Gb_scratch, abs_stats* stats, long long* T_out, long long* b_dev,
                           void* stream);

#ifdef __cplusplus
}
#endif
#endif  /* ABS_H_ */
