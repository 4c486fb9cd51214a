// Causal attention over packed sequences: entry points, and the plan of a batch.
#include "abs_attention.cuh"

namespace absk {
namespace {

constexpr int kPlanThreads = 1024;

__device__ __forceinline__ int block_scan(int v, int* red, bool maximum) {      // inclusive, over the CTA
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v = maximum ? max(v, o) : v + o;
  }
  __syncthreads();                       // the previous use of red is over
  if (lane == 31) red[warp] = v;
  __syncthreads();
  if (warp == 0) {
    int w = red[lane];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, w, off);
      if (lane >= off) w = maximum ? max(w, o) : w + o;
    }
    red[lane] = w;
  }
  __syncthreads();
  if (warp > 0) v = maximum ? max(v, red[warp - 1]) : v + red[warp - 1];
  return v;
}

// The tiles of the sequences to `out`, ordered by their work: most first (forward: tile i reads the keys of i + 1 tiles) or
// least first (backward: tile j is read by the queries of the tiles from j on).  With sequences in the order of their lengths, those
// with at least w tiles come first, so a tile's place is (tiles in front by their work) + (its sequence's place).  Which of two
// sequences of one length comes first is left to chance; no result depends on it.  Returns the number of tiles.
// counts: [3][bins], sequences of exactly b tiles, of at least b, and the tiles in front of those of work b.
__device__ int order_tiles(const int* starts, int n, int rows, bool most_first, int* counts, int bins, int4* out, int cap, int* red) {
  const int tid = threadIdx.x;
  int longest = 0;
  for (int i = tid; i < n; i += kPlanThreads) longest = max(longest, (starts[i + 1] - starts[i] + rows - 1) / rows);
  block_scan(longest, red, true);
  __syncthreads();
  longest = red[31];
  const int used = longest + 2;                    // bins 0 to longest + 1, the last one empty
  int *exact = counts, *least = counts + bins, *before = least + bins;
  for (int b = tid; b < used; b += kPlanThreads) exact[b] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) atomicAdd(exact + (starts[i + 1] - starts[i] + rows - 1) / rows, 1);
  __syncthreads();
  int carry = 0;
  for (int at = 0; at < used; at += kPlanThreads) {
    const int b = used - 1 - (at + tid);
    const int v = carry + block_scan(b >= 0 ? exact[b] : 0, red, false);
    if (b >= 0) least[b] = v;
    __syncthreads();
    carry += red[31];
  }
  __syncthreads();
  carry = 0;
  for (int at = 0; at < used; at += kPlanThreads) {
    const int i = at + tid, b = most_first ? used - 1 - i : i;
    const int own = b >= 1 && b < used ? least[b] : 0;
    const int v = carry + block_scan(own, red, false);
    if (b >= 0 && b < used) before[b] = v - own;
    __syncthreads();
    carry += red[31];
  }
  __syncthreads();
  const int lane = tid & 31;
  for (int i = tid >> 5; i < n; i += kPlanThreads / 32) {          // a warp a sequence
    const int begin = starts[i], end = starts[i + 1], tiles = (end - begin + rows - 1) / rows;
    int place = 0;
    if (lane == 0) place = least[tiles + 1] + atomicSub(exact + tiles, 1) - 1;
    place = __shfl_sync(0xffffffffu, place, 0);
    for (int t = lane; t < tiles; t += 32) {
      const int at = before[most_first ? t + 1 : tiles - t] + place;
      if (at < cap) out[at] = make_int4(begin, end, t, begin / kAttnBwdRows + i);
    }
  }
  __syncthreads();
  return carry;
}

// One CTA, once a batch: 8 us for a few sequences, 10 for 128 of 1024 tokens; sequences of one length take their places one after another
// (2000 of 64 tokens 89 us, 100000 of one 4.9 ms).  Forward, the longest tiles first, so that the last ones to start are short.  Backward, the shortest first, because the
// sums of dq pass from the last tile of a sequence to the first.  (Within groups of 16384 to 262144 rows, so that the sums under way
// stay in L2, 32 x 2048 tokens, 16 heads of 128, took 2510 to 2535 us instead of 2535, and 128 x 1024, 12 heads of 64, as long.)
__global__ void __launch_bounds__(kPlanThreads)
attn_plan_kernel(const int* __restrict__ offsets, int n, int total, AttnPlanLayout l, int* plan) {
  __shared__ int red[32];
  __shared__ int bad;
  const int tid = threadIdx.x;
  int *starts = plan + l.starts, *counts = plan + l.counts;
  if (tid == 0) bad = 0;
  pdl_wait();
  __syncthreads();
  // offsets inside [0, total] that never fall
  int carry = 0;
  for (int at = 0; at <= n; at += kPlanThreads) {
    const int i = at + tid, given = i <= n ? offsets[i] : 0;
    const int v = max(carry, block_scan(min(max(given, 0), total), red, true));
    if (i <= n) {
      starts[i] = v;
      if (v != given) bad = 1;
    }
    __syncthreads();
    carry = max(carry, red[31]);
  }
  __syncthreads();
  const int fwd = order_tiles(starts, n, kAttnFwdRows, true, counts, l.bins, reinterpret_cast<int4*>(plan + l.fwd), l.fwd_cap, red);
  const int tiles = order_tiles(starts, n, kAttnBwdRows, false, counts, l.bins, reinterpret_cast<int4*>(plan + l.bwd), l.bwd_cap, red);
  if (tid == 0) {
    plan[kPlanFwdTiles] = fwd;
    plan[kPlanBwdTiles] = tiles;
    plan[kPlanBad] = bad;
    plan[kPlanTotal] = total;
    plan[kPlanSequences] = n;
  }
}

struct DeviceGuardAttn {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuardAttn(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuardAttn() { if (prev >= 0) cudaSetDevice(prev); }
};

int validate_sequences(abs_ctx* ctx, int sequences, long long total) {
  if (sequences < 0 || total < 0)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "sequences and total must be >= 0 (%d, %lld)", sequences, total);
  if (sequences > (1 << 24) || total > (1ll << 30))
    return set_error(ctx, ABS_ERR_UNSUPPORTED, "sequences <= 2^24 and total <= 2^30 (%d, %lld)", sequences, total);
  return ABS_OK;
}
int validate_heads(abs_ctx* ctx, int sequences, long long total, int q_heads, int kv_heads, int head_dim) {
  if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "q_heads %d must be a multiple of kv_heads %d", q_heads, kv_heads);
  if (head_dim < 1) return set_error(ctx, ABS_ERR_INVALID_ARG, "head_dim must be >= 1 (%d)", head_dim);
  if (head_dim > kAttnMaxHead || q_heads > 4096 || total * q_heads > (1ll << 32) || static_cast<long long>(sequences) * q_heads > (1ll << 28))
    return set_error(ctx, ABS_ERR_UNSUPPORTED,
                     "head_dim <= %d, q_heads <= 4096, total * q_heads <= 2^32 and sequences * q_heads <= 2^28 (%d, %d, %lld, %d)", kAttnMaxHead,
                     head_dim, q_heads, total, sequences);
  return ABS_OK;
}
int validate_scale(abs_ctx* ctx, float scale) {       // (the kernels take it log2 e times)
  return scale > -2.0e38f && scale < 2.0e38f ? ABS_OK : set_error(ctx, ABS_ERR_INVALID_ARG, "scale must be within 2e38 of zero");
}
// Rows are disjoint from one another: a token's heads lie within its row (stride of tokens the larger) or a head's tokens within
// the head's block.
int validate_tensor(abs_ctx* ctx, const char* what, const abs_heads* t, long long total, int heads, int head_dim) {
  if (t == nullptr || t->data == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "%s is null", what);
  const long long r = t->row_stride, h = t->head_stride;
  const bool by_row = h >= head_dim && r >= (heads - 1) * h + head_dim;
  const bool by_head = r >= head_dim && h >= (total - 1) * r + head_dim;
  if ((heads > 1 || total > 1) && !(heads == 1 ? r >= head_dim : total == 1 ? h >= head_dim : by_row || by_head))
    return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: rows of %d at strides %lld (token) and %lld (head) overlap", what, head_dim, r, h);
  return ABS_OK;
}
AttnRows rows_of(const abs_heads* t) { return {t->data, t->row_stride, t->head_stride}; }
AttnOut out_of(const abs_heads* t) { return {t->data, t->row_stride, t->head_stride}; }

// Whether the tensor-core kernels take a tensor: bf16 rows that copies of 16 bytes can address, within a tensor map's limits.
bool tc_tensor(const abs_heads* t) {
  const unsigned long long row = static_cast<unsigned long long>(t->row_stride) * 2, head = static_cast<unsigned long long>(t->head_stride) * 2;
  return ((reinterpret_cast<uintptr_t>(t->data) | row | head) & 15u) == 0 && row > 0 && head > 0 && row < (1ull << 40) && head < (1ull << 40);
}

}  // namespace
}  // namespace absk

using namespace absk;

extern "C" int abs_attention_plan_bytes(int sequences, long long total, size_t* out) {
  if (out == nullptr) return set_error(nullptr, ABS_ERR_INVALID_ARG, "out is null");
  const int rc = validate_sequences(nullptr, sequences, total);
  if (rc != ABS_OK) return rc;
  *out = static_cast<size_t>(attn_plan_layout(sequences, static_cast<int>(total)).words) * sizeof(int);
  return ABS_OK;
}

extern "C" int abs_attention_plan(abs_ctx* ctx, const int* offsets, int sequences, long long total, void* plan, size_t plan_bytes,
                                  void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  int rc = validate_sequences(ctx, sequences, total);
  if (rc != ABS_OK) return rc;
  if (plan == nullptr || (offsets == nullptr && sequences > 0)) return set_error(ctx, ABS_ERR_INVALID_ARG, "offsets or plan is null");
  const AttnPlanLayout l = attn_plan_layout(sequences, static_cast<int>(total));
  if (plan_bytes < static_cast<size_t>(l.words) * sizeof(int))
    return set_error(ctx, ABS_ERR_WORKSPACE, "the plan needs %lld bytes, %zu given", l.words * 4, plan_bytes);
  if (reinterpret_cast<uintptr_t>(plan) & 15u) return set_error(ctx, ABS_ERR_INVALID_ARG, "plan must be 16-byte aligned");
  DeviceGuardAttn guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (sequences == 0) {
    ABS_CUDA_TRY(ctx, cudaMemsetAsync(plan, 0, kPlanHeader * sizeof(int), st));
    return ABS_OK;
  }
  ABS_CUDA_TRY(ctx, launch_dependent(attn_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, offsets, sequences, static_cast<int>(total), l,
                                     static_cast<int*>(plan)));
  return ABS_OK;
}

extern "C" int abs_attention_scratch_bytes(long long total, int q_heads, int kv_heads, int head_dim, int sequences, size_t* out) {
  if (out == nullptr) return set_error(nullptr, ABS_ERR_INVALID_ARG, "out is null");
  int rc = validate_sequences(nullptr, sequences, total);
  if (rc == ABS_OK) rc = validate_heads(nullptr, sequences, total, q_heads, kv_heads, head_dim);
  if (rc != ABS_OK) return rc;
  *out = attn_scratch(static_cast<int>(total), q_heads, kv_heads, head_dim, sequences).bytes;
  return ABS_OK;
}

extern "C" int abs_attention(abs_ctx* ctx, const abs_heads* Q, const abs_heads* K, const abs_heads* V, abs_dtype dtype, const void* plan,
                             int sequences, long long total, int q_heads, int kv_heads, int head_dim, float scale, const abs_heads* O,
                             float* lse, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (dtype != ABS_F32 && dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  int rc = validate_sequences(ctx, sequences, total);
  if (rc == ABS_OK) rc = validate_heads(ctx, sequences, total, q_heads, kv_heads, head_dim);
  if (rc != ABS_OK) return rc;
  if ((rc = validate_scale(ctx, scale)) != ABS_OK) return rc;
  if (total == 0 || sequences == 0) return ABS_OK;
  if (plan == nullptr || (reinterpret_cast<uintptr_t>(plan) & 15u)) return set_error(ctx, ABS_ERR_INVALID_ARG, "plan is null or not 16-byte aligned");
  if ((rc = validate_tensor(ctx, "Q", Q, total, q_heads, head_dim)) != ABS_OK) return rc;
  if ((rc = validate_tensor(ctx, "K", K, total, kv_heads, head_dim)) != ABS_OK) return rc;
  if ((rc = validate_tensor(ctx, "V", V, total, kv_heads, head_dim)) != ABS_OK) return rc;
  if ((rc = validate_tensor(ctx, "O", O, total, q_heads, head_dim)) != ABS_OK) return rc;
  DeviceGuardAttn guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  const AttnForward a{rows_of(Q), rows_of(K), rows_of(V), out_of(O), lse, static_cast<const int*>(plan), sequences,
                      static_cast<int>(total), q_heads, kv_heads, head_dim, scale};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // (the running maximum is taken before the scale is applied: a scale of zero or below goes the other way)
  if (dtype == ABS_BF16 && head_dim % 8 == 0 && scale > 0.f && tc_tensor(Q) && tc_tensor(K) && tc_tensor(V) && tc_tensor(O))
    return launch_attention_tc(ctx, a, st);
  return launch_attention_any(ctx, a, dtype, st);
}

extern "C" int abs_attention_backward(abs_ctx* ctx, const abs_heads* dO, const abs_heads* Q, const abs_heads* K, const abs_heads* V,
                                      const abs_heads* O, const float* lse, abs_dtype dtype, const void* plan, int sequences,
                                      long long total, int q_heads, int kv_heads, int head_dim, float scale, const abs_heads* dQ,
                                      const abs_heads* dK, const abs_heads* dV, void* scratch, size_t scratch_bytes, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (dtype != ABS_F32 && dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  int rc = validate_sequences(ctx, sequences, total);
  if (rc == ABS_OK) rc = validate_heads(ctx, sequences, total, q_heads, kv_heads, head_dim);
  if (rc != ABS_OK) return rc;
  if ((rc = validate_scale(ctx, scale)) != ABS_OK) return rc;
  if (total == 0 || sequences == 0) return ABS_OK;
  if (plan == nullptr || (reinterpret_cast<uintptr_t>(plan) & 15u)) return set_error(ctx, ABS_ERR_INVALID_ARG, "plan is null or not 16-byte aligned");
  if (lse == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "lse is null");
  const struct { const char* what; const abs_heads* t; int heads; } all[8] = {
      {"dO", dO, q_heads}, {"Q", Q, q_heads}, {"K", K, kv_heads}, {"V", V, kv_heads}, {"O", O, q_heads},
      {"dQ", dQ, q_heads}, {"dK", dK, kv_heads}, {"dV", dV, kv_heads}};
  for (const auto& x : all)
    if ((rc = validate_tensor(ctx, x.what, x.t, total, x.heads, head_dim)) != ABS_OK) return rc;
  const AttnScratch s = attn_scratch(static_cast<int>(total), q_heads, kv_heads, head_dim, sequences);
  if (scratch == nullptr || scratch_bytes < s.bytes)
    return set_error(ctx, ABS_ERR_WORKSPACE, "scratch of %zu bytes needed, %zu given", s.bytes, scratch ? scratch_bytes : 0);
  if (reinterpret_cast<uintptr_t>(scratch) & 255u) return set_error(ctx, ABS_ERR_INVALID_ARG, "scratch must be 256-byte aligned");
  DeviceGuardAttn guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  const AttnBackward a{rows_of(dO), rows_of(Q), rows_of(K), rows_of(V), rows_of(O), lse, static_cast<const int*>(plan), out_of(dQ),
                       out_of(dK), out_of(dV), sequences, static_cast<int>(total), q_heads, kv_heads, head_dim, scale, scratch};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool tc = dtype == ABS_BF16 && head_dim % 8 == 0;
  for (const auto& x : all) tc = tc && tc_tensor(x.t);
  return tc ? launch_attention_tc_backward(ctx, a, st) : launch_attention_any_backward(ctx, a, dtype, st);
}
