// Causal attention on the CUDA cores: fp32, and bf16 tensors whose layout the tensor-core kernels do not take.
//
//   s_tj = scale <q_t, k_j>, j <= t,   p_tj = exp(s_tj - lse_t),   o_t = sum_j p_tj v_j
//   delta_t = <do_t, o_t>,  ds_tj = p_tj (<do_t, v_j> - delta_t)
//   dv_j = sum_t p_tj do_t,  dk_j = scale sum_t ds_tj q_t,  dq_t = scale sum_j ds_tj k_j
//
// Everything is fp32 from the first product on; outputs are rounded once.  Tiles of 64 x 64 scores, 256 threads with 4 x 4
// scores and 4 rows of the results each; rows lie in shared memory with four words between them, so that eight threads reading
// 16 bytes of eight rows touch all banks once.  128 of 1024 tokens, 12 heads of 64: fp32 9.7 ms forward and 27.9 backward, 21 and 19
// TFLOP/s, bf16 8.8 and 27.7.  What the counters show (16 x 1024 fp32): the pipe that reads shared memory, one read of 16 bytes for eight
// FMAs, is 60 to 69 % busy, issue slots 54 to 57 %, the FMA pipe 37 to 44 %; two CTAs an SM, and tiles are loaded element by element
// with nothing ahead of the products, which is the rest.  Backward in two kernels, keys outside and queries outside: seven products
// instead of five, and no sums across CTAs, so results repeat bit for bit.
#include "abs_attention.cuh"

namespace absk {
namespace {

constexpr int kT = 64;                       // rows and columns of a tile
constexpr int kThreadsA = 256;
constexpr int kStrideS = kT + 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ld_f32(const float* p) { return *p; }
__device__ __forceinline__ float ld_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

struct TileRec {
  int begin, end, block;
};
__device__ __forceinline__ TileRec tile_rec(const int* p, int i) {
  const int4 r = *reinterpret_cast<const int4*>(p + 4 * static_cast<long long>(i));
  return {r.x, r.y, r.z};
}

// Warps of the CTAs of the grid's first row.
__device__ __forceinline__ int warp_of_row() { return blockIdx.x * (kThreadsA / 32) + threadIdx.x / 32; }
__device__ __forceinline__ int warps_of_row() { return gridDim.x * (kThreadsA / 32); }

// Rows [row0, row0 + 64) of one head into shared memory, zeros from `end` on and behind the head's width.
template <typename T, int HDP>
__device__ __forceinline__ void load_rows(float* to, const AttnRows& t, int head, int row0, int end, int hd) {
  const T* base = static_cast<const T*>(t.p) + head * t.head;
  for (int e = threadIdx.x; e < kT * HDP; e += kThreadsA) {
    const int r = e / HDP, c = e - r * HDP;
    const bool in = row0 + r < end && c < hd;
    to[r * (HDP + 4) + c] = in ? ld_f32(base + (row0 + r) * t.row + c) : 0.f;
  }
}

// c[r][k] += <a row ty + 16 r, b row tx + 16 k>
template <int HDP>
__device__ __forceinline__ void products(const float* a, const float* b, int ty, int tx, float (&c)[4][4]) {
#pragma unroll 4
  for (int k = 0; k < HDP; k += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[r] = *reinterpret_cast<const float4*>(a + (ty + 16 * r) * (HDP + 4) + k);
      y[r] = *reinterpret_cast<const float4*>(b + (tx + 16 * r) * (HDP + 4) + k);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        c[r][q] = fmaf(x[r].w, y[q].w, fmaf(x[r].z, y[q].z, fmaf(x[r].y, y[q].y, fmaf(x[r].x, y[q].x, c[r][q]))));
  }
}
// acc[r][.] += sum_j s[j][ty + 16 r] rows[j][.]: a thread has four rows and the columns 4 tx + 64 c
template <int HDP, int NC>
__device__ __forceinline__ void add_rows(const float* s, const float* rows, int ty, int tx, float (&acc)[4][NC][4]) {
#pragma unroll 4
  for (int j = 0; j < kT; ++j) {
    float w[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = s[j * kStrideS + ty + 16 * r];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (HDP < 64 && 4 * tx >= HDP) continue;
      const float4 v = *reinterpret_cast<const float4*>(rows + j * (HDP + 4) + 4 * tx + 64 * c);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        acc[r][c][0] = fmaf(w[r], v.x, acc[r][c][0]);
        acc[r][c][1] = fmaf(w[r], v.y, acc[r][c][1]);
        acc[r][c][2] = fmaf(w[r], v.z, acc[r][c][2]);
        acc[r][c][3] = fmaf(w[r], v.w, acc[r][c][3]);
      }
    }
  }
}
template <typename T, int NC>
__device__ __forceinline__ void store_rows(const AttnOut& t, int head, int row0, int end, int hd, int ty, int tx,
                                           const float (&acc)[4][NC][4], const float (&by)[4]) {
  T* base = static_cast<T*>(t.p) + head * t.head;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = row0 + ty + 16 * r;
    if (row >= end) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = 4 * tx + 64 * c + e;
        if (col < hd) st_f32(base + row * t.row + col, acc[r][c][e] * by[r]);
      }
  }
}

template <typename T, int HDP>
__global__ void __launch_bounds__(kThreadsA)
attn_any_forward_kernel(const AttnForward a, const int* tiles) {
  constexpr int NC = (HDP + 63) / 64;
  extern __shared__ float sm[];
  float *Q = sm, *K = Q + kT * (HDP + 4), *V = K + kT * (HDP + 4), *S = V + kT * (HDP + 4);
  constexpr int kParts = kAttnFwdRows / kT;
  pdl_wait();
  const int tile = blockIdx.x / kParts, part = blockIdx.x % kParts, head = blockIdx.y;
  if (!plan_fits(a.plan, a.n, a.total)) {
    if (head > 0) return;
    fill_nan<T>(a.o, a.total, a.hq, a.hd, warp_of_row(), warps_of_row());
    if (a.lse) fill_nan<float>({a.lse, 1, a.total}, a.total, a.hq, 1, warp_of_row(), warps_of_row());
    return;
  }
  if (tile >= a.plan[kPlanFwdTiles]) return;
  const TileRec rec = tile_rec(tiles, tile);
  const int row0 = rec.begin + rec.block * kAttnFwdRows + part * kT;
  if (row0 >= rec.end) return;
  const int kv = head / (a.hq / a.hk), ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  load_rows<T, HDP>(Q, a.q, head, row0, rec.end, a.hd);
  const float by = a.scale * kLog2e;
  float acc[4][NC][4] = {}, top[4], sum[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    top[r] = -INFINITY;
    sum[r] = 0.f;
  }
  for (int k0 = rec.begin; k0 < row0 + kT && k0 < rec.end; k0 += kT) {
    __syncthreads();
    load_rows<T, HDP>(K, a.k, kv, k0, rec.end, a.hd);
    load_rows<T, HDP>(V, a.v, kv, k0, rec.end, a.hd);
    __syncthreads();
    float c[4][4] = {};
    products<HDP>(Q, K, ty, tx, c);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = row0 + ty + 16 * r;
      float m = -INFINITY;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int key = k0 + tx + 16 * q;
        c[r][q] = key <= row && key < rec.end ? c[r][q] * by : -INFINITY;
        m = fmaxf(m, c[r][q]);
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
      m = fmaxf(m, top[r]);
      const float ref = m == -INFINITY ? 0.f : m, old = exp2f(top[r] - ref);
      top[r] = m;
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float p = exp2f(c[r][q] - ref);
        s += p;
        S[(tx + 16 * q) * kStrideS + ty + 16 * r] = p;
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      sum[r] = fmaf(sum[r], old, s);
#pragma unroll
      for (int q = 0; q < NC; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][q][e] *= old;
    }
    __syncthreads();
    add_rows<HDP, NC>(S, V, ty, tx, acc);
  }
  float inv[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    inv[r] = 1.f / sum[r];
    const int row = row0 + ty + 16 * r;
    if (a.lse && tx == 0 && row < rec.end) a.lse[static_cast<long long>(head) * a.total + row] = fmaf(top[r], kLn2, logf(sum[r]));
  }
  store_rows<T, NC>(a.o, head, row0, rec.end, a.hd, ty, tx, acc, inv);
}

// delta_t = <do_t, o_t>: a warp a row and head.
template <typename T>
__global__ void __launch_bounds__(kThreadsA)
attn_delta_kernel(const AttnBackward a) {
  pdl_wait();
  const long long w = (static_cast<long long>(blockIdx.x) * kThreadsA + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (w >= static_cast<long long>(a.total) * a.hq) return;
  const long long row = w / a.hq, head = w - row * a.hq;
  const T* x = static_cast<const T*>(a.dout.p) + row * a.dout.row + head * a.dout.head;
  const T* y = static_cast<const T*>(a.o.p) + row * a.o.row + head * a.o.head;
  float s = 0.f;
  for (int c = lane; c < a.hd; c += 32) s = fmaf(ld_f32(x + c), ld_f32(y + c), s);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  if (lane == 0) static_cast<float*>(a.scratch)[head * a.total + row] = s;
}

// p and ds of a tile from its scores and products with dout, into shared memory: [query][key] (by_key: [key][query]).
__device__ __forceinline__ void softmax_gradient(const AttnBackward& a, const float* lse, const float* delta, int q0, int k0, int end,
                                                 int ty, int tx, const float (&c)[4][4], const float (&d)[4][4], float* P,
                                                 float* D, bool by_key) {
  const float by = a.scale * kLog2e;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = q0 + ty + 16 * r;
    const float l = row < end ? lse[row] * kLog2e : 0.f, dl = row < end ? delta[row] : 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int key = k0 + tx + 16 * q;
      const bool in = key <= row && row < end;
      const float p = in ? exp2f(fmaf(c[r][q], by, -l)) : 0.f, ds = in ? p * (d[r][q] - dl) : 0.f;
      const int at = by_key ? (tx + 16 * q) * kStrideS + ty + 16 * r : (ty + 16 * r) * kStrideS + tx + 16 * q;
      if (P) P[at] = p;
      D[at] = ds;
    }
  }
}

template <typename T, int HDP>
__global__ void __launch_bounds__(kThreadsA)
attn_any_keys_kernel(const AttnBackward a, const int* tiles) {
  constexpr int NC = (HDP + 63) / 64, kRow = kT * (HDP + 4);
  extern __shared__ float sm[];
  float *K = sm, *V = K + kRow, *Q = V + kRow, *G = Q + kRow, *P = G + kRow, *D = P + kT * kStrideS;
  constexpr int kParts = kAttnBwdRows / kT;
  pdl_wait();
  const int tile = blockIdx.x / kParts, part = blockIdx.x % kParts, kv = blockIdx.y;
  if (!plan_fits(a.plan, a.n, a.total)) {
    if (kv > 0) return;
    fill_nan<T>(a.dk, a.total, a.hk, a.hd, warp_of_row(), warps_of_row());
    fill_nan<T>(a.dv, a.total, a.hk, a.hd, warp_of_row(), warps_of_row());
    return;
  }
  if (tile >= a.plan[kPlanBwdTiles]) return;
  const TileRec rec = tile_rec(tiles, tile);
  const int k0 = rec.begin + rec.block * kAttnBwdRows + part * kT;
  if (k0 >= rec.end) return;
  const int group = a.hq / a.hk, ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  load_rows<T, HDP>(K, a.k, kv, k0, rec.end, a.hd);
  load_rows<T, HDP>(V, a.v, kv, k0, rec.end, a.hd);
  float dk[4][NC][4] = {}, dv[4][NC][4] = {};
  for (int head = kv * group; head < (kv + 1) * group; ++head) {
    const float* lse = a.lse + static_cast<long long>(head) * a.total;
    const float* delta = static_cast<const float*>(a.scratch) + static_cast<long long>(head) * a.total;
    for (int q0 = k0; q0 < rec.end; q0 += kT) {
      __syncthreads();
      load_rows<T, HDP>(Q, a.q, head, q0, rec.end, a.hd);
      load_rows<T, HDP>(G, a.dout, head, q0, rec.end, a.hd);
      __syncthreads();
      float c[4][4] = {}, d[4][4] = {};
      products<HDP>(Q, K, ty, tx, c);
      products<HDP>(G, V, ty, tx, d);
      softmax_gradient(a, lse, delta, q0, k0, rec.end, ty, tx, c, d, P, D, false);
      __syncthreads();
      add_rows<HDP, NC>(P, G, ty, tx, dv);
      add_rows<HDP, NC>(D, Q, ty, tx, dk);
    }
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, by[4] = {a.scale, a.scale, a.scale, a.scale};
  store_rows<T, NC>(a.dk, kv, k0, rec.end, a.hd, ty, tx, dk, by);
  store_rows<T, NC>(a.dv, kv, k0, rec.end, a.hd, ty, tx, dv, one);
}

template <typename T, int HDP>
__global__ void __launch_bounds__(kThreadsA)
attn_any_queries_kernel(const AttnBackward a, const int* tiles) {
  constexpr int NC = (HDP + 63) / 64, kRow = kT * (HDP + 4);
  extern __shared__ float sm[];
  float *K = sm, *V = K + kRow, *Q = V + kRow, *G = Q + kRow, *D = G + kRow;
  constexpr int kParts = kAttnFwdRows / kT;
  pdl_wait();
  const int tile = blockIdx.x / kParts, part = blockIdx.x % kParts, head = blockIdx.y;
  if (!plan_fits(a.plan, a.n, a.total)) {
    if (head > 0) return;
    fill_nan<T>(a.dq, a.total, a.hq, a.hd, warp_of_row(), warps_of_row());
    return;
  }
  if (tile >= a.plan[kPlanFwdTiles]) return;
  const TileRec rec = tile_rec(tiles, tile);
  const int q0 = rec.begin + rec.block * kAttnFwdRows + part * kT;
  if (q0 >= rec.end) return;
  const int kv = head / (a.hq / a.hk), ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  const float* lse = a.lse + static_cast<long long>(head) * a.total;
  const float* delta = static_cast<const float*>(a.scratch) + static_cast<long long>(head) * a.total;
  load_rows<T, HDP>(Q, a.q, head, q0, rec.end, a.hd);
  load_rows<T, HDP>(G, a.dout, head, q0, rec.end, a.hd);
  float dq[4][NC][4] = {};
  for (int k0 = rec.begin; k0 < q0 + kT && k0 < rec.end; k0 += kT) {
    __syncthreads();
    load_rows<T, HDP>(K, a.k, kv, k0, rec.end, a.hd);
    load_rows<T, HDP>(V, a.v, kv, k0, rec.end, a.hd);
    __syncthreads();
    float c[4][4] = {}, d[4][4] = {};
    products<HDP>(Q, K, ty, tx, c);
    products<HDP>(G, V, ty, tx, d);
    softmax_gradient(a, lse, delta, q0, k0, rec.end, ty, tx, c, d, nullptr, D, true);
    __syncthreads();
    add_rows<HDP, NC>(D, K, ty, tx, dq);
  }
  const float by[4] = {a.scale, a.scale, a.scale, a.scale};
  store_rows<T, NC>(a.dq, head, q0, rec.end, a.hd, ty, tx, dq, by);
}

size_t smem_any(int hdp, int tensors, int scores) {
  return (static_cast<size_t>(tensors) * kT * (hdp + 4) + static_cast<size_t>(scores) * kT * kStrideS) * sizeof(float);
}

template <typename T, int HDP>
int run_forward_any(abs_ctx* ctx, const AttnForward& a, cudaStream_t st) {
  const AttnPlanLayout l = attn_plan_layout(a.n, a.total);
  const size_t smem = smem_any(HDP, 3, 1);
  auto kern = attn_any_forward_kernel<T, HDP>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(l.fwd_cap * (kAttnFwdRows / kT), a.hq), dim3(kThreadsA), smem, st, a, a.plan + l.fwd));
  return ABS_OK;
}
template <typename T, int HDP>
int run_backward_any(abs_ctx* ctx, const AttnBackward& a, cudaStream_t st) {
  const AttnPlanLayout l = attn_plan_layout(a.n, a.total);
  const long long warps = static_cast<long long>(a.total) * a.hq;
  ABS_CUDA_TRY(ctx, launch_dependent(attn_delta_kernel<T>, dim3(static_cast<unsigned>((warps * 32 + kThreadsA - 1) / kThreadsA)),
                                     dim3(kThreadsA), 0, st, a));
  auto keys = attn_any_keys_kernel<T, HDP>;
  auto queries = attn_any_queries_kernel<T, HDP>;
  const size_t smem_k = smem_any(HDP, 4, 2), smem_q = smem_any(HDP, 4, 1);
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, keys, smem_k));
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, queries, smem_q));
  ABS_CUDA_TRY(ctx, launch_dependent(keys, dim3(l.bwd_cap * (kAttnBwdRows / kT), a.hk), dim3(kThreadsA), smem_k, st, a, a.plan + l.bwd));
  ABS_CUDA_TRY(ctx, launch_dependent(queries, dim3(l.fwd_cap * (kAttnFwdRows / kT), a.hq), dim3(kThreadsA), smem_q, st, a, a.plan + l.fwd));
  return ABS_OK;
}

}  // namespace

int launch_attention_any(abs_ctx* ctx, const AttnForward& a, abs_dtype dtype, cudaStream_t st) {
  const bool f = dtype == ABS_F32;
  if (a.hd <= 32) return f ? run_forward_any<float, 32>(ctx, a, st) : run_forward_any<__nv_bfloat16, 32>(ctx, a, st);
  if (a.hd <= 64) return f ? run_forward_any<float, 64>(ctx, a, st) : run_forward_any<__nv_bfloat16, 64>(ctx, a, st);
  return f ? run_forward_any<float, 128>(ctx, a, st) : run_forward_any<__nv_bfloat16, 128>(ctx, a, st);
}
int launch_attention_any_backward(abs_ctx* ctx, const AttnBackward& a, abs_dtype dtype, cudaStream_t st) {
  const bool f = dtype == ABS_F32;
  if (a.hd <= 32) return f ? run_backward_any<float, 32>(ctx, a, st) : run_backward_any<__nv_bfloat16, 32>(ctx, a, st);
  if (a.hd <= 64) return f ? run_backward_any<float, 64>(ctx, a, st) : run_backward_any<__nv_bfloat16, 64>(ctx, a, st);
  return f ? run_backward_any<float, 128>(ctx, a, st) : run_backward_any<__nv_bfloat16, 128>(ctx, a, st);
}

}  // namespace absk
