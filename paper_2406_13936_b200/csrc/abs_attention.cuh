// Causal attention over packed sequences: what the host side and plan (abs_attention.cu), the CUDA-core kernels
// (abs_attention_any.cu) and the tensor-core kernels (abs_attention_fwd.cu, abs_attention_bwd.cu) share.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "abs_internal.cuh"

namespace absk {

constexpr int kAttnMaxHead = 128;
constexpr int kAttnFwdRows = 256;          // query rows of a forward tile
constexpr int kAttnBwdRows = 128;          // keys of a backward tile

// The plan of a batch, int32 words on the device: the header, then the records of the forward and of the backward tiles in
// the order in which they are worked off, then what the plan's own kernel needs.
//   record: first row and end of the tile's sequence, number of the tile in the sequence, and the sequence's first slot: a number
//   such that slot + (tile of 128 rows) is each tile's own, below bwd_cap
struct AttnPlanLayout {
  long long fwd, bwd, starts, counts, words;   // places of the parts, and their end
  int fwd_cap, bwd_cap, bins;
};
enum { kPlanFwdTiles = 0, kPlanBwdTiles = 1, kPlanBad = 2, kPlanTotal = 3, kPlanSequences = 4, kPlanHeader = 16 };
inline AttnPlanLayout attn_plan_layout(int n, int total) {
  AttnPlanLayout l;
  l.fwd_cap = total / kAttnFwdRows + n;
  l.bwd_cap = total / kAttnBwdRows + n;
  l.bins = total / kAttnBwdRows + 3;           // tiles of one sequence, and one more: 0 to bins - 1
  l.fwd = kPlanHeader;
  l.bwd = l.fwd + 4ll * l.fwd_cap;
  l.starts = l.bwd + 4ll * l.bwd_cap;
  l.counts = l.starts + n + 1;
  l.words = l.counts + 3ll * l.bins;
  l.words = (l.words + 3) & ~3ll;
  return l;
}

// One tensor's rows: row r, head h at p + r * row + h * head.
struct AttnRows {
  const void* p;
  long long row, head;
};
struct AttnOut {
  void* p;
  long long row, head;
};
#ifdef __CUDACC__
// Whether the plan was made for the call's numbers: where its records lie depends on them, and what they say are rows.
__device__ __forceinline__ bool plan_fits(const int* plan, int n, int total) {
  return __ldg(plan + kPlanTotal) == total && __ldg(plan + kPlanSequences) == n;
}
// Every row of every head, NaN: what a plan that does not fit gives.  The caller is warp `at` of `step`.
template <typename T>
__device__ __forceinline__ void fill_nan(const AttnOut& o, int total, int heads, int hd, int at, int step) {
  for (long long row = at; row < total; row += step)
    for (int head = 0; head < heads; ++head)
      for (int c = threadIdx.x & 31; c < hd; c += 32) static_cast<T*>(o.p)[row * o.row + head * o.head + c] = static_cast<T>(__int_as_float(0x7fc00000));
}
#endif
// Whether every row of every head is whole sectors of 32 bytes of a 16-bit type.
inline bool in_sectors(const AttnOut& o, int hd) {
  return reinterpret_cast<uintptr_t>(o.p) % 32 == 0 && o.row % 16 == 0 && o.head % 16 == 0 && hd % 16 == 0;
}
bool encode_heads_map(const AttnRows& t, int total, int heads, int hd, CUtensorMap* map);      // boxes of 128 rows x 64 columns of a head
struct AttnForward {
  AttnRows q, k, v;
  AttnOut o;
  float* lse;                                  // [hq][total] or NULL
  const int* plan;
  int n, total, hq, hk, hd;
  float scale;
};
struct AttnBackward {
  AttnRows dout, q, k, v, o;
  const float* lse;
  const int* plan;
  AttnOut dq, dk, dv;
  int n, total, hq, hk, hd;
  float scale;
  void* scratch;
};

// Into how many parts the tensor-core kernel's backward pass splits a group's query heads: a key tile and head is one CTA's work for all
// queries of the group, and with fewer than eight tiles an SM the last ones to finish (128 keys of a long sequence, 8 query heads:
// hundreds of blocks) are most of the time: 9 sequences of 1 to 1500 rows, 16 heads of 128 and 2 of keys, whole 502 us, in parts 263 (since then 130).
// (A rule of sizes alone: the scratch depends on it.)
inline int attn_parts(int total, int hq, int hk, int n) {
  const long long tiles = (static_cast<long long>(total) / kAttnBwdRows + n) * hk;
  const int group = hq / hk;
  int parts = 1;
  while (parts < group && tiles * parts < 8 * kSmCountFallback) {
    ++parts;
    while (group % parts != 0) ++parts;
  }
  return parts;
}
// Scratch of a backward pass: two rows of [hq][total] fp32 (delta; the tensor-core kernel: -lse log2 e and -delta), then, for the
// tensor-core kernel, the sums of dq [hq][total][dpad] fp32, dv and dk of the parts of a group, a counter for each 128 rows of a
// sequence, head and 64 columns, and one of the tiles taken.
struct AttnScratch {
  size_t delta, sums, partial, counters, bytes;
  int dpad;
};
inline AttnScratch attn_scratch(int total, int hq, int hk, int hd, int n) {
  AttnScratch s;
  auto up = [](size_t v) { return (v + 255) & ~static_cast<size_t>(255); };
  const int parts = attn_parts(total, hq, hk, n);
  s.dpad = hd <= 64 ? 64 : 128;
  const size_t head = static_cast<size_t>(total) * s.dpad * sizeof(float);
  s.delta = 0;
  s.sums = up(static_cast<size_t>(hq) * total * 2 * sizeof(float));
  s.partial = up(s.sums + hq * head);
  s.counters = up(s.partial + (parts > 1 ? 2 * static_cast<size_t>(parts) * hk * head : 0));
  s.bytes = up(s.counters + (static_cast<size_t>(hq) * (static_cast<size_t>(total) / kAttnBwdRows + n) * (s.dpad / 64) + 1) * sizeof(unsigned));
  return s;
}

inline uint32_t fault_steps(const abs_ctx* ctx) {
  const long long n = ctx->tuning.attention_fault_stop_after;
  return n > 0 && n < 0xffffffffll ? static_cast<uint32_t>(n) : 0xffffffffu;
}

int launch_attention_tc(abs_ctx* ctx, const AttnForward& a, cudaStream_t st);          // bf16 rows of 16-byte pieces, scale > 0
int launch_attention_tc_backward(abs_ctx* ctx, const AttnBackward& a, cudaStream_t st);
int launch_attention_any(abs_ctx* ctx, const AttnForward& a, abs_dtype dtype, cudaStream_t st);
int launch_attention_any_backward(abs_ctx* ctx, const AttnBackward& a, abs_dtype dtype, cudaStream_t st);

}  // namespace absk
