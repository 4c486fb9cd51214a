// Causal attention, backward, bf16 on the tcgen05 tensor cores.
//
//   p_tj = 2^(c <q_t, k_j> - lse_t log2 e),  c = scale log2 e
//   ds_tj = p_tj (<do_t, v_j> - delta_t),  delta_t = <do_t, o_t>
//   dv_j = sum_t p_tj do_t,  dk_j = scale sum_t ds_tj q_t,  dq_t = scale sum_j ds_tj k_j
//
// A tile is 128 keys of one key head.  Its CTA goes over the queries that see them in blocks of 128, of every query head of the group;
// dk and dv stay in tensor memory until the tile is done.  Five products a block, all transposed so that a thread of the softmax has a
// key's row and the sums over queries run along k: S' = K Q', dP' = V dO', then dV += P' dO with P' written back over S' in tensor
// memory, dK += dS' Q and dQ = dS K with dS' in shared memory once, read along its rows for the one and along its columns (MN-major)
// for the other.
//
// dQ is a sum over key tiles, which different CTAs have.  They add to fp32 sums in scratch (bulk reductions, L2), for each block of
// queries in a fixed order, so results repeat bit for bit: tile j of a sequence starts at query block j and goes up, so block i is
// reached first by tile i, then by i - 1, and so on, each a step later than the one before; a counter a block says whose turn it is,
// and the wait is rarely one.  The first of them stores instead of adding (nothing is cleared), and the last, tile 0, adds its own part
// to the sums and writes dq: sequences of up to 128 rows never touch the sums.  Tiles are worked off shortest first within a group of
// sequences and some of the heads (attn_plan_kernel), so that the sums under way stay in L2.
// The grid is resident (a cooperative launch) and every CTA takes its tiles in that order, in which each comes after those that it waits
// for, so the first unfinished tile of all never waits.
//
// Rounded to fewer bits than 32: P and dS to bf16, as operands of the tensor core, and the results.
//
// Bound by the products at 128 columns a head (five of 512 clocks per 128 x 128 scores), at 64 (five of 256) by the products and by
// what the softmax warps issue alike.
//
// Roles of the 16 warps: 0 loads (TMA), 1 issues the products, 2 loads lse and delta, 3 sends dq's sums, 4-7 take dq out of tensor memory,
// 8-15 are the softmax: 64 of a block's 128 queries each half.  While they compute P' of a block, dQ and dK of the block before and
// dP' of this one run; while they compute dS', dV and the next S'.  All waits are bounded: one that runs out raises the CTA's
// abort flag, every role falls through, copies in flight are waited for, tensor memory is freed, and what was not finished is NaN.
#include "abs_attention.cuh"
#include "abs_tc.cuh"

namespace absk {
namespace {

constexpr int kThreadsB = 512;
constexpr int kBlock = 128;                   // keys of a tile, queries of a block
constexpr int kRegsLoad = 72, kRegsOut = 104, kRegsSoft = 168;      // of a thread; together what 128 a thread are at the launch
static_assert(128 * (kRegsLoad + kRegsOut + 2 * kRegsSoft) == kThreadsB * 128, "");
constexpr float kLog2eB = 1.4426950408889634f;

template <int HD> struct BwdShape {
  static constexpr uint32_t kRows = kBlock * HD * 2;              // 128 rows of one head, bf16
  static constexpr uint32_t kKv = HD == 64 ? 2 : 1;               // places for a tile's K and V
  static constexpr uint32_t kQ = 2, kDo = HD == 64 ? 2 : 1;       // places for Q and dO
  static constexpr uint32_t kDs = kBlock * kBlock * 2;
  static constexpr int kPart = 32;                                // columns of dq that a place for sums has
  static constexpr int kParts = HD / kPart;
  static constexpr uint32_t kStage = kBlock * kPart * 4;          // 16 KB
  static constexpr uint32_t kStages = HD == 64 ? 3 : 1;
  static constexpr uint32_t kStats = 2 * kBlock * 4;              // -lse and -delta of a block
  static constexpr uint32_t kData = 2 * kKv * kRows + (kQ + kDo) * kRows + kDs + kStages * kStage + 2 * kStats;
  static constexpr size_t kSmem = kData + 1024 + 512;
  // tensor memory: S' (P' over it), dP', dV, dK, dQ (128 columns a head: over dP')
  static constexpr uint32_t kS = 0, kDp = 128, kDv = 256, kDk = 256 + HD, kDq = HD == 64 ? 384 : kDp;
};
static_assert(BwdShape<64>::kSmem <= 232448 && BwdShape<128>::kSmem <= 232448, "");

struct BwdMaps {
  CUtensorMap q, k, v, dout;
};
struct BwdParams {
  AttnOut dq, dk, dv;
  const float* stats;                         // [2][hq][total]
  float* sums;                                // [hq][total][HD], 16-byte pieces of row r permuted by r
  unsigned* counters;                         // [hq][cap]
  const int* plan;
  const int* tiles;
  const int* groups;
  int total, hq, hk, group, hd, cap;
  int heads_at_once;
  float by, scale;                            // scale log2 e, scale
  long long limit;
  int drop_loads;
};
struct BwdItem {
  int begin, len, slot, tile, kv;
  int blocks, steps;                          // query blocks from the tile on, and of all the group's heads
};
__device__ __forceinline__ BwdItem bwd_item(const BwdParams& p, int i) {
  const int4* recs = reinterpret_cast<const int4*>(p.tiles);
  const int g = __ldg(recs + i / p.hk).x >> kAttnGroupBits;
  const int t0 = __ldg(p.groups + g), n = __ldg(p.groups + g + 1) - t0, local = i - p.hk * t0;
  const int chunk = local / (n * p.heads_at_once), first = chunk * p.heads_at_once, rem = local - first * n;
  const int heads = min(p.heads_at_once, p.hk - first);
  const int4 r = __ldg(recs + t0 + rem / heads);
  BwdItem it;
  it.kv = first + rem % heads;
  it.begin = r.x;
  it.len = r.y - r.x;
  it.tile = r.z;
  it.slot = r.w;
  it.blocks = (it.len + kBlock - 1) / kBlock - r.z;
  it.steps = it.blocks * p.group;
  return it;
}
// Step t of a tile: the query head and the block.
__device__ __forceinline__ void bwd_step(const BwdParams& p, const BwdItem& it, int t, int& head, int& block) {
  const int h = t / it.blocks;
  head = it.kv * p.group + h;
  block = it.tile + t - h * it.blocks;
}

// Waits (bounded) until the counter has reached `target`.
__device__ __forceinline__ bool wait_turn(const unsigned* c, unsigned target, volatile unsigned* abort_flag, long long limit) {
  const long long t0 = clock64();
  for (;;) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(c) : "memory");
    if (v >= target) return true;
    if (*abort_flag || clock64() - t0 > limit) {
      *abort_flag = 1u;
      return false;
    }
    __nanosleep(64);
  }
}

template <int HD>
__global__ void __launch_bounds__(kThreadsB, 1)
attn_backward_kernel(const __grid_constant__ BwdMaps maps, const __grid_constant__ BwdParams p) {
  typedef BwdShape<HD> Sh;
  constexpr uint32_t kRows = Sh::kRows;
  extern __shared__ unsigned char smem_dyn[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_dyn), kv_at = (raw + 1023u) & ~1023u, q_at = kv_at + 2u * Sh::kKv * kRows,
                 do_at = q_at + Sh::kQ * kRows, ds_at = do_at + Sh::kDo * kRows, stage_at = ds_at + Sh::kDs,
                 stats_at = stage_at + Sh::kStages * Sh::kStage;
  unsigned char* base = smem_dyn + (kv_at - raw);
  float* stats = reinterpret_cast<float*>(base + (stats_at - kv_at));
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(base + Sh::kData);
  constexpr int kBars = 36;
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + kBars);
  unsigned* tmem_slot = const_cast<unsigned*>(abort_flag) + 1;
  const uint32_t b0 = smem_u32(bars);
  // two (sums: three) of each of the first ones
  const uint32_t kv_full = b0, kv_free = b0 + 16u, q_full = b0 + 32u, q_free = b0 + 48u, do_full = b0 + 64u, do_free = b0 + 80u,
                 st_full = b0 + 96u, st_free = b0 + 112u, staged = b0 + 128u, stage_free = b0 + 152u, sums_in = b0 + 176u, s_full = b0 + 200u,
                 p_full = b0 + 208u, dp_full = b0 + 216u, ds_full = b0 + 224u, dq_full = b0 + 232u, dq_read = b0 + 240u, acc_full = b0 + 248u,
                 acc_free = b0 + 256u, landed = b0 + 264u, done_bar = b0 + 272u;
  if (threadIdx.x == 0) {
    for (uint32_t k = 0; k < 2; ++k) {
      mbar_init(kv_full + 8u * k, 1);
      mbar_init(kv_free + 8u * k, 1);
      mbar_init(q_full + 8u * k, 1);
      mbar_init(q_free + 8u * k, 1);
      mbar_init(do_full + 8u * k, 1);
      mbar_init(do_free + 8u * k, 1);
      mbar_init(st_full + 8u * k, 1);
      mbar_init(st_free + 8u * k, 8);
    }
    for (uint32_t k = 0; k < 3; ++k) {
      mbar_init(staged + 8u * k, 4);
      mbar_init(stage_free + 8u * k, 1);
      mbar_init(sums_in + 8u * k, 1);
    }
    mbar_init(s_full, 1);
    mbar_init(p_full, 8);
    mbar_init(dp_full, 1);
    mbar_init(ds_full, 8);
    mbar_init(dq_full, 1);
    mbar_init(dq_read, 4);
    mbar_init(acc_full, 1);
    mbar_init(acc_free, 8);
    mbar_init(landed, 1);
    mbar_init(done_bar, 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_all(smem_u32(tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int items = __ldg(p.plan + kPlanBwdTiles) * p.hk;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLoad));
    if (warp == 0) {
      // ---- loads -----------------------------------------------------------------------------------
      uint32_t lands = 0, tiles = 0, n = 0;                      // tiles and steps so far
      bool ok = !p.drop_loads;
      auto copy = [&](const CUtensorMap* map, uint32_t to, int head, int row, uint32_t bar) {
        if (elect_lane()) {
#pragma unroll
          for (uint32_t c = 0; c < HD / 64; ++c) tma_load_3d(to + c * (kBlock * 128u), map, 64 * static_cast<int>(c), head, row, bar);
        }
        __syncwarp();
      };
      auto expect = [&](uint32_t bar, uint32_t bytes) {
        if (elect_lane()) mbar_expect_tx(bar, bytes);
        __syncwarp();
      };
      // 128 rows of one head from the sequence's row `first` on; those behind the sequence, which may hold anything, become zeros
      // (all of them are operands of products that run along these rows)
      auto copy_rows = [&](const CUtensorMap* map, uint32_t to, const BwdItem& it, int head, int first, uint32_t bar) {
        const int in = it.len - first;
        if (in >= kBlock) {
          expect(bar, kRows);
          copy(map, to, head, it.begin + first, bar);
          return;
        }
        expect(landed, kRows);
        copy(map, to, head, it.begin + first, landed);
        ok = warp_wait(landed, lands & 1u, abort_flag, p.limit);
        ++lands;
        for (uint32_t c = 0; c < HD / 64; ++c)
          for (uint32_t e = static_cast<uint32_t>(in) * 128u + lane * 16u; e < kBlock * 128u; e += 512u)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + c * (kBlock * 128u) + e), "r"(0u) : "memory");
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      };
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const BwdItem it = bwd_item(p, i);
        const uint32_t kv = tiles % Sh::kKv, kvs = kv_at + kv * 2u * kRows;
        if (tiles >= Sh::kKv) ok = warp_wait(kv_free + 8u * kv, (tiles / Sh::kKv - 1) & 1u, abort_flag, p.limit);
        if (!ok) break;
        // V is an operand along its rows only once, of products whose rows behind the sequence are masked: as it comes
        if (it.len - it.tile * kBlock >= kBlock) {
          expect(kv_full + 8u * kv, 2u * kRows);
          copy(&maps.k, kvs, it.kv, it.begin + it.tile * kBlock, kv_full + 8u * kv);
          copy(&maps.v, kvs + kRows, it.kv, it.begin + it.tile * kBlock, kv_full + 8u * kv);
        } else {
          expect(landed, kRows);
          copy(&maps.v, kvs + kRows, it.kv, it.begin + it.tile * kBlock, landed);
          ok = warp_wait(landed, lands & 1u, abort_flag, p.limit);
          ++lands;
          if (ok) copy_rows(&maps.k, kvs, it, it.kv, it.tile * kBlock, kv_full + 8u * kv);
        }
        ++tiles;
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          int head, block;
          bwd_step(p, it, t, head, block);
          const uint32_t qs = n % Sh::kQ, ds = n % Sh::kDo;
          if (n >= Sh::kQ) ok = warp_wait(q_free + 8u * qs, (n / Sh::kQ - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          copy_rows(&maps.q, q_at + qs * kRows, it, head, block * kBlock, q_full + 8u * qs);
          if (ok && n >= Sh::kDo) ok = warp_wait(do_free + 8u * ds, (n / Sh::kDo - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          copy_rows(&maps.dout, do_at + ds * kRows, it, head, block * kBlock, do_full + 8u * ds);
        }
      }
      // Waits (bounded) until every copy that was issued has arrived, whatever made the other roles stop.  (After an abort a place's last
      // copy may be one further on than the count says: its wait may run out for nothing, which is bounded too.)
      volatile unsigned ignore = 0u;
      const bool stopped = *abort_flag != 0u;
      for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t f_kv = k < Sh::kKv ? tiles / Sh::kKv + (k < tiles % Sh::kKv ? 1u : 0u) : 0u;
        const uint32_t f_q = n / Sh::kQ + (k < n % Sh::kQ ? 1u : 0u);
        const uint32_t f_do = k < Sh::kDo ? n / Sh::kDo + (k < n % Sh::kDo ? 1u : 0u) : 0u;
        if (f_kv > 0) mbar_wait(kv_full + 8u * k, (f_kv - 1) & 1u, &ignore, p.limit);
        if (f_q > 0) mbar_wait(q_full + 8u * k, (f_q - 1) & 1u, &ignore, p.limit);
        if (f_do > 0) mbar_wait(do_full + 8u * k, (f_do - 1) & 1u, &ignore, p.limit);
      }
      if (stopped) mbar_wait(q_full + 8u * (n % Sh::kQ), (n / Sh::kQ) & 1u, &ignore, 1000000);
    } else if (warp == 1) {
      // ---- products --------------------------------------------------------------------------------
      constexpr uint32_t idesc_s = mma_idesc(kBlock, kBlock, false, false), idesc_k = mma_idesc(kBlock, HD, false, true),
                         idesc_q = mma_idesc(kBlock, HD, true, true);
      constexpr uint64_t mn = desc_mn(kBlock * 128);
      uint32_t tiles = 0, n = 0;
      bool ok = true;
      // S' or dP' = rows of keys times rows of queries
      auto scores = [&](uint32_t to, uint32_t a_at, uint32_t b_at, uint32_t bar) {
        if (elect_lane()) {
          const uint32_t a = desc_at(a_at), b = desc_at(b_at);
#pragma unroll
          for (uint32_t k = 0; k < HD / 16; ++k) {
            const uint32_t off = (k / 4) * (kBlock * 128u / 16u) + (k % 4) * 2u;
            mma_ss(tmem + to, kDescK | (a + off), kDescK | (b + off), idesc_s, k > 0);
          }
          mma_commit(bar);
        }
        __syncwarp();
      };
      // dQ and dK of step m (counted over all tiles) from its dS'
      auto gradients = [&](uint32_t m, bool first, uint32_t kvs) {
        ok = ok && warp_wait(ds_full, m & 1u, abort_flag, p.limit);
        if (ok && m > 0 && HD == 64) ok = warp_wait(dq_read, (m - 1) & 1u, abort_flag, p.limit);
        if (!ok) return;
        tc_fence_after();
        if (elect_lane()) {
          const uint32_t d = desc_at(ds_at), k_ = desc_at(kvs), q = desc_at(q_at + (m % Sh::kQ) * kRows);
#pragma unroll
          for (uint32_t k = 0; k < kBlock / 16; ++k) mma_ss(tmem + Sh::kDq, mn | (d + 128u * k), mn | (k_ + 128u * k), idesc_q, k > 0);
          mma_commit(dq_full);
#pragma unroll
          for (uint32_t k = 0; k < kBlock / 16; ++k) {
            const uint32_t off = (k / 4) * (kBlock * 128u / 16u) + (k % 4) * 2u;
            mma_ss(tmem + Sh::kDk, kDescK | (d + off), mn | (q + 128u * k), idesc_k, (!first || k > 0) ? 1u : 0u);
          }
          mma_commit(q_free + 8u * (m % Sh::kQ));
        }
        __syncwarp();
      };
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const BwdItem it = bwd_item(p, i);
        const uint32_t kv = tiles % Sh::kKv, kvs = kv_at + kv * 2u * kRows;
        ok = warp_wait(kv_full + 8u * kv, (tiles / Sh::kKv) & 1u, abort_flag, p.limit);
        ok = ok && warp_wait(q_full + 8u * (n % Sh::kQ), (n / Sh::kQ) & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        scores(Sh::kS, kvs, q_at + (n % Sh::kQ) * kRows, s_full);
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          if (t > 0) gradients(n - 1, t == 1, kvs);
          const uint32_t ds = n % Sh::kDo;
          ok = ok && warp_wait(do_full + 8u * ds, (n / Sh::kDo) & 1u, abort_flag, p.limit);
          if (HD == 128 && n > 0) ok = ok && warp_wait(dq_read, (n - 1) & 1u, abort_flag, p.limit);       // dQ of the step before lies over dP'
          if (!ok) break;
          tc_fence_after();
          scores(Sh::kDp, kvs + kRows, do_at + ds * kRows, dp_full);
          ok = warp_wait(p_full, n & 1u, abort_flag, p.limit);
          if (ok && t == 0 && tiles > 0) ok = warp_wait(acc_free, (tiles - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          tc_fence_after();
          if (elect_lane()) {
            const uint32_t d = desc_at(do_at + ds * kRows);
#pragma unroll
            for (uint32_t k = 0; k < kBlock / 16; ++k)       // P' of the first 64 queries lies at columns 0-31, of the others at 64-95
              mma_ts(tmem + Sh::kDv, tmem + Sh::kS + 64u * (k / 4) + 8u * (k % 4), mn | (d + 128u * k), idesc_k, (t > 0 || k > 0) ? 1u : 0u);
            mma_commit(do_free + 8u * ds);
          }
          __syncwarp();
          if (t + 1 < it.steps) {
            const uint32_t next = n + 1;
            ok = warp_wait(q_full + 8u * (next % Sh::kQ), (next / Sh::kQ) & 1u, abort_flag, p.limit);
            if (!ok) break;
            tc_fence_after();
            scores(Sh::kS, kvs, q_at + (next % Sh::kQ) * kRows, s_full);
          }
        }
        if (!ok) break;
        gradients(n - 1, it.steps == 1, kvs);
        if (elect_lane()) {
          mma_commit(acc_full);
          mma_commit(kv_free + 8u * kv);
        }
        __syncwarp();
        ++tiles;
      }
      if (elect_lane()) mma_commit(done_bar);
      __syncwarp();
      volatile unsigned ignore = 0u;
      mbar_wait(done_bar, 0u, &ignore, p.limit);                 // no product in flight when tensor memory is freed
    } else if (warp == 2) {
      // ---- lse and delta of a block's queries ------------------------------------------------------
      uint32_t n = 0;
      bool ok = true;
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const BwdItem it = bwd_item(p, i);
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          int head, block;
          bwd_step(p, it, t, head, block);
          const float* from = p.stats + static_cast<long long>(head) * p.total + it.begin;
          const long long other = static_cast<long long>(p.hq) * p.total;
          float l[4], d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = block * kBlock + 32 * e + lane;
            const bool in = row < it.len;
            l[e] = in ? __ldg(from + row) : -INFINITY;           // (rows behind the sequence weigh nothing)
            d[e] = in ? __ldg(from + other + row) : 0.f;
          }
          const uint32_t s = n & 1u;
          if (n >= 2) ok = warp_wait(st_free + 8u * s, (n / 2 - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          float* to = stats + s * 2 * kBlock;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            to[32 * e + lane] = l[e];
            to[kBlock + 32 * e + lane] = d[e];
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(st_full + 8u * s);
        }
      }
    } else if (lane == 0) {
      // ---- dq's sums: taken to scratch in turn, and for tile 0 fetched from there ------------------
      // A place is filled by the dq warps (staged) and sent, or filled from scratch (sums_in) and read by them (staged); either way
      // stage_free ends the use, here, before the next one begins: nobody is ever two uses ahead of anybody.
      uint32_t m = 0, read = 0;                                  // places used so far; bit s: place s was last read by the dq warps
      bool ok = true;
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const BwdItem it = bwd_item(p, i);
        for (int t = 0; t < it.steps && ok; ++t) {
          int head, block;
          bwd_step(p, it, t, head, block);
          if (block == 0) continue;                              // tile 0's own block: no sums
          unsigned* turn = p.counters + static_cast<long long>(head) * p.cap + it.slot + block;
          const int rows = min(kBlock, it.len - block * kBlock);
          float* to = p.sums + (static_cast<long long>(head) * p.total + it.begin + block * kBlock) * HD;
          const uint32_t bytes = static_cast<uint32_t>(rows) * Sh::kPart * 4u;
          const unsigned before = static_cast<unsigned>(block - it.tile);      // tiles whose parts are in
          for (int part = 0; part < Sh::kParts && ok; ++part, ++m) {
            const uint32_t s = m % Sh::kStages, use = m / Sh::kStages, at = stage_at + s * Sh::kStage;
            // parts lie one after the other: [part][rows of the block][kPart]
            float* dst = to + static_cast<long long>(part) * rows * Sh::kPart;
            if ((read >> s) & 1u) {
              ok = mbar_wait(staged + 8u * s, (use - 1) & 1u, abort_flag, p.limit);
              if (ok) mbar_arrive(stage_free + 8u * s);
            }
            if (ok && it.tile != 0) ok = mbar_wait(staged + 8u * s, use & 1u, abort_flag, p.limit);
            if (ok && part == 0 && before > 0) ok = wait_turn(turn, before, abort_flag, p.limit);
            if (!ok) break;
            asm volatile("fence.proxy.async.global;" ::: "memory");
            if (it.tile == 0) {
              read |= 1u << s;
              mbar_expect_tx(sums_in + 8u * s, bytes);
              asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(at), "l"(dst),
                           "r"(bytes), "r"(sums_in + 8u * s)
                           : "memory");
            } else {
              read &= ~(1u << s);
              if (before == 0)
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(at), "r"(bytes) : "memory");
              else
                asm volatile("cp.reduce.async.bulk.global.shared::cta.bulk_group.add.f32 [%0], [%1], %2;" ::"l"(dst), "r"(at), "r"(bytes) : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
              mbar_arrive(stage_free + 8u * s);
            }
          }
          if (ok && it.tile != 0) {
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            asm volatile("fence.acq_rel.gpu;" ::: "memory");
            asm volatile("red.relaxed.gpu.global.add.u32 [%0], 1;" ::"l"(turn) : "memory");
          }
        }
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      // (what was fetched and not waited for by its readers, after an abort)
      volatile unsigned ignore = 0u;
      if (*abort_flag)
        for (uint32_t s = 0; s < Sh::kStages; ++s)
          for (uint32_t ph = 0; ph < 2; ++ph) mbar_wait(sums_in + 8u * s, ph, &ignore, 1000000);
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOut));
    // ---- dq out of tensor memory: a thread has a query's row -----------------------------------------
    const int r = (warp & 3) * 32 + lane;
    const uint32_t at_t = tmem + Sh::kDq + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    uint32_t n = 0, m = 0;
    uint32_t fetched = 0;                                        // bit s: parity of the fetches into place s
    bool ok = true;
    for (int i = blockIdx.x; i < items; i += gridDim.x) {
      const BwdItem it = bwd_item(p, i);
      for (int t = 0; t < it.steps; ++t, ++n) {
        int head, block;
        bwd_step(p, it, t, head, block);
        const int row = block * kBlock + r;
        const bool live = row < it.len, last = it.tile == 0, alone = block == 0;
        const uint32_t sw = static_cast<uint32_t>(r) & (Sh::kPart / 4 - 1);
        ok = ok && warp_wait(dq_full, n & 1u, abort_flag, p.limit);
        tc_fence_after();
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.dq.p) + (it.begin + row) * p.dq.row + head * p.dq.head;
#pragma unroll
        for (int part = 0; part < Sh::kParts; ++part) {
          uint32_t v[Sh::kPart];
          if (ok) {
#pragma unroll
            for (int c = 0; c < Sh::kPart; c += 32) tmem_load32(at_t + part * Sh::kPart + c, v + c);
#pragma unroll
            for (int c = 0; c < Sh::kPart; c += 32) tmem_loaded(v + c);
          }
          if (part == Sh::kParts - 1 && ok) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(dq_read);
          }
          const uint32_t s = m % Sh::kStages, mine = stage_at + s * Sh::kStage + static_cast<uint32_t>(r) * (Sh::kPart * 4u);
          if (!last) {
            const uint32_t use = m / Sh::kStages;
            if (ok && use > 0) ok = warp_wait(stage_free + 8u * s, (use - 1) & 1u, abort_flag, p.limit);
            if (ok) {
#pragma unroll
              for (uint32_t c = 0; c < Sh::kPart / 4; ++c)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mine + ((c ^ sw) << 4)), "r"(v[4 * c]), "r"(v[4 * c + 1]),
                             "r"(v[4 * c + 2]), "r"(v[4 * c + 3])
                             : "memory");
              fence_async_smem();
              __syncwarp();
              if (lane == 0) mbar_arrive(staged + 8u * s);
            }
          } else {
            if (!alone && ok) {
              ok = warp_wait(sums_in + 8u * s, (fetched >> s) & 1u, abort_flag, p.limit);
              fetched ^= 1u << s;
              if (ok) {
#pragma unroll
                for (uint32_t c = 0; c < Sh::kPart / 4; ++c) {
                  const uint4 x = lds128(mine + ((c ^ sw) << 4));
                  v[4 * c] = __float_as_uint(__uint_as_float(v[4 * c]) + __uint_as_float(x.x));
                  v[4 * c + 1] = __float_as_uint(__uint_as_float(v[4 * c + 1]) + __uint_as_float(x.y));
                  v[4 * c + 2] = __float_as_uint(__uint_as_float(v[4 * c + 2]) + __uint_as_float(x.z));
                  v[4 * c + 3] = __float_as_uint(__uint_as_float(v[4 * c + 3]) + __uint_as_float(x.w));
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(staged + 8u * s);
              }
            }
#pragma unroll
            for (int c = 0; c < Sh::kPart; c += 8) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                w[k] = ok ? bf16_pair(__uint_as_float(v[c + 2 * k]) * p.scale, __uint_as_float(v[c + 2 * k + 1]) * p.scale) : 0x7fc07fc0u;
              if (live && part * Sh::kPart + c < p.hd) *reinterpret_cast<uint4*>(out + part * Sh::kPart + c) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
          if (!alone) ++m;
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    // ---- softmax: a thread has a key's row and 64 of a block's queries ---------------------------------
    const int half = (warp - 8) >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + Sh::kS + 64u * half + lanes, dp_at = tmem + Sh::kDp + 64u * half + lanes;
    const uint32_t ds_row = ds_at + static_cast<uint32_t>(half) * (kBlock * 128u) + static_cast<uint32_t>(r) * 128u, sw = static_cast<uint32_t>(r) & 7u;
    const uint64_t by2 = pack2f(p.by, p.by);
    uint32_t n = 0, tiles = 0;
    bool ok = true;
    for (int i = blockIdx.x; i < items; i += gridDim.x, ++tiles) {
      const BwdItem it = bwd_item(p, i);
      for (int t = 0; t < it.steps && ok; ++t, ++n) {
        const bool diagonal = t % it.blocks == 0;
        const uint32_t st = n & 1u;
        const float4* lse = reinterpret_cast<const float4*>(stats + st * 2 * kBlock + 64 * half);
        ok = warp_wait(st_full + 8u * st, (n / 2) & 1u, abort_flag, p.limit) && warp_wait(s_full, n & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        uint64_t w[32];                                          // P', in pairs of queries
        {
          uint32_t s[64];
          tmem_load32(s_at, s);
          tmem_load32(s_at + 32, s + 32);
          tmem_loaded(s);
          tmem_loaded(s + 32);
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const float4 l = lse[c / 4];
            const float2 a = unpack2f(fma2f(pack2f(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), by2, pack2f(l.x, l.y)));
            const float2 b = unpack2f(fma2f(pack2f(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), by2, pack2f(l.z, l.w)));
            w[c / 2] = pack2f(exp2_approx(a.x), exp2_approx(a.y));
            w[c / 2 + 1] = pack2f(exp2_approx(b.x), exp2_approx(b.y));
          }
        }
        if (diagonal) {
          const int from = r - 64 * half;                        // queries before the key see nothing of it
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const float2 x = unpack2f(w[c]);
            w[c] = pack2f(2 * c < from ? 0.f : x.x, 2 * c + 1 < from ? 0.f : x.y);
          }
        }
        {
          uint32_t b[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const float2 x = unpack2f(w[c]);
            b[c] = bf16_pair(x.x, x.y);
          }
          tmem_store32(s_at, b);
        }
        tmem_stored();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
        ok = warp_wait(dp_full, n & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        const float4* delta = lse + kBlock / 4;
#pragma unroll
        for (int h = 0; h < 64; h += 32) {
          uint32_t d[32];
          tmem_load32(dp_at + h, d);
          tmem_loaded(d);
#pragma unroll
          for (int c = 0; c < 32; c += 8) {
            uint32_t b[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float4 e = delta[(h + c) / 4 + k];
              const int q = (h + c) / 2 + 2 * k;
              float2 x = unpack2f(mul2f(w[q], add2f(pack2f(__uint_as_float(d[c + 4 * k]), __uint_as_float(d[c + 4 * k + 1])), pack2f(e.x, e.y))));
              float2 y = unpack2f(mul2f(w[q + 1], add2f(pack2f(__uint_as_float(d[c + 4 * k + 2]), __uint_as_float(d[c + 4 * k + 3])), pack2f(e.z, e.w))));
              if (diagonal) {                                    // (zero whatever dP' is there)
                const int from = r - 64 * half - (h + c + 4 * k);
                x = make_float2(0 < from ? 0.f : x.x, 1 < from ? 0.f : x.y);
                y = make_float2(2 < from ? 0.f : y.x, 3 < from ? 0.f : y.y);
              }
              b[2 * k] = bf16_pair(x.x, x.y);
              b[2 * k + 1] = bf16_pair(y.x, y.y);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(ds_row + ((static_cast<uint32_t>((h + c) / 8) ^ sw) << 4)), "r"(b[0]),
                         "r"(b[1]), "r"(b[2]), "r"(b[3])
                         : "memory");
          }
        }
        tc_fence_before();
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(ds_full);
          mbar_arrive(st_free + 8u * st);
        }
      }
      // the tile's results: one half of the warps has dv, the other dk
      ok = ok && warp_wait(acc_full, tiles & 1u, abort_flag, p.limit);
      tc_fence_after();
      const int row = it.tile * kBlock + r;
      const bool live = row < it.len;
      const AttnOut& to = half == 0 ? p.dv : p.dk;
      const float by = half == 0 ? 1.f : p.scale;
      const uint32_t acc = tmem + (half == 0 ? Sh::kDv : Sh::kDk) + lanes;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(to.p) + (it.begin + row) * to.row + it.kv * to.head;
#pragma unroll
      for (int c = 0; c < HD; c += 32) {
        uint32_t v[32];
        if (ok) {
          tmem_load32(acc + c, v);
          tmem_loaded(v);
        }
        if (c + 32 >= HD && ok) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(acc_free);
        }
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          uint32_t x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[k] = ok ? bf16_pair(__uint_as_float(v[e + 2 * k]) * by, __uint_as_float(v[e + 2 * k + 1]) * by) : 0x7fc07fc0u;
          if (live && c + e < p.hd) *reinterpret_cast<uint4*>(out + c + e) = make_uint4(x[0], x[1], x[2], x[3]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
}

// -lse log2 e and -delta of every row and head, and the counters' start: `lanes` threads a row and head, 16 bytes each.
__global__ void __launch_bounds__(256)
attn_backward_start_kernel(const AttnBackward a, float* stats, unsigned* counters, long long n_counters, int lanes) {
  pdl_wait();
  const long long id = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, w = id / lanes;
  if (id < n_counters) counters[id] = 0u;
  for (long long c = id + static_cast<long long>(gridDim.x) * 256; c < n_counters; c += static_cast<long long>(gridDim.x) * 256) counters[c] = 0u;
  const int c = static_cast<int>(id - w * lanes) * 8;
  const long long rows = static_cast<long long>(a.total) * a.hq;
  const long long row = w / a.hq, head = w - row * a.hq;
  float s = 0.f;
  if (w < rows && c < a.hd) {
    float x[8], y[8];
    Vec<__nv_bfloat16>::unpack(__ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.dout.p) + row * a.dout.row + head * a.dout.head + c)), x);
    Vec<__nv_bfloat16>::unpack(__ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.o.p) + row * a.o.row + head * a.o.head + c)), y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  }
  for (int off = lanes / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  if (w < rows && c == 0) {
    stats[head * a.total + row] = -a.lse[head * a.total + row] * kLog2eB;
    stats[rows + head * a.total + row] = -s;
  }
}

template <int HD>
int run_backward_tc(abs_ctx* ctx, const AttnBackward& a, cudaStream_t st) {
  typedef BwdShape<HD> Sh;
  BwdMaps maps;
  if (!encode_heads_map(a.q, a.total, a.hq, a.hd, &maps.q) || !encode_heads_map(a.k, a.total, a.hk, a.hd, &maps.k) ||
      !encode_heads_map(a.v, a.total, a.hk, a.hd, &maps.v) || !encode_heads_map(a.dout, a.total, a.hq, a.hd, &maps.dout))
    return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled (%d rows, head_dim %d) failed", a.total, a.hd);
  const AttnPlanLayout l = attn_plan_layout(a.n, a.total);
  const AttnScratch s = attn_scratch(a.total, a.hq, a.hd, a.n);
  char* mem = static_cast<char*>(a.scratch);
  auto kern = attn_backward_kernel<HD>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, Sh::kSmem));
  // the softmax warps' registers come out of what the launch has: with fewer than 128 a thread they would never get them
  static const int regs = [&] {
    cudaFuncAttributes fa;
    return cudaFuncGetAttributes(&fa, kern) == cudaSuccess ? fa.numRegs : 0;
  }();
  if (regs != 128) return set_error(ctx, ABS_ERR_CUDA, "the backward kernel was built with %d registers a thread, not 128", regs);
  const long long counters = static_cast<long long>(a.hq) * l.bwd_cap;
  const int lanes = HD / 8;
  const long long threads = static_cast<long long>(a.total) * a.hq * lanes;
  ABS_CUDA_TRY(ctx, launch_dependent(attn_backward_start_kernel, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, st, a,
                                     reinterpret_cast<float*>(mem + s.delta), reinterpret_cast<unsigned*>(mem + s.counters), counters, lanes));
  // heads whose sums of dq are under way at a time: 48 MB of them
  const long long group = a.hq / a.hk, rows = a.total < (1 << kAttnGroupBits) ? a.total : 1 << kAttnGroupBits;
  long long heads = (48ll << 20) / (rows * group * HD * 4);
  heads = heads < 1 ? 1 : heads > a.hk ? a.hk : heads;
  const BwdParams p{a.dq, a.dk, a.dv, reinterpret_cast<float*>(mem + s.delta), reinterpret_cast<float*>(mem + s.sums),
                    reinterpret_cast<unsigned*>(mem + s.counters), a.plan, a.plan + l.bwd, a.plan + l.groups, a.total, a.hq, a.hk,
                    static_cast<int>(group), a.hd, l.bwd_cap, static_cast<int>(heads), a.scale * kLog2eB, a.scale,
                    ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles,
                    ctx->tuning.stats_fault_drop_loads ? 1 : 0};
  const long long most = static_cast<long long>(l.bwd_cap) * a.hk;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(most < ctx->sm_count ? most : ctx->sm_count));
  cfg.blockDim = dim3(kThreadsB);
  cfg.dynamicSmemBytes = Sh::kSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ABS_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, kern, maps, p));
  return ABS_OK;
}

}  // namespace

int launch_attention_tc_backward(abs_ctx* ctx, const AttnBackward& a, cudaStream_t st) {
  if (encode_tiled_fn() == nullptr) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  return a.hd <= 64 ? run_backward_tc<64>(ctx, a, st) : run_backward_tc<128>(ctx, a, st);
}

}  // namespace absk
