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
// dQ is a sum over key tiles, which different CTAs have.  They add to fp32 sums in scratch (bulk reductions in L2), for each block of
// queries in a fixed order, so results repeat bit for bit: tile j of a sequence starts at query block j and goes up, so block i is
// reached first by tile i, then by i - 1, and so on, each a step later than the one before; a counter says whose turn
// it is, and the wait is rarely one.  The first of them stores instead of adding (nothing is cleared), and the last, tile 0, adds its own part
// to the sums and writes dq: sequences of up to 128 rows never touch the sums.  Tiles are worked off shortest first
// (attn_plan_kernel), each for all heads before the next: a tile's predecessors in the order of the sums are then far ahead.  (Some
// heads at a time, so that the sums under way stay in L2, costs more in waits than it saves: 32768 tokens, 8 heads of 128, 1 at a
// time 11.7 ms, all 7.5; 16 x 2048, 12 heads of 64, 1, 2, 4, 12: 1263, 793, 568, 550 us.)
// The grid is resident (a cooperative launch) and CTAs take the tiles in that order as they are free, in which each comes after those that it
// waits for, so the first unfinished tile of all never waits.
//
// Rounded to fewer bits than 32: P and dS to bf16, as operands of the tensor core, and the results.
//
// At 64 columns a head the softmax warps are busiest (1024 clocks of exponentials per 128 x 128 scores and as many of everything else, while
// five products take 1280), and a block's steps depend on one another: 128 of 1024 tokens, 12 heads of 64, 1.38 to 1.45 ms, 355 to
// 375 TFLOP/s; 65536 tokens in one 560.  At 128 columns five products take 2560 clocks and the sums of dq, 64 KB a block to L2, about
// as long: 32768 tokens, 8 heads, 735 TFLOP/s, 32 of 2048, 16 heads, 540; that kernel spills (264 bytes of stores and 376 of loads a thread,
// most likely the 64 weights that a softmax thread holds beside as many scores; at 64 columns 8 and 16).  Heads of other widths cost what 64
// and 128 do: 4 of 4096 tokens, 8 heads and 2 of keys, 32, 64, 80, 96 and 128 columns 330, 341, 561, 573, 598 us.
//
// Roles of the 16 warps: 0 takes tiles and loads (TMA), 1 issues the products, 2 and 3 look after the sums, 4-7 take results out of tensor memory,
// 8-15 are the softmax: 64 of a block's 128 queries each half.  While they compute P' of a block, dQ and dK of the block before and
// dP' of this one run; while they compute dS', dV and the next S'.  All waits are bounded: one that runs out raises the CTA's
// abort flag, every role falls through, copies in flight are waited for, tensor memory is freed, and what was not finished is NaN.
#include "abs_attention.cuh"
#include "abs_tc.cuh"

namespace absk {
namespace {

constexpr int kThreadsB = 512;
constexpr uint32_t kItems = 4;                // tiles of a CTA that are known ahead of time
constexpr int kBlock = 128;                   // keys of a tile, queries of a block
constexpr float kLog2eB = 1.4426950408889634f;

template <int HD> struct BwdShape {
  static constexpr uint32_t kRows = kBlock * HD * 2;              // 128 rows of one head, bf16
  static constexpr uint32_t kKv = HD == 64 ? 2 : 1;               // places for a tile's K and V
  static constexpr uint32_t kQ = 2, kDo = HD == 64 ? 2 : 1;       // places for Q and dO
  static constexpr uint32_t kDs = kBlock * kBlock * 2;
  static constexpr uint32_t kHalves = HD / 64;                    // dq leaves in pieces of 64 columns
  static constexpr uint32_t kStage = kBlock * 64 * 4, kStages = HD == 64 ? 2 : 1;      // places for these
  static constexpr uint32_t kStats = 2 * kBlock * 4;              // -lse and -delta of a block
  static constexpr uint32_t kData = 2 * kKv * kRows + (kQ + kDo) * kRows + kDs + kStages * kStage + 2 * kStats;
  static constexpr size_t kSmem = kData + 512;
  // registers of a thread of warps 0-3, of dq's and of the softmax; together what 128 a thread are at the launch
  static constexpr int kRegsLoad = HD == 64 ? 88 : 72, kRegsOut = HD == 64 ? 120 : 168, kRegsSoft = HD == 64 ? 152 : 136;
  static_assert(128 * (kRegsLoad + kRegsOut + 2 * kRegsSoft) == kThreadsB * 128, "");
  // tensor memory: S' (P' over it), dP', dV, dK, dQ (128 columns a head: over dP')
  static constexpr uint32_t kS = 0, kDp = 128, kDv = 256, kDk = 256 + HD, kDq = HD == 64 ? 384 : kDp, kDqs = HD == 64 ? 2 : 1;      // (two of dQ)
};
static_assert(BwdShape<64>::kSmem <= 232448 && BwdShape<128>::kSmem <= 232448, "");

struct BwdMaps {
  CUtensorMap q, k, v, dout;
};
struct BwdParams {
  AttnOut dq, dk, dv;
  const float* stats;                         // [2][hq][total]
  float* sums;                                // [hq][total][HD]; of a block: [HD / 64][16][rows] pieces of 16 bytes
  unsigned* counters;                         // [hq][cap][HD / 64], then the next tile that nobody has
  const int* plan;
  const int* tiles;
  int n, total, hq, hk, parts, hd, cap;
  // A key head's group of query heads in `parts` of `group` heads, each a head of its own in the list of tiles, `heads` in all.
  int heads, group;
  float* partial;                             // [parts][dv, dk][hk][total][HD], laid out as sums; NULL: parts = 1
  float by, scale;                            // scale log2 e, scale
  long long limit;
  int drop_loads;                             // test hooks, as the forward pass's; steps of blocks here
  uint32_t stop_after;
  bool sectors;                               // whether dq, dk and dv are rows of whole sectors of 32 bytes
};
struct BwdItem {
  int begin, len, slot, tile, head;           // head: of the list of tiles
  int blocks, steps;                          // query blocks from the tile on, and of all the group's heads
};
// Tile i of the list: all heads of a tile come after one another.
__device__ __forceinline__ BwdItem bwd_item(const BwdParams& p, int i) {
  const int at = i / p.heads;
  const int4 r = __ldg(reinterpret_cast<const int4*>(p.tiles) + at);
  BwdItem it;
  it.head = i - at * p.heads;
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
  head = it.head * p.group + h;
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
  }
}

template <int HD>
__global__ void __launch_bounds__(kThreadsB, 1)
attn_backward_kernel(const __grid_constant__ BwdMaps maps, const __grid_constant__ BwdParams p) {
  typedef BwdShape<HD> Sh;
  constexpr uint32_t kRows = Sh::kRows;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];       // (there is no room to align it here; checked below)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t kv_at = smem_u32(smem_dyn), q_at = kv_at + 2u * Sh::kKv * kRows,
                 do_at = q_at + Sh::kQ * kRows, ds_at = do_at + Sh::kDo * kRows, stage_at = ds_at + Sh::kDs,
                 stats_at = stage_at + Sh::kStages * Sh::kStage;
  float* stats = reinterpret_cast<float*>(smem_dyn + (stats_at - kv_at));
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem_dyn + Sh::kData);
  constexpr int kBars = 44;
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + kBars);
  unsigned *tmem_slot = const_cast<unsigned*>(abort_flag) + 1, *untold = tmem_slot + 1;    // untold: a tile that was taken when a wait ran out
  int4* ring = reinterpret_cast<int4*>(bars + kBars + 2);          // four items of two pieces of 16 bytes
  const uint32_t b0 = smem_u32(bars);
  // two of each of the first ones (where one is waited for by several who may be a step apart, steps alternate between the two: with a
  // single one it could be two phases on when the slower looks, which looks like none)
  const uint32_t kv_full = b0, kv_free = b0 + 16u, q_full = b0 + 32u, q_free = b0 + 48u, do_full = b0 + 64u, do_free = b0 + 80u,
                 st_full = b0 + 96u, st_free = b0 + 112u, turn_ok = b0 + 128u, staged = b0 + 144u, stage_free = b0 + 160u, dq_full = b0 + 176u,
                 dq_read = b0 + 192u, item_full = b0 + 208u, item_free = b0 + 240u, s_full = b0 + 272u, p_full = b0 + 280u, dp_full = b0 + 288u,
                 ds_full = b0 + 296u, acc_full = b0 + 304u, dv_free = b0 + 312u, dk_free = b0 + 320u, landed = b0 + 328u,
                 done_bar = b0 + 336u, dv_full = b0 + 344u;
  if (threadIdx.x == 0) {
    for (uint32_t k = 0; k < 2; ++k) {
      mbar_init(kv_full + 8u * k, 1);
      mbar_init(kv_free + 8u * k, 1);
      mbar_init(q_full + 8u * k, 1);
      mbar_init(q_free + 8u * k, 1);
      mbar_init(do_full + 8u * k, 1);
      mbar_init(do_free + 8u * k, 1);
      mbar_init(st_full + 8u * k, 32);
      mbar_init(st_free + 8u * k, 8);
      mbar_init(turn_ok + 8u * k, 1);
      mbar_init(staged + 8u * k, 4);
      mbar_init(stage_free + 8u * k, 1);
      mbar_init(dq_full + 8u * k, 1);
      mbar_init(dq_read + 8u * k, 4);
    }
    for (uint32_t k = 0; k < kItems; ++k) {
      mbar_init(item_full + 8u * k, 1);
      mbar_init(item_free + 8u * k, 15);                           // products, two of sums, four of dq, eight of the softmax
    }
    mbar_init(s_full, 1);
    mbar_init(p_full, 8);
    mbar_init(dp_full, 1);
    mbar_init(ds_full, 8);
    mbar_init(acc_full, 1);
    mbar_init(dv_full, 1);
    mbar_init(dv_free, 4);
    mbar_init(dk_free, 4);
    mbar_init(landed, 1);
    mbar_init(done_bar, 1);
    *abort_flag = (kv_at & 1023u) ? 1u : 0u;
    *untold = ~0u;
    for (uint32_t k = 0; k < 2 * kItems; ++k) ring[k] = make_int4(0, 0, 0, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_all(smem_u32(tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int items = plan_fits(p.plan, p.n, p.total) ? __ldg(p.plan + kPlanBwdTiles) * p.heads : 0;
  unsigned* next_item = p.counters + static_cast<long long>(p.hq) * p.cap * Sh::kHalves;
  // The CTA's k-th tile; false: there is none (or a wait ran out).  last: whether this role is done with the place in the ring.
  auto read_item = [&](uint32_t k) {
    const int4 a = ring[2 * (k % kItems)], b = ring[2 * (k % kItems) + 1];
    return BwdItem{a.x, a.y, a.z, a.w, b.x, b.y, b.z};
  };
  auto take_item = [&](uint32_t k, BwdItem& it) {
    if (!warp_wait(item_full + 8u * (k % kItems), (k / kItems) & 1u, abort_flag, p.limit)) return false;
    it = read_item(k);
    __syncwarp();
    if (lane == 0) mbar_arrive(item_free + 8u * (k % kItems));
    return it.steps > 0;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kRegsLoad));
    if (warp == 0) {
      // ---- loads -----------------------------------------------------------------------------------
      uint32_t lands = 0, tiles = 0, n = 0, fills_q = 0, fills_do = 0, fills_st = 0;       // tiles and steps so far, and places filled
      bool ok = !p.drop_loads && *abort_flag == 0u;
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
      auto zero_behind = [&](const CUtensorMap* map, uint32_t to, const BwdItem& it, int head, int first) {
        expect(landed, kRows);
        copy(map, to, head, it.begin + first, landed);
        ok = warp_arrival(landed, lands & 1u, abort_flag, p.limit);
        ++lands;
        if (!ok) return;
        for (uint32_t c = 0; c < HD / 64; ++c)
          for (uint32_t e = static_cast<uint32_t>(it.len - first) * 128u + lane * 16u; e < kBlock * 128u; e += 512u)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + c * (kBlock * 128u) + e), "r"(0u) : "memory");
        fence_async_smem();
        __syncwarp();
      };
      auto copy_rows = [&](const CUtensorMap* map, uint32_t to, const BwdItem& it, int head, int first, uint32_t bar) {
        if (it.len - first >= kBlock) {
          expect(bar, kRows);
          copy(map, to, head, it.begin + first, bar);
        } else {
          zero_behind(map, to, it, head, first);
          if (ok && lane == 0) mbar_arrive(bar);
        }
      };
      // Tiles are taken in order by whoever is free, one ahead of the one whose rows are being fetched; after the last comes one without
      // steps.
      // (taking one is a way to L2 and back, which is under way while the next copies are issued)
      uint32_t told = 0;
      unsigned taken = 0;
      bool has_taken = false;
      auto take = [&]() {
        if (lane == 0) taken = atomicAdd(next_item, 1u);
        has_taken = true;
      };
      auto tell = [&]() {
        if (told >= kItems) ok = ok && warp_wait(item_free + 8u * (told % kItems), (told / kItems - 1) & 1u, abort_flag, p.limit);
        if (!ok) return;
        const unsigned i = __shfl_sync(0xffffffffu, taken, 0);
        BwdItem next = {};
        if (i < static_cast<unsigned>(items)) next = bwd_item(p, static_cast<int>(i));
        if (lane == 0) {
          ring[2 * (told % kItems)] = make_int4(next.begin, next.len, next.slot, next.tile);
          ring[2 * (told % kItems) + 1] = make_int4(next.head, next.blocks, next.steps, 0);
          mbar_arrive(item_full + 8u * (told % kItems));
        }
        __syncwarp();
        ++told;
        has_taken = false;
      };
      // -lse and -delta of a block's queries; zeros behind the sequence, where Q and dO are zeros and what the weights are changes nothing
      auto copy_stats = [&](const BwdItem& it, int head, int block) {
        const uint32_t s = n & 1u, to = stats_at + s * Sh::kStats + lane * 4u;
        if (n >= 2) ok = warp_wait(st_free + 8u * s, (n / 2 - 1) & 1u, abort_flag, p.limit);
        if (!ok) return;
        const float* from = p.stats + static_cast<long long>(head) * p.total + it.begin;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = block * kBlock + 32 * (e & 3) + lane;
          const float* at = from + (row < it.len ? row : 0) + (e < 4 ? 0ll : static_cast<long long>(p.hq) * p.total);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 128u * e), "l"(at), "r"(row < it.len ? 4 : 0) : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(st_full + 8u * s) : "memory");
        ++fills_st;
      };
      take();
      if (ok) tell();
      while (ok) {
        const BwdItem it = read_item(tiles);
        if (it.steps == 0) break;
        const uint32_t kv = tiles % Sh::kKv, kvs = kv_at + kv * 2u * kRows;
        if (tiles >= Sh::kKv) ok = warp_wait(kv_free + 8u * kv, (tiles / Sh::kKv - 1) & 1u, abort_flag, p.limit);
        if (!ok) break;
        const int kv_head = it.head / p.parts;
        // (two copies of a full tile arrive as one; V's zeros make dP' of rows behind the sequence zero, so that p = 0 times it is)
        if (it.len - it.tile * kBlock >= kBlock) {
          expect(kv_full + 8u * kv, 2u * kRows);
          copy(&maps.k, kvs, kv_head, it.begin + it.tile * kBlock, kv_full + 8u * kv);
          copy(&maps.v, kvs + kRows, kv_head, it.begin + it.tile * kBlock, kv_full + 8u * kv);
        } else {
          zero_behind(&maps.v, kvs + kRows, it, kv_head, it.tile * kBlock);
          if (ok) copy_rows(&maps.k, kvs, it, kv_head, it.tile * kBlock, kv_full + 8u * kv);
        }
        if (!ok) break;
        ++tiles;
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          int head, block;
          bwd_step(p, it, t, head, block);
          const uint32_t qs = n % Sh::kQ, ds = n % Sh::kDo;
          if (n >= p.stop_after && (blockIdx.x & 1u) == 0u) ok = false;
          if (ok && n >= Sh::kQ) ok = warp_wait(q_free + 8u * qs, (n / Sh::kQ - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          copy_rows(&maps.q, q_at + qs * kRows, it, head, block * kBlock, q_full + 8u * qs);
          if (!ok) break;
          ++fills_q;
          copy_stats(it, head, block);
          if (ok && n >= Sh::kDo) ok = warp_wait(do_free + 8u * ds, (n / Sh::kDo - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          copy_rows(&maps.dout, do_at + ds * kRows, it, head, block * kBlock, do_full + 8u * ds);
          if (!ok) break;
          ++fills_do;
          if (t == 0) take();
          if (ok && (t == 1 || it.steps == 1)) tell();
        }
      }
      if (has_taken && lane == 0) *untold = taken;
      asm volatile("cp.async.wait_all;" ::: "memory");
      // Waits (bounded) until every copy that was issued has arrived, whatever made the other roles stop.
      for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t f_kv = k < Sh::kKv ? tiles / Sh::kKv + (k < tiles % Sh::kKv ? 1u : 0u) : 0u;
        const uint32_t f_q = fills_q / Sh::kQ + (k < fills_q % Sh::kQ ? 1u : 0u);
        const uint32_t f_do = k < Sh::kDo ? fills_do / Sh::kDo + (k < fills_do % Sh::kDo ? 1u : 0u) : 0u;
        if (f_kv > 0) warp_arrival(kv_full + 8u * k, (f_kv - 1) & 1u, abort_flag, p.limit);
        if (f_q > 0) warp_arrival(q_full + 8u * k, (f_q - 1) & 1u, abort_flag, p.limit);
        const uint32_t f_st = fills_st / 2 + (k < fills_st % 2 ? 1u : 0u);
        if (f_do > 0) warp_arrival(do_full + 8u * k, (f_do - 1) & 1u, abort_flag, p.limit);
        if (f_st > 0) warp_arrival(st_full + 8u * k, (f_st - 1) & 1u, abort_flag, p.limit);
      }
      if (lands > 0) warp_arrival(landed, (lands - 1) & 1u, abort_flag, p.limit);
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
      // dK and dQ of step m (counted over all tiles) from its dS'
      auto key_gradient = [&](uint32_t m, bool first) {
        if (elect_lane()) {
          const uint32_t d = desc_at(ds_at), q = desc_at(q_at + (m % Sh::kQ) * kRows);
#pragma unroll
          for (uint32_t k = 0; k < kBlock / 16; ++k) {
            const uint32_t off = (k / 4) * (kBlock * 128u / 16u) + (k % 4) * 2u;
            mma_ss(tmem + Sh::kDk, kDescK | (d + off), mn | (q + 128u * k), idesc_k, (!first || k > 0) ? 1u : 0u);
          }
          mma_commit(q_free + 8u * (m % Sh::kQ));
        }
        __syncwarp();
      };
      auto query_gradient = [&](uint32_t m, uint32_t kvs) {
        if (elect_lane()) {
          const uint32_t d = desc_at(ds_at), k_ = desc_at(kvs), to = tmem + Sh::kDq + (m % Sh::kDqs) * 64u;
#pragma unroll
          for (uint32_t k = 0; k < kBlock / 16; ++k) mma_ss(to, mn | (d + 128u * k), mn | (k_ + 128u * k), idesc_q, k > 0);
          mma_commit(dq_full + 8u * (m & 1u));
        }
        __syncwarp();
      };
      // the first S' of the CTA's k-th tile, whose first step is the m-th
      auto first_scores = [&](uint32_t k, uint32_t m) {
        const uint32_t kv = k % Sh::kKv;
        ok = warp_wait(kv_full + 8u * kv, (k / Sh::kKv) & 1u, abort_flag, p.limit);
        ok = ok && warp_wait(q_full + 8u * (m % Sh::kQ), (m / Sh::kQ) & 1u, abort_flag, p.limit);
        if (!ok) return;
        tc_fence_after();
        scores(Sh::kS, kv_at + kv * 2u * kRows, q_at + (m % Sh::kQ) * kRows, s_full);
      };
      BwdItem it, following;
      bool more = take_item(0, it);
      if (more) first_scores(0, 0);
      while (ok && more) {
        const uint32_t kv = tiles % Sh::kKv, kvs = kv_at + kv * 2u * kRows;
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          // dQ and dK of the step before and this one's dP'.  At 128 columns dQ lies over dP' and is taken out, while dK runs, before dP' is
          // written; at 64 it has two places of its own.
          if (t > 0) {
            ok = warp_wait(ds_full, (n - 1) & 1u, abort_flag, p.limit);
            if (HD == 64 && n > 2) ok = ok && warp_wait(dq_read + 8u * ((n - 3) & 1u), ((n - 3) >> 1) & 1u, abort_flag, p.limit);
            if (!ok) break;
            tc_fence_after();
            query_gradient(n - 1, kvs);
            if (t == 1 && tiles > 0) ok = warp_wait(dk_free, (tiles - 1) & 1u, abort_flag, p.limit);
            if (!ok) break;
            tc_fence_after();
            key_gradient(n - 1, t == 1);
          }
          const uint32_t ds = n % Sh::kDo;
          ok = warp_wait(do_full + 8u * ds, (n / Sh::kDo) & 1u, abort_flag, p.limit);
          if (HD == 128 && n > 0) ok = ok && warp_wait(dq_read + 8u * ((n - 1) & 1u), ((n - 1) >> 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          tc_fence_after();
          scores(Sh::kDp, kvs + kRows, do_at + ds * kRows, dp_full);
          ok = warp_wait(p_full, n & 1u, abort_flag, p.limit);
          if (ok && t == 0 && tiles > 0) ok = warp_wait(dv_free, (tiles - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          tc_fence_after();
          if (elect_lane()) {
            const uint32_t d = desc_at(do_at + ds * kRows);
#pragma unroll
            for (uint32_t k = 0; k < kBlock / 16; ++k)       // P' of the first 64 queries lies at columns 0-31, of the others at 64-95
              mma_ts(tmem + Sh::kDv, tmem + Sh::kS + 64u * (k / 4) + 8u * (k % 4), mn | (d + 128u * k), idesc_k, (t > 0 || k > 0) ? 1u : 0u);
            mma_commit(do_free + 8u * ds);
            if (t + 1 == it.steps) mma_commit(dv_full);
          }
          __syncwarp();
          if (t + 1 < it.steps) {
            const uint32_t next = n + 1;
            ok = warp_wait(q_full + 8u * (next % Sh::kQ), (next / Sh::kQ) & 1u, abort_flag, p.limit);
            if (!ok) break;
            tc_fence_after();
            scores(Sh::kS, kvs, q_at + (next % Sh::kQ) * kRows, s_full);
          } else {                                               // (with places for two tiles' K and V the next tile's S' comes before this one's last dQ and dK)
            more = take_item(tiles + 1, following);
            if (Sh::kKv == 2 && more) first_scores(tiles + 1, n + 1);
          }
        }
        if (!ok) break;
        ok = warp_wait(ds_full, (n - 1) & 1u, abort_flag, p.limit);
        if (HD == 64 && n > 2) ok = ok && warp_wait(dq_read + 8u * ((n - 3) & 1u), ((n - 3) >> 1) & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        query_gradient(n - 1, kvs);
        if (it.steps == 1 && tiles > 0) ok = warp_wait(dk_free, (tiles - 1) & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        key_gradient(n - 1, it.steps == 1);
        if (elect_lane()) {
          mma_commit(acc_full);
          mma_commit(kv_free + 8u * kv);
        }
        __syncwarp();
        ++tiles;
        if (Sh::kKv == 1 && more) first_scores(tiles, n);
        it = following;
      }
      if (elect_lane()) mma_commit(done_bar);
      __syncwarp();
      volatile unsigned ignore = 0u;
      mbar_wait(done_bar, 0u, &ignore, p.limit);                 // no product in flight when tensor memory is freed
    } else if (lane == 0) {
      // ---- dq's sums: two threads, every other piece of 64 columns each, so that one's way to L2 and back is hidden behind the other's ---
      // A piece's place is filled by the dq warps (staged) and sent from here, or, for tile 0, it is their turn to read (turn_ok, then
      // staged); either way stage_free ends the use.
      const uint32_t h = static_cast<uint32_t>(warp) - 2u;
      uint32_t n = 0;
      bool ok = true;
      for (uint32_t k = 0; ok; ++k) {
        ok = mbar_wait(item_full + 8u * (k % kItems), (k / kItems) & 1u, abort_flag, p.limit);
        if (!ok) break;
        const BwdItem it = read_item(k);
        mbar_arrive(item_free + 8u * (k % kItems));
        if (it.steps == 0) break;
        for (int t = 0; t < it.steps && ok; ++t, ++n) {
          if (HD == 64 && (n & 1u) != h) continue;
          const uint32_t half = HD == 64 ? 0u : h, u = HD == 64 ? n : 2u * n + h, s = u % Sh::kStages;
          int head, block;
          bwd_step(p, it, t, head, block);
          const unsigned before = static_cast<unsigned>(block - it.tile);      // tiles whose parts are in
          unsigned* turn = p.counters + (static_cast<long long>(head) * p.cap + it.slot + block) * Sh::kHalves + half;
          if (before > 0) ok = wait_turn(turn, before, abort_flag, p.limit);
          if (ok && it.tile == 0) mbar_arrive(turn_ok + 8u * h);
          ok = ok && mbar_wait(staged + 8u * h, (u >> 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          if (it.tile != 0) {
            const int rows = min(kBlock, it.len - block * kBlock);
            float* to = p.sums + (static_cast<long long>(head) * p.total + it.begin + block * kBlock) * HD + half * rows * 64;
            const uint32_t bytes = static_cast<uint32_t>(rows) * 256u, from = stage_at + s * Sh::kStage;
            asm volatile("fence.proxy.async.global;" ::: "memory");
            if (before == 0)
              asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
            else
              asm volatile("cp.reduce.async.bulk.global.shared::cta.bulk_group.add.f32 [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            mbar_arrive(stage_free + 8u * s);
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            asm volatile("fence.acq_rel.gpu;" ::: "memory");
            asm volatile("red.relaxed.gpu.global.add.u32 [%0], 1;" ::"l"(turn) : "memory");
          } else {
            mbar_arrive(stage_free + 8u * s);
          }
        }
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
  } else if (warp < 8) {
    if constexpr (Sh::kRegsOut <= 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kRegsOut));
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kRegsOut));
    // ---- dq out of tensor memory and into the sums: a thread has a query's row -------
    const int sub = warp & 3, r = sub * 32 + lane;
    const uint32_t at_t = tmem + Sh::kDq + (static_cast<uint32_t>(sub * 32) << 16);
    uint32_t n = 0, reads = 0;                                   // bit h: parity of what helper h let this warp read
    bool ok = true;
    BwdItem it;
#pragma unroll 1
    for (uint32_t k = 0; take_item(k, it); ++k) {
      // the tile's dv before its last dq (it is complete while the softmax warps are on their last dS', and the next tile's waits for the
      // place: with both results last the first dV of a tile waited for a step's time), its dk after it
#pragma unroll 1
      for (int t = 0; t <= it.steps; ++t) {
        if (t + 1 >= it.steps) {
          const bool is_dk = t == it.steps;
          ok = ok && warp_wait(is_dk ? acc_full : dv_full, k & 1u, abort_flag, p.limit);
          tc_fence_after();
          const int row = it.tile * kBlock + r, rows = min(32, it.len - it.tile * kBlock - 32 * sub), kv = it.head / p.parts;
#pragma unroll 1
          for (int c0 = 0; c0 < HD; c0 += 32) {
            uint32_t v[32];
            if (ok) {
              tmem_load32(tmem + (is_dk ? Sh::kDk : Sh::kDv) + c0 + (static_cast<uint32_t>(sub * 32) << 16), v);
              tmem_loaded(v);
            } else {
#pragma unroll
              for (int c = 0; c < 32; ++c) v[c] = 0x7fc00000u;
            }
            if (c0 + 32 == HD && ok) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(is_dk ? dk_free : dv_free);
            }
            if (row < it.len && p.parts > 1) {
              float4* part = reinterpret_cast<float4*>(p.partial + ((static_cast<long long>((it.head - kv * p.parts) * 2 + is_dk) * p.hk + kv) * p.total +
                                                                    it.begin + it.tile * kBlock + 32 * sub) * HD) + static_cast<long long>(c0 / 4) * rows + lane;
    #pragma unroll
              for (int c = 0; c < 8; ++c)
                part[c * rows] = make_float4(__uint_as_float(v[4 * c]), __uint_as_float(v[4 * c + 1]), __uint_as_float(v[4 * c + 2]), __uint_as_float(v[4 * c + 3]));
            } else if (row < it.len) {
              const AttnOut to = is_dk ? p.dk : p.dv;
              store_row32(static_cast<__nv_bfloat16*>(to.p) + (it.begin + row) * to.row + kv * to.head + c0, v, is_dk ? p.scale : 1.f, true, p.hd - c0, p.sectors);
            }
          }
        }
        if (t == it.steps) break;
        int head, block;
        bwd_step(p, it, t, head, block);
        const int row = block * kBlock + r, rows = min(kBlock, it.len - block * kBlock);
        const bool live = row < it.len;
        ok = ok && warp_wait(dq_full + 8u * (n & 1u), (n >> 1) & 1u, abort_flag, p.limit);
        tc_fence_after();
        // all of it first: at 128 columns a head the next dP' waits for the place
        uint32_t v[HD];
        if (ok) {
#pragma unroll
          for (int c = 0; c < HD; c += 32) tmem_load32(at_t + (n % Sh::kDqs) * 64u + c, v + c);
#pragma unroll
          for (int c = 0; c < HD; c += 32) tmem_loaded(v + c);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(dq_read + 8u * (n & 1u));
        }
#pragma unroll
        for (uint32_t half = 0; half < Sh::kHalves; ++half) {
          const uint32_t u = Sh::kHalves * n + half, s = u % Sh::kStages;
          uint32_t* x = v + 64 * half;
          if (u >= Sh::kStages) ok = ok && warp_wait(stage_free + 8u * s, (u / Sh::kStages - 1) & 1u, abort_flag, p.limit);
          if (it.tile != 0) {
            if (ok && live) {
#pragma unroll
              for (int c = 0; c < 16; ++c)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage_at + s * Sh::kStage + static_cast<uint32_t>(c * rows + r) * 16u), "r"(x[4 * c]),
                             "r"(x[4 * c + 1]), "r"(x[4 * c + 2]), "r"(x[4 * c + 3])
                             : "memory");
            }
            fence_async_smem();
          } else {
            const uint32_t who = u & 1u;                           // of the two threads that look after the sums
            ok = ok && warp_wait(turn_ok + 8u * who, (reads >> who) & 1u, abort_flag, p.limit);
            reads ^= 1u << who;
            if (ok && live && block > 0) {
              const float4* sums = reinterpret_cast<const float4*>(p.sums + (static_cast<long long>(head) * p.total + it.begin + block * kBlock) * HD +
                                                                   half * rows * 64) + r;
#pragma unroll
              for (int h = 0; h < 16; h += 4) {
                float4 y[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) y[c] = __ldcg(sums + (h + c) * rows);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  x[4 * (h + c)] = __float_as_uint(__uint_as_float(x[4 * (h + c)]) + y[c].x);
                  x[4 * (h + c) + 1] = __float_as_uint(__uint_as_float(x[4 * (h + c) + 1]) + y[c].y);
                  x[4 * (h + c) + 2] = __float_as_uint(__uint_as_float(x[4 * (h + c) + 2]) + y[c].z);
                  x[4 * (h + c) + 3] = __float_as_uint(__uint_as_float(x[4 * (h + c) + 3]) + y[c].w);
                }
              }
            }
            if (live) {
              __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.dq.p) + (it.begin + row) * p.dq.row + head * p.dq.head;
#pragma unroll
              for (int c = 0; c < 64; c += 32) store_row32(out + 64 * half + c, x + c, p.scale, ok, p.hd - 64 * static_cast<int>(half) - c, p.sectors);
            }
          }
          __syncwarp();
          if (ok && lane == 0) mbar_arrive(staged + 8u * (u & 1u));
        }
        ++n;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kRegsSoft));
    // ---- softmax: a thread has a key's row and 64 of a block's queries ---------------------------------
    const int half = (warp - 8) >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + Sh::kS + 64u * half + lanes, dp_at = tmem + Sh::kDp + 64u * half + lanes;
    const uint32_t ds_row = ds_at + static_cast<uint32_t>(half) * (kBlock * 128u) + static_cast<uint32_t>(r) * 128u, sw = static_cast<uint32_t>(r) & 7u;
    const uint64_t by2 = pack2f(p.by, p.by);
    uint32_t n = 0, tiles = 0;
    bool ok = true;
    BwdItem it;
#pragma unroll 1
    for (; take_item(tiles, it); ++tiles) {
#pragma unroll 1
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
            // (all on their unit: a quarter of them on the FMA pipe, as the forward pass does, is 1 % slower here)
            w[c / 2] = exp2_pair(fma2f(pack2f(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), by2, pack2f(l.x, l.y)));
            w[c / 2 + 1] = exp2_pair(fma2f(pack2f(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), by2, pack2f(l.z, l.w)));
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
              const float2 x = unpack2f(mul2f(w[q], add2f(pack2f(__uint_as_float(d[c + 4 * k]), __uint_as_float(d[c + 4 * k + 1])), pack2f(e.x, e.y))));
              const float2 y = unpack2f(mul2f(w[q + 1], add2f(pack2f(__uint_as_float(d[c + 4 * k + 2]), __uint_as_float(d[c + 4 * k + 3])), pack2f(e.z, e.w))));
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
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
  if (*abort_flag) {                          // a wait ran out: NaN for what this CTA had taken and for what nobody has
    for (uint32_t k = 0;; ++k) {
      __syncthreads();
      if (warp == 0 && k >= kItems) {
        unsigned i = 0;
        if (lane == 0) i = k == kItems && *untold != ~0u ? *untold : atomicAdd(next_item, 1u);
        i = __shfl_sync(0xffffffffu, i, 0);
        BwdItem next = {};
        if (i < static_cast<unsigned>(items)) next = bwd_item(p, static_cast<int>(i));
        if (lane == 0) {
          ring[0] = make_int4(next.begin, next.len, next.slot, next.tile);
          ring[1] = make_int4(next.head, next.blocks, next.steps, 0);
        }
      }
      __syncthreads();
      const BwdItem it = read_item(k < kItems ? k : 0);
      if (it.steps == 0) {
        if (k < kItems) continue;
        break;
      }
      const __nv_bfloat16 nan = __ushort_as_bfloat16(0x7fc0);
      auto fill = [&](const AttnOut& o, int head, int from, int to) {
        for (long long e = threadIdx.x; e < static_cast<long long>(to - from) * p.hd; e += kThreadsB) {
          const long long row = it.begin + from + e / p.hd;
          static_cast<__nv_bfloat16*>(o.p)[row * o.row + head * o.head + e % p.hd] = nan;
        }
      };
      const int first = it.tile * kBlock, end = min(it.len, first + kBlock), kv = it.head / p.parts;
      if (p.parts == 1) {
        fill(p.dk, kv, first, end);
        fill(p.dv, kv, first, end);
      } else {
        for (int which = 0; which < 2; ++which) {
          float* part = p.partial + ((static_cast<long long>((it.head - kv * p.parts) * 2 + which) * p.hk + kv) * p.total + it.begin + first) * HD;
          for (int e = threadIdx.x; e < (end - first) * HD; e += kThreadsB) part[e] = __int_as_float(0x7fc00000);
        }
      }
      for (int h = 0; h < p.group && it.tile == 0; ++h) fill(p.dq, it.head * p.group + h, 0, it.len);
    }
  }
}

// dv and dk of a tile and key head from the parts of its group, in order: a thread has 8 columns of a row of one of them.  (A thread a row
// and all its columns one after another, 9 sequences of 1 to 1500 rows, 16 heads of 128 and 2 of keys: 139 us for 13.)
template <int HD>
__global__ void __launch_bounds__(kBlock)
attn_join_kernel(const BwdParams p) {
  pdl_wait();
  const int tile = blockIdx.x, kv = blockIdx.y, r = threadIdx.x;
  if (!plan_fits(p.plan, p.n, p.total) || tile >= __ldg(p.plan + kPlanBwdTiles)) return;
  const int4 rec = __ldg(reinterpret_cast<const int4*>(p.tiles) + tile);
  const int row = rec.z * kBlock + r, rows = min(32, rec.y - rec.x - rec.z * kBlock - (r & ~31));
  if (row >= rec.y - rec.x) return;
  const int which = blockIdx.z & 1, c = 8 * (blockIdx.z >> 1);
  if (c >= p.hd) return;
  const AttnOut& to = which == 0 ? p.dv : p.dk;
  const float by = which == 0 ? 1.f : p.scale;
  const float* from = p.partial + ((static_cast<long long>(which) * p.hk + kv) * p.total + rec.x + rec.z * kBlock + (r & ~31)) * HD;
  const float4* at = reinterpret_cast<const float4*>(from) + (r & 31) + static_cast<long long>(c / 4) * rows;
  const long long apart = 2ll * p.hk * p.total * (HD / 4);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll 4
  for (int part = 0; part < p.parts; ++part) {
    const float4 x = __ldcs(at + part * apart), y = __ldcs(at + part * apart + rows);
    a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
    b.x += y.x; b.y += y.y; b.z += y.z; b.w += y.w;
  }
  *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(to.p) + (rec.x + row) * to.row + kv * to.head + c) =
      make_uint4(bf16_pair(a.x * by, a.y * by), bf16_pair(a.z * by, a.w * by), bf16_pair(b.x * by, b.y * by), bf16_pair(b.z * by, b.w * by));
}

// -lse log2 e and -delta of every row and head, and the counters' start: LANES threads a row and head, 16 bytes each, four of these at
// a time; 32 rows of one head before the next head's, so that what is written are whole sectors.  With a plan of another batch, NaN in all
// results instead: the kernels behind this one find nothing to do.
template <int LANES>
__global__ void __launch_bounds__(256)
attn_backward_start_kernel(const AttnBackward a, float* stats, unsigned* counters, long long n_counters) {
  constexpr int kRowsOf = 256 / LANES, kUnroll = 4;
  pdl_wait();
  for (long long c = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; c < n_counters; c += static_cast<long long>(gridDim.x) * 256) counters[c] = 0u;
  if (!plan_fits(a.plan, a.n, a.total)) {
    const int at = blockIdx.x * 8 + threadIdx.x / 32, step = gridDim.x * 8;
    fill_nan<__nv_bfloat16>(a.dq, a.total, a.hq, a.hd, at, step);
    fill_nan<__nv_bfloat16>(a.dk, a.total, a.hk, a.hd, at, step);
    fill_nan<__nv_bfloat16>(a.dv, a.total, a.hk, a.hd, at, step);
    return;
  }
  const int lane = threadIdx.x % LANES, c = lane * 8;
  uint4 x[kUnroll], y[kUnroll];
  long long at[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const long long w = (static_cast<long long>(blockIdx.x) * kUnroll + u) * kRowsOf + threadIdx.x / LANES;
    const unsigned block = static_cast<unsigned>(w >> 5) / static_cast<unsigned>(a.hq), head = static_cast<unsigned>(w >> 5) - block * a.hq;
    const long long row = 32ll * block + (w & 31);
    at[u] = row < a.total ? head * static_cast<long long>(a.total) + row : -1;
    x[u] = y[u] = make_uint4(0u, 0u, 0u, 0u);
    if (row < a.total && c < a.hd) {
      x[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.dout.p) + row * a.dout.row + head * a.dout.head + c));
      y[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.o.p) + row * a.o.row + head * a.o.head + c));
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    float f[8], g[8], s = 0.f;
    Vec<__nv_bfloat16>::unpack(x[u], f);
    Vec<__nv_bfloat16>::unpack(y[u], g);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(f[e], g[e], s);
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (at[u] >= 0 && lane == 0) {
      stats[at[u]] = -a.lse[at[u]] * kLog2eB;
      stats[static_cast<long long>(a.hq) * a.total + at[u]] = -s;
    }
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
  const AttnScratch s = attn_scratch(a.total, a.hq, a.hk, a.hd, a.n);
  char* mem = static_cast<char*>(a.scratch);
  auto kern = attn_backward_kernel<HD>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, Sh::kSmem));
  // the softmax warps' registers come out of what the launch has: with fewer than 128 a thread they would never get them
  static const int regs = [&] {
    cudaFuncAttributes fa;
    return cudaFuncGetAttributes(&fa, kern) == cudaSuccess ? fa.numRegs : 0;
  }();
  if (regs != 128) return set_error(ctx, ABS_ERR_CUDA, "the backward kernel was built with %d registers a thread, not 128", regs);
  const long long counters = static_cast<long long>(a.hq) * l.bwd_cap * Sh::kHalves + 1;
  const long long rows = (a.total + 31ll) / 32 * 32 * a.hq, ctas = (rows * (HD / 8) + 1023) / 1024;
  ABS_CUDA_TRY(ctx, launch_dependent(attn_backward_start_kernel<HD / 8>, dim3(static_cast<unsigned>(ctas)), dim3(256), 0, st, a,
                                     reinterpret_cast<float*>(mem + s.delta), reinterpret_cast<unsigned*>(mem + s.counters), counters));
  const int parts = attn_parts(a.total, a.hq, a.hk, a.n), group = a.hq / a.hk / parts, all = a.hk * parts;
  const BwdParams p{a.dq, a.dk, a.dv, reinterpret_cast<float*>(mem + s.delta), reinterpret_cast<float*>(mem + s.sums),
                    reinterpret_cast<unsigned*>(mem + s.counters), a.plan, a.plan + l.bwd, a.n, a.total, a.hq, a.hk,
                    parts, a.hd, l.bwd_cap, all, group, reinterpret_cast<float*>(mem + s.partial), a.scale * kLog2eB, a.scale,
                    ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles,
                    ctx->tuning.stats_fault_drop_loads ? 1 : 0, fault_steps(ctx),
                    in_sectors(a.dq, a.hd) && in_sectors(a.dk, a.hd) && in_sectors(a.dv, a.hd)};
  const long long most = static_cast<long long>(l.bwd_cap) * all;
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
  if (parts > 1) ABS_CUDA_TRY(ctx, launch_dependent(attn_join_kernel<HD>, dim3(l.bwd_cap, a.hk, 2 * (HD / 8)), dim3(kBlock), 0, st, p));
  return ABS_OK;
}

}  // namespace

int launch_attention_tc_backward(abs_ctx* ctx, const AttnBackward& a, cudaStream_t st) {
  if (encode_tiled_fn() == nullptr) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  return a.hd <= 64 ? run_backward_tc<64>(ctx, a, st) : run_backward_tc<128>(ctx, a, st);
}

}  // namespace absk
