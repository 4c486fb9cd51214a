// Causal attention, forward, bf16 on the tcgen05 tensor cores.
//
//   s = c q k' (c = scale log2 e),  p = 2^(s - m),  o = (sum_j p_j v_j) / sum_j p_j,  lse = ln 2 (m + log2 sum_j p_j)
//
// One pass over the keys with a running reference m of each row.  A resident CTA an SM walks the plan's tiles of 256 queries of one
// head, two halves of 128, longest first.  Per 128 keys and half: S = Q K' into tensor memory (128 columns of fp32); the half's four
// warps, a thread a row, read it, take the exponentials and write P as bf16 over the first half of S, from where the tensor core takes
// it as the operand of O += P V (P never touches shared memory).  While one half's warps work on their exponentials the other's
// products run.
//
// m is raised only where a row's largest score is more than 8 above it: p is then at most 2^8, which costs nothing in fp32 sums or
// bf16's relative steps, and O, which stays in tensor memory, is rescaled a few times a tile instead of once per 128 keys.
// Rounded to fewer bits than 32: P to bf16, as an operand of the tensor core (its sums of p are taken before that), and O.
//
// The floor is the exponentials at 64 columns a head (16 a clock and SM: 1024 clocks per 128 x 128 scores, whose products take 512) and
// both at 128; what bounds it are the softmax warps, two a scheduler, whose steps depend on one another (issue slots 45 % busy): two
// passes over S from tensor memory, the first for its largest, because 128 scores a thread held in registers spill (672 us for 500).
// 128 of 1024 tokens, 12 heads of 64: 455 us over the same tensors again and again, 505 over others each time (all exponentials on their
// unit alone 200, products 146 at the sustained rate); 8191 and 4097 tokens, 8 heads of 128 and 2 of keys: 225 us, 760 TFLOP/s.  A sequence of
// up to 128 tokens has one half's warps idle (2000 of 64 tokens, 12 heads of 64: 480 us), half 0 of a tile has a step less than half 1, and
// heads of other widths than 64 and 128 cost what these do (4 of 4096 tokens, 8 heads and 2 of keys, 32, 64, 80, 96 and 128 columns: 146,
// 147, 160, 160, 161 us).
//
// Roles of the 12 warps: 0 loads (TMA; Q once a tile, K and V through a ring of 128-row places), 1 issues the products, 4-7 and 8-11
// are the two halves.  All waits are bounded: one that runs out raises the CTA's abort flag, every role falls through, copies in
// flight are waited for, tensor memory is freed, and the rows of tiles that were not finished are NaN.
#include "abs_attention.cuh"
#include "abs_tc.cuh"

namespace absk {
namespace {

constexpr int kThreadsF = 384;
constexpr int kFewRegs = 88, kManyRegs = 208;  // of a thread of warps 0-3 and of the halves; together what 168 a thread are at the launch
static_assert(128 * kFewRegs + 256 * kManyRegs == kThreadsF * 168, "");
constexpr int kHalf = 128;                    // rows of a half, keys of a step
constexpr float kRaise = 8.f;
constexpr float kLn2F = 0.6931471805599453f, kLog2eF = 1.4426950408889634f;

template <int HD> struct FwdShape {
  static constexpr uint32_t kRowsBytes = kHalf * HD * 2;          // 128 rows of one head
  static constexpr int kPlaces = HD == 64 ? 8 : 5;
  // Of 16 pairs of exponentials how many are taken on the FMA pipe.  0, 2, 4, 5, 6: 486, 478, 475, 480, 488 us (128 of 1024 tokens, 12 heads
  // of 64), 171, 168, 170, 171, 176 (4 of 4096, 8 heads of 128 and 2 of keys): what issues is soon as scarce as the unit.
  static constexpr int kFmaPairs = HD == 64 ? 4 : 2;
  // tensor memory: S of the halves, O of the halves from 256 on; P over S, or beside it where there is room
  static __device__ __forceinline__ uint32_t p_at(uint32_t t) { return HD == 64 ? 384u + 64u * t : 128u * t; }
  static constexpr size_t kSmem = (2 + kPlaces) * static_cast<size_t>(kRowsBytes) + 1024 + 512;
};

struct FwdMaps {
  CUtensorMap q, k, v;
};
struct FwdParams {
  AttnOut o;
  float* lse;
  const int* plan;
  const int* tiles;
  int n, total, hq, group, hd;
  float by;                                   // scale log2 e
  long long limit;
  bool sectors;                               // whether O is rows of whole sectors of 32 bytes
  int drop_loads;                             // test hook: nothing is loaded, so every wait must run out
  uint32_t stop_after;                        // test hook: no more than so many keys' and values' places are filled by CTAs of even numbers
};
struct FwdItem {
  int begin, len, row, head, kv, n0, n1;      // row: the tile's first in the sequence; n0, n1: steps of its halves
};
__device__ __forceinline__ FwdItem item_of(const FwdParams& p, int i) {
  FwdItem it;
  const int tile = i / p.hq;
  it.head = i - tile * p.hq;
  const int4 r = __ldg(reinterpret_cast<const int4*>(p.tiles) + tile);
  it.begin = r.x;
  it.len = r.y - r.x;
  it.row = r.z * kAttnFwdRows;
  it.kv = it.head / p.group;
  it.n0 = 2 * r.z + 1;
  it.n1 = it.row + kHalf < it.len ? it.n0 + 1 : 0;
  return it;
}

template <int HD>
__global__ void __launch_bounds__(kThreadsF, 1)
attn_forward_kernel(const __grid_constant__ FwdMaps maps, const FwdParams p) {
  constexpr uint32_t kRows = FwdShape<HD>::kRowsBytes;
  constexpr int kPlaces = FwdShape<HD>::kPlaces;
  extern __shared__ unsigned char smem_dyn[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_dyn), q_at = (raw + 1023u) & ~1023u, ring = q_at + 2u * kRows;
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem_dyn + (q_at - raw) + (2 + kPlaces) * kRows);
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + 18 + 2 * kPlaces);
  unsigned* tmem_slot = const_cast<unsigned*>(abort_flag) + 1;
  const uint32_t q_full = smem_u32(bars), q_free = q_full + 16u, s_full = q_free + 16u, p_full = s_full + 16u, o_full = p_full + 16u,
                 o_free = o_full + 16u, s_read = o_free + 16u, pv_done = s_read + 16u, landed = pv_done + 16u, done_bar = landed + 8u, full = done_bar + 8u, freed = full + 8u * kPlaces;
  if (threadIdx.x == 0) {
    for (uint32_t t = 0; t < 2; ++t) {
      mbar_init(q_full + 8u * t, 1);
      mbar_init(q_free + 8u * t, 1);
      mbar_init(s_full + 8u * t, 1);
      mbar_init(p_full + 8u * t, 4);
      mbar_init(o_full + 8u * t, 1);
      mbar_init(o_free + 8u * t, 4);
      mbar_init(s_read + 8u * t, 4);
      mbar_init(pv_done + 8u * t, 1);
    }
    mbar_init(landed, 1);
    mbar_init(done_bar, 1);
    for (uint32_t s = 0; s < kPlaces; ++s) {
      mbar_init(full + 8u * s, 1);
      mbar_init(freed + 8u * s, 1);
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_all(smem_u32(tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  const int items = plan_fits(p.plan, p.n, p.total) ? __ldg(p.plan + kPlanFwdTiles) * p.hq : 0;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
    if (warp == 0) {
      // ---- loads ---------------------------------------------------------------------------------
      uint32_t n = 0, lands = 0, uses[2] = {0, 0};
      bool ok = !p.drop_loads;
      // 128 rows of one head from the sequence's row r on
      auto copy = [&](const CUtensorMap* map, uint32_t to, int head, int row, uint32_t bar) {
        if (elect_lane()) {
          mbar_expect_tx(bar, kRows);
#pragma unroll
          for (uint32_t c = 0; c < HD / 64; ++c) tma_load_3d(to + c * (kHalf * 128u), map, 64 * static_cast<int>(c), head, row, bar);
        }
        __syncwarp();
      };
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const FwdItem it = item_of(p, i);
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) {
          if (t == 1 && it.n1 == 0) continue;
          if (uses[t] > 0) ok = ok && warp_wait(q_free + 8u * t, (uses[t] - 1) & 1u, abort_flag, p.limit);
          if (!ok) break;
          copy(&maps.q, q_at + t * kRows, it.head, it.begin + it.row + static_cast<int>(t) * kHalf, q_full + 8u * t);
          ++uses[t];
        }
        const int steps = max(it.n0, it.n1);
        for (int j = 0; j < 2 * steps && ok; ++j, ++n) {
          const uint32_t s = n % kPlaces, pass = n / kPlaces, to = ring + s * kRows;
          if (pass > 0) ok = warp_wait(freed + 8u * s, (pass - 1) & 1u, abort_flag, p.limit);
          if (n >= p.stop_after && (blockIdx.x & 1u) == 0u) ok = false;
          if (!ok) break;
          const int key = (j >> 1) * kHalf, in = it.len - key;                   // rows of the sequence from the step's first key on
          if ((j & 1) == 0) {
            copy(&maps.k, to, it.kv, it.begin + key, full + 8u * s);
          } else if (in >= kHalf) {
            copy(&maps.v, to, it.kv, it.begin + key, full + 8u * s);
          } else {
            // rows of V behind the sequence have weights of zero, but may hold anything: zeros in their place
            copy(&maps.v, to, it.kv, it.begin + key, landed);
            ok = warp_arrival(landed, lands & 1u, abort_flag, p.limit);
            ++lands;
            if (!ok) break;
            for (uint32_t c = 0; c < HD / 64; ++c)
              for (uint32_t e = static_cast<uint32_t>(in) * 128u + lane * 16u; e < kHalf * 128u; e += 512u)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + c * (kHalf * 128u) + e), "r"(0u) : "memory");
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(full + 8u * s);
          }
        }
      }
      // Waits (bounded) until every copy that was issued has arrived, whatever made the other roles stop.
      for (uint32_t s = 0; s < kPlaces; ++s) {
        const uint32_t fills = n / kPlaces + (s < n % kPlaces ? 1u : 0u);
        if (fills > 0) warp_arrival(full + 8u * s, (fills - 1) & 1u, abort_flag, p.limit);
      }
      for (uint32_t t = 0; t < 2; ++t)
        if (uses[t] > 0) warp_arrival(q_full + 8u * t, (uses[t] - 1) & 1u, abort_flag, p.limit);
      if (lands > 0) warp_arrival(landed, (lands - 1) & 1u, abort_flag, p.limit);
    } else if (warp == 1) {
      // ---- products --------------------------------------------------------------------------------
      constexpr uint32_t idesc_s = mma_idesc(kHalf, kHalf, false, false), idesc_o = mma_idesc(kHalf, HD, false, true);
      constexpr uint64_t desc_v = desc_mn(kHalf * 128);
      uint32_t n = 0, uses[2] = {0, 0}, done[2] = {0, 0};        // places; tiles and steps of each half so far
      bool ok = true;
      auto scores = [&](uint32_t t, uint32_t place) {            // S of half t from Q and the K at the place
        if (elect_lane()) {
          const uint32_t a = desc_at(q_at + t * kRows), b = desc_at(ring + place * kRows);
#pragma unroll
          for (uint32_t k = 0; k < HD / 16; ++k) {
            const uint32_t off = (k / 4) * (kHalf * 128u / 16u) + (k % 4) * 2u;
            mma_ss(tmem + t * kHalf, kDescK | (a + off), kDescK | (b + off), idesc_s, k > 0);
          }
          mma_commit(s_full + 8u * t);
        }
        __syncwarp();
      };
      for (int i = blockIdx.x; i < items && ok; i += gridDim.x) {
        const FwdItem it = item_of(p, i);
        const int steps = max(it.n0, it.n1);
        ok = warp_wait(full + 8u * (n % kPlaces), (n / kPlaces) & 1u, abort_flag, p.limit);
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) {
          if (t == 1 && it.n1 == 0) continue;
          ok = ok && warp_wait(q_full + 8u * t, uses[t] & 1u, abort_flag, p.limit);
          tc_fence_after();
          scores(t, n % kPlaces);
          if ((t == 0 ? it.n0 : it.n1) == 1 && elect_lane()) mma_commit(q_free + 8u * t);
          __syncwarp();
        }
        if (elect_lane()) mma_commit(freed + 8u * (n % kPlaces));
        __syncwarp();
        for (int j = 0; j < steps && ok; ++j) {
          const uint32_t v = n + 2 * j + 1, k = v + 1;           // places of this step's V and the next one's K
          ok = warp_wait(full + 8u * (v % kPlaces), (v / kPlaces) & 1u, abort_flag, p.limit);
          const uint32_t b = desc_at(ring + (v % kPlaces) * kRows);
          // P beside S: the next S as soon as this one has been read, while its exponentials are still being taken
#pragma unroll
          for (uint32_t t = 0; t < 2; ++t) {
            const int last = t == 0 ? it.n0 : it.n1;
            if (HD != 64 || j + 1 >= last || !ok) continue;
            ok = warp_wait(full + 8u * (k % kPlaces), (k / kPlaces) & 1u, abort_flag, p.limit);
            ok = ok && warp_wait(s_read + 8u * t, done[t] & 1u, abort_flag, p.limit);
            if (!ok) continue;
            tc_fence_after();
            scores(t, k % kPlaces);
            if (j + 2 == last && elect_lane()) mma_commit(q_free + 8u * t);
            __syncwarp();
          }
#pragma unroll
          for (uint32_t t = 0; t < 2; ++t) {
            const int last = t == 0 ? it.n0 : it.n1;
            if (j >= last || !ok) continue;
            if (j == 0 && uses[t] > 0) ok = warp_wait(o_free + 8u * t, (uses[t] - 1) & 1u, abort_flag, p.limit);
            ok = ok && warp_wait(p_full + 8u * t, done[t] & 1u, abort_flag, p.limit);
            if (!ok) continue;
            ++done[t];
            tc_fence_after();
            if (elect_lane()) {
#pragma unroll
              for (uint32_t kk = 0; kk < kHalf / 16; ++kk)
                mma_ts(tmem + 256u + t * HD, tmem + FwdShape<HD>::p_at(t) + 8u * kk, desc_v | (b + 128u * kk), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
              if (HD == 64) mma_commit(pv_done + 8u * t);
              if (j == last - 1) mma_commit(o_full + 8u * t);
            }
            __syncwarp();
            if (HD == 128 && j + 1 < last) {
              ok = warp_wait(full + 8u * (k % kPlaces), (k / kPlaces) & 1u, abort_flag, p.limit);
              tc_fence_after();
              scores(t, k % kPlaces);
              if (j + 2 == last && elect_lane()) mma_commit(q_free + 8u * t);
              __syncwarp();
            }
          }
          if (elect_lane()) {
            mma_commit(freed + 8u * (v % kPlaces));
            if (j + 1 < steps) mma_commit(freed + 8u * (k % kPlaces));
          }
          __syncwarp();
        }
        n += 2 * steps;
        ++uses[0];
        if (it.n1 > 0) ++uses[1];
      }
      if (elect_lane()) mma_commit(done_bar);
      __syncwarp();
      volatile unsigned ignore = 0u;
      mbar_wait(done_bar, 0u, &ignore, p.limit);                 // no product in flight when tensor memory is freed
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs));
    // ---- softmax: a thread has a row ------------------------------------------------------------------
    const uint32_t t = static_cast<uint32_t>(warp - 4) >> 2;
    const int r = (warp & 3) * 32 + lane;                        // row of the half
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + t * kHalf + lanes, o_at = tmem + 256u + t * HD + lanes,
                   p_at = tmem + FwdShape<HD>::p_at(t) + lanes;
    const uint64_t by2 = pack2f(p.by, p.by);
    uint32_t steps_done = 0, uses = 0;
    bool ok = true;
    for (int i = blockIdx.x; i < items; i += gridDim.x) {
      const FwdItem it = item_of(p, i);
      const int steps = t == 0 ? it.n0 : it.n1;
      if (steps == 0) continue;
      const int row = it.row + static_cast<int>(t) * kHalf + r;
      const bool live = row < it.len;
      float m = -INFINITY;                                       // the reference
      float sum = 0.f;
      for (int j = 0; j < steps && ok; ++j, ++steps_done) {
        ok = warp_wait(s_full + 8u * t, steps_done & 1u, abort_flag, p.limit);
        if (!ok) break;
        tc_fence_after();
        // S is read twice, 32 columns at a time and the next ones under way, instead of being held: 128 more registers a thread spill.
        // Loops of two pieces, not unrolled further: a warp that runs through long straight code waits for its instructions.
        const bool diagonal = j == steps - 1;
        uint32_t s[2][32];
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        tmem_load32(s_at, s[0]);
#pragma unroll 1
        for (int c = 0; c < kHalf; c += 64) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t* x = s[q];
            tmem_loaded(x);
            tmem_load32(s_at + ((c + 32 * q + 32) & (kHalf - 1)), s[q ^ 1]);       // (after the last: the first again)
            if (diagonal) {
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = e > r - c - 32 * q ? 0xff800000u : x[e];
            }
#pragma unroll
            for (int e = 0; e < 32; e += 8)
#pragma unroll
              for (int k = 0; k < 4; ++k) top[k] = max3f(top[k], __uint_as_float(x[e + k]), __uint_as_float(x[e + k + 4]));
          }
        }
        const float most = max3f(max3f(top[0], top[1], top[2]), top[3], top[3]) * p.by;
        // the products of the step before, which read P and add to O (with P over S they came before this S)
        if (HD == 64 && steps_done > 0) ok = warp_wait(pv_done + 8u * t, (steps_done - 1) & 1u, abort_flag, p.limit);
        if (!ok) {
          tmem_loaded(s[0]);                                       // (the load ahead: its registers are somebody else's from here on)
          break;
        }
        tc_fence_after();
        // (rows behind the sequence, which may hold anything, have no say, and a row's reference depends on that row alone)
        const bool raise = live && most > m + kRaise;
        if (__any_sync(0xffffffffu, raise)) {
          const float next = raise ? most : m;
          const float less = m == next ? 1.f : m == -INFINITY ? 0.f : exp2_approx(m - next);       // (0: nothing has been added yet)
          m = next;
          sum *= less;
          if (j > 0) {
#pragma unroll
            for (int c = 0; c < HD; c += 32) {
              uint32_t o[32];
              tmem_load32(o_at + c, o);
              tmem_loaded(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * less);
              tmem_store32(o_at + c, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : -m;
        const uint64_t ref2 = pack2f(ref, ref);
        uint64_t part[2] = {pack2f(0.f, 0.f), pack2f(0.f, 0.f)};
#pragma unroll 1
        for (int c = 0; c < kHalf; c += 64) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t* x = s[q];
            tmem_loaded(x);
            if (c + 32 * q + 32 < kHalf) {
              tmem_load32(s_at + c + 32 * q + 32, s[q ^ 1]);
            } else if (HD == 64) {                                 // the last of S has been read
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(s_read + 8u * t);
            }
            if (diagonal) {
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = e > r - c - 32 * q ? 0xff800000u : x[e];
            }
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              uint64_t y = fma2f(pack2f(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), by2, ref2);
              y = e >= 16 - FwdShape<HD>::kFmaPairs ? exp2_pair_fma(y) : exp2_pair(y);
              part[e & 1] = add2f(part[e & 1], y);
              const float2 a = unpack2f(y);
              w[e] = bf16_pair(a.x, a.y);
            }
            tmem_store16(p_at + (c + 32 * q) / 2, w);              // (over S: columns that have been read)
          }
        }
        const float2 all = unpack2f(add2f(part[0], part[1]));
        sum += all.x + all.y;
        tmem_stored();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8u * t);
      }
      ok = ok && warp_wait(o_full + 8u * t, uses & 1u, abort_flag, p.limit);
      ++uses;
      tc_fence_after();
      const float inv = ok ? 1.f / sum : __int_as_float(0x7fc00000);
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.o.p) + (it.begin + row) * p.o.row + it.head * p.o.head;
#pragma unroll
      for (int c = 0; c < HD; c += 32) {
        uint32_t o[32];
        if (ok) {
          tmem_load32(o_at + c, o);
          tmem_loaded(o);
        }
        if (c + 32 >= HD && ok) {                                // the last of O has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(o_free + 8u * t);
        }
        if (live) store_row32(out + c, o, inv, ok, p.hd - c, p.sectors);
      }
      if (live && p.lse)
        p.lse[static_cast<long long>(it.head) * p.total + it.begin + row] = ok ? fmaf(m, kLn2F, logf(sum)) : __int_as_float(0x7fc00000);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_free_all(tmem);
  }
  if (items == 0 && !plan_fits(p.plan, p.n, p.total)) {
    const int at = blockIdx.x * (kThreadsF / 32) + warp, step = gridDim.x * (kThreadsF / 32);
    fill_nan<__nv_bfloat16>(p.o, p.total, p.hq, p.hd, at, step);
    if (p.lse) fill_nan<float>({p.lse, 1, p.total}, p.total, p.hq, 1, at, step);
  }
}

template <int HD>
int run_forward_tc(abs_ctx* ctx, const AttnForward& a, cudaStream_t st) {
  FwdMaps maps;
  if (!encode_heads_map(a.q, a.total, a.hq, a.hd, &maps.q) || !encode_heads_map(a.k, a.total, a.hk, a.hd, &maps.k) ||
      !encode_heads_map(a.v, a.total, a.hk, a.hd, &maps.v))
    return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled (%d rows, head_dim %d) failed", a.total, a.hd);
  const AttnPlanLayout l = attn_plan_layout(a.n, a.total);
  const FwdParams p{a.o, a.lse, a.plan, a.plan + l.fwd, a.n, a.total, a.hq, a.hq / a.hk, a.hd, a.scale * kLog2eF,
                    ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles,
                    in_sectors(a.o, a.hd), ctx->tuning.stats_fault_drop_loads ? 1 : 0, fault_steps(ctx)};
  auto kern = attn_forward_kernel<HD>;
  const size_t smem = FwdShape<HD>::kSmem;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  // the halves' registers come out of what the launch has: with fewer than 168 a thread they would never get them
  static const int regs = [&] {
    cudaFuncAttributes fa;
    return cudaFuncGetAttributes(&fa, kern) == cudaSuccess ? fa.numRegs : 0;
  }();
  if (regs != 168) return set_error(ctx, ABS_ERR_CUDA, "the forward kernel was built with %d registers a thread, not 168", regs);
  const long long most = static_cast<long long>(l.fwd_cap) * a.hq;
  const unsigned grid = static_cast<unsigned>(most < ctx->sm_count ? most : ctx->sm_count);
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(grid), dim3(kThreadsF), smem, st, maps, p));
  return ABS_OK;
}

}  // namespace

bool encode_heads_map(const AttnRows& t, int total, int heads, int hd, CUtensorMap* map) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(total)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(t.head) * 2, static_cast<cuuint64_t>(t.row) * 2};
  const cuuint32_t box[3] = {64u, 1u, static_cast<cuuint32_t>(kHalf)}, ones[3] = {1u, 1u, 1u};
  return encode_tiled_fn()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(t.p), dims, strides, box, ones,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int launch_attention_tc(abs_ctx* ctx, const AttnForward& a, cudaStream_t st) {
  if (encode_tiled_fn() == nullptr) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  return a.hd <= 64 ? run_forward_tc<64>(ctx, a, st) : run_forward_tc<128>(ctx, a, st);
}

}  // namespace absk
