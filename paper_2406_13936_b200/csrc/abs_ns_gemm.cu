// All steps of the Newton-Schulz iteration of a group of matrices in one launch, on the tcgen05 tensor
// cores.  A step is three products:
//   kGram    A = X X'
//   kPoly    B = b A + c A A
//   kUpdate  X <- a X + B X
// A and B are symmetric: only their tiles on and below the diagonal are computed and stored.  A block
// above the diagonal is read as the transpose of the stored one, which the tensor core does by itself:
// an operand whose k index runs along the rows of the stored matrix is MN-major (as X is in kUpdate),
// one whose k index runs along the columns is K-major; the TMA box and the descriptor differ, no more.
//
// The tiles of all steps, products and matrices form one list, in that order; a resident grid walks it
// with a fixed stride.  A tile starts when the row blocks that it reads are complete, which other CTAs
// announce in per-matrix counters (release / acquire in global memory): no launch, grid barrier or idle
// wave between products.  (Three parts of the matrices a product apart, so that a product and the one that
// reads it were never neighbours in the list, took as long: 8 x 1024 x 1024 264 us against 261, 96 x 768 x
// 768 1408 against 1389; what the waits gained the longer start and end lost.)
// Nothing that is still read is overwritten: a tile of a product needs the row blocks of the one before,
// which need all of the one before that that touches them, and so on; written out, every tile that reads
// a buffer is complete before the tile that writes the same rows of it again may start.  The launch is
// cooperative, so every CTA that is waited for is resident.
//
// CG = 1: a CTA has 128 x 128 tiles.  CG = 2: a pair of CTAs has 256 x 256 tiles (tcgen05 cta_group::2:
// each CTA loads its 128 rows of the first operand and half the columns of the second, and holds its
// 128 rows of the accumulator), which halves the operand bytes per product.
//
// An SM takes in about 64 bytes a clock from L2 (measured: a k-block of 64 of a 128 x 128 tile, 32 KB,
// takes 556 clocks, its products 256), which is what a pair's tile needs at the tensor cores' full rate.
//
// Roles of a CTA's 14 warps: 0 loads operands by TMA into a ring of 32 KB stages, 12 looks out for the inputs of
// the next tile meanwhile, 1 issues the products (fp32 accumulators in tensor memory, two of them, so the next
// tile's products run while this one is read back), 4-7 and 8-11 are the two halves of the epilogue (each reads back
// half the tile's columns and applies the coefficients in place, in shared memory), 2 loads what the
// coefficients apply to, 3 and 13 store one half's results by TMA and announce the half tile.  Loads, stores and
// announcements (a fence of 1000 to 4000 clocks) have threads of their own because one after the other they took
// longer than a tile's products.  All waits are bounded; one that runs out raises the CTA's abort flag and the call's
// flag word, every role falls through, copies in flight are waited for and tensor memory is freed.
#include "abs_ns.cuh"
#include "abs_pipeline.cuh"

namespace absk {
namespace {

enum { kGram = 0, kPoly = 1, kUpdate = 2 };

constexpr int kBM = 128;                     // rows of a CTA's tile
constexpr int kEpiWarpsN = 8;
constexpr int kFirstEpi = 4;
constexpr int kLookout = kFirstEpi + kEpiWarpsN;
constexpr int kThreadsN = (kLookout + 2) * 32;             // 448
constexpr uint32_t kStageN = 32768;
// Units of the epilogue: 32 columns of the tile's 128 rows, changed in place in shared memory: 8 KB of fp16
// values (A, B) or 16 KB of values and remainders (X; with split operands any matrix).  Each half of the epilogue has
// a ring of three places for them, which runs on from tile to tile.
constexpr int kUnitCols = 32;
constexpr uint32_t kUnitBytes = kBM * kUnitCols * 2;       // 8 KB
constexpr int kStagesN = 4;
constexpr uint32_t kPlaces = 3;
constexpr uint32_t kHalfArea = kPlaces * 2 * kUnitBytes;
constexpr size_t kSmemN = static_cast<size_t>(kStagesN) * kStageN + 2 * kHalfArea + 1024 + 512;      // alignment, barriers
// Split operands: an accumulator of the main products takes kFold k-blocks of 32 (2 kFold additions) and is
// then added, rounded to nearest, to sums in registers: the tensor core adds without rounding to nearest.  With 8
// instead of 4, error against 64 bits and time: 662 x 1510 4.4e-6, 306 us for 2.6e-6, 314 (plain fp32 products 2.8e-6);
// 8 of 784 x 1024 1.7e-6, 428 for 1.0e-6, 438 (2.4e-6).
constexpr int kFold = 4;

struct NsMaps {
  // operands: boxes of [128 rows][k-block] (K-major) and [k-block][64 columns] (MN-major); _l: remainders
  CUtensorMap xk_h[2], xk_l[2], xm_h[2], xm_l[2], ak_h, ak_l, am_h, am_l, bk_h, bk_l, bm_h, bm_l;
  // units of the epilogue: boxes of [128 rows][32 columns]
  CUtensorMap xu_h[2], xu_l[2], au_h, au_l, bu_h, bu_l;
};
struct NsStepsParams {
  int Z, m, n, steps;
  int row_blocks;             // of 128 CG rows
  int col_tiles;              // of 128 CG columns of X
  int tri;                    // tiles of a symmetric result
  long long per_step, tiles;
  unsigned* progress;         // [Z][3][row_blocks]: X, A, B
  unsigned* flag;
  long long timeout_cycles;
  int drop_loads;             // test hook: nothing is loaded, so every wait must run out
  NsCoef coef[kNsMaxSteps][3];
};

// ---- PTX ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void fence_async_n() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// (of global memory alone: 900 clocks less than of every state space, on the way from one product to the next; 4 of 256 x 256 84 -> 79 us)
__device__ __forceinline__ void fence_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }
__device__ __forceinline__ void tcn_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcn_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ bool elect_one_n() {
  uint32_t is_leader;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(is_leader));
  return is_leader != 0;
}
template <int CG>
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrives on the barrier (of both CTAs of a pair) when the products issued so far are complete.
template <int CG>
__device__ __forceinline__ void umma_commit_n(uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"(static_cast<unsigned short>(3))
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Tile load into this CTA's shared memory; `bar` may be the barrier of the pair's first CTA.
template <int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    tma_load_3d(dst, map, x, y, z, bar);
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src),
               "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
// 32 consecutive columns of this thread's lane; the values may be used after tmem_wait on the same registers.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
        "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
        "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
        "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      :
      : "memory");
}
__device__ __forceinline__ void sts128_n(uint32_t addr, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// ---- the list of tiles ---------------------------------------------------------------------------------
struct Tile {
  int step, mode, z, i, j;
};
__device__ __forceinline__ Tile tile_of(const NsStepsParams& p, long long t) {
  Tile q;
  q.step = static_cast<int>(t / p.per_step);
  long long r = t - q.step * p.per_step;
  const long long sym = static_cast<long long>(p.Z) * p.tri;
  if (r < 2 * sym) {
    q.mode = r < sym ? kGram : kPoly;
    if (q.mode == kPoly) r -= sym;
    q.z = static_cast<int>(r / p.tri);
    const int k = static_cast<int>(r - static_cast<long long>(q.z) * p.tri);
    q.i = static_cast<int>((sqrtf(8.f * static_cast<float>(k) + 1.f) - 1.f) * 0.5f);      // corrected to i (i + 1) / 2 <= k
    while (q.i * (q.i + 1) / 2 > k) --q.i;
    while ((q.i + 1) * (q.i + 2) / 2 <= k) ++q.i;
    q.j = k - q.i * (q.i + 1) / 2;
  } else {
    r -= 2 * sym;
    q.mode = kUpdate;
    const int per = p.row_blocks * p.col_tiles;
    q.z = static_cast<int>(r / per);
    const int k = static_cast<int>(r - static_cast<long long>(q.z) * per);
    q.i = k / p.col_tiles;
    q.j = k - q.i * p.col_tiles;
  }
  return q;
}

__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float2 unpack_f32x2(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}

// Whether an operand's block at k0 is the transpose of the stored one (above the diagonal of A or B), or X in
// kUpdate: its k index then runs along the rows of the stored matrix.
__device__ __forceinline__ bool a_is_mn(const Tile& q, int k0, int bn) { return q.mode != kGram && k0 / bn > q.i; }
__device__ __forceinline__ bool b_is_mn(const Tile& q, int k0, int bn) {
  return q.mode == kUpdate || (q.mode == kPoly && k0 / bn > q.j);
}

// Waits (bounded) until the counter has reached `target`.
__device__ __forceinline__ bool wait_count(const unsigned* c, unsigned target, const NsStepsParams& p, volatile unsigned* abort_flag) {
  const long long t0 = clock64();
  for (;;) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(c) : "memory");
    if (v >= target) return true;
    if (*abort_flag || *static_cast<volatile unsigned*>(p.flag) || clock64() - t0 > p.timeout_cycles) {
      *abort_flag = 1u;
      return false;
    }
    __nanosleep(32);
  }
}
// ... until what a tile reads is complete.  Row block i of a symmetric result is read from the tiles of row
// i and, transposed, of column i: row_blocks tiles.  Every CTA announces a tile twice (two epilogue halves).
template <int CG>
__device__ __forceinline__ bool wait_inputs(const NsStepsParams& p, const Tile& q, volatile unsigned* abort_flag) {
  const unsigned* base = p.progress + static_cast<long long>(q.z) * 3 * p.row_blocks;
  bool ok = true;
  if (q.mode == kGram) {
    if (q.step == 0) return true;
    const unsigned target = static_cast<unsigned>(q.step) * p.col_tiles * (2 * CG);
    ok = wait_count(base + q.i, target, p, abort_flag);
    if (ok && q.j != q.i) ok = wait_count(base + q.j, target, p, abort_flag);
  } else {
    const unsigned target = static_cast<unsigned>(q.step + 1) * p.row_blocks * (2 * CG);
    const unsigned* c = base + (q.mode == kPoly ? 1 : 2) * p.row_blocks;
    ok = wait_count(c + q.i, target, p, abort_flag);
    if (ok && q.mode == kPoly && q.j != q.i) ok = wait_count(c + q.j, target, p, abort_flag);
  }
  fence_async_global();                    // the copies that follow read what was announced
  return ok;
}
__device__ __forceinline__ void announce(unsigned* c) { asm volatile("red.relaxed.gpu.global.add.u32 [%0], 1;" ::"l"(c) : "memory"); }

// ---- the kernel ------------------------------------------------------------------------------------------
template <int CG, bool SPLIT>
__global__ void __launch_bounds__(kThreadsN, 1)
ns_steps_kernel(const __grid_constant__ NsMaps maps, const __grid_constant__ NsStepsParams p) {
  static_assert(CG == 1 || !SPLIT, "split operands use single CTAs");
  constexpr int BN = 128 * CG;                               // columns of a tile
  constexpr int kBK = SPLIT ? 32 : 64;                       // k-block
  constexpr uint32_t kOperand = SPLIT ? 8192u : 16384u;      // bytes of one operand tile of a stage
  constexpr int kUnits = BN / 2 / kUnitCols;                 // units of a tile per half of the epilogue
  extern __shared__ unsigned char smem_dyn[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank = 0;
  if (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const uint32_t raw = smem_u32(smem_dyn), ring = (raw + 1023u) & ~1023u;
  const uint32_t epi_at = ring + kStagesN * kStageN;
  unsigned char* tail = smem_dyn + (ring - raw) + kStagesN * kStageN + 2 * kHalfArea;
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(tail);
  constexpr int kBars = 2 * kStagesN + 11 + 6 * kPlaces;
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + kBars);
  unsigned* tmem_slot = const_cast<unsigned*>(abort_flag) + 1;
  const uint32_t full = smem_u32(bars), empty = full + 8u * kStagesN, accfull = empty + 8u * kStagesN, accempty = accfull + 16u,
                 crossempty = accempty + 16u, done = crossempty + 16u, ready = done + 8u, filled = ready + 16u * kPlaces,
                 freed = filled + 16u * kPlaces, inputs = freed + 16u * kPlaces, taken = inputs + 16u;
  if (tid == 0) {
    for (int s = 0; s < kStagesN; ++s) {
      mbar_init(full + 8u * s, 1);
      mbar_init(empty + 8u * s, 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(accfull + 8u * k, 1);
      mbar_init(accempty + 8u * k, kEpiWarpsN * CG);
      mbar_init(crossempty + 8u * k, kEpiWarpsN);
      mbar_init(inputs + 8u * k, 1);                       // a tile's inputs are complete
      mbar_init(taken + 8u * k, 2);                        // ... and both loaders know
    }
    mbar_init(done, 1);
    for (uint32_t k = 0; k < 2 * kPlaces; ++k) {         // per half and place
      mbar_init(ready + 8u * k, 1);                      // loaded (or free)
      mbar_init(filled + 8u * k, kEpiWarpsN / 2);        // finished
      mbar_init(freed + 8u * k, 1);                      // ... and stored
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tcn_before();
  __syncthreads();
  if constexpr (CG == 2) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  tcn_after();
  const uint32_t tmem = *tmem_slot;
  const long long first = blockIdx.x / CG, step = gridDim.x / CG;
  const int row_in_tile = static_cast<int>(rank) * kBM;      // this CTA's rows of a tile of 128 CG

  if (warp == 0) {
    // ---- operand loads ---------------------------------------------------------------------------
    if (elect_one_n()) {
      int s = 0;
      uint32_t pass = 0, it = 0;
      const uint32_t full0 = CG == 2 ? map_to_rank(full, 0) : full;       // the pair's barrier is its first CTA's
      for (long long t = first; t < p.tiles && !p.drop_loads; t += step) {
        const Tile q = tile_of(p, t);
        const int cur = q.step & 1;
        const int K = q.mode == kGram ? p.n : p.m, n_kb = (K + kBK - 1) / kBK;
        const int row = q.i * BN + row_in_tile, col = q.j * BN + row_in_tile;      // (the tile is square)
        if (!mbar_wait(inputs + 8u * (it & 1u), (it >> 1) & 1u, abort_flag, p.timeout_cycles)) break;
        mbar_arrive(taken + 8u * (it & 1u));
        ++it;
        for (int kb = 0; kb < n_kb; ++kb) {
          if (pass > 0 && !mbar_wait(empty + 8u * s, (pass - 1) & 1u, abort_flag, p.timeout_cycles)) break;
          const uint32_t st = ring + static_cast<uint32_t>(s) * kStageN, bar = full0 + 8u * s;
          if (rank == 0) mbar_expect_tx(full + 8u * s, CG * kStageN);
          const int k0 = kb * kBK;
          auto operand = [&](uint32_t at, const CUtensorMap* k_map, const CUtensorMap* m_map, int r, bool mn) {
            if (mn) {                                       // two blocks of [k-block] x [64 columns]
              load_tile<CG>(at, m_map, r, k0, q.z, bar);
              load_tile<CG>(at + kOperand / 2, m_map, r + 64, k0, q.z, bar);
            } else {
              load_tile<CG>(at, k_map, k0, r, q.z, bar);
            }
          };
          const bool mn_a = a_is_mn(q, k0, BN), mn_b = b_is_mn(q, k0, BN);
          const CUtensorMap *ak = q.mode == kGram ? &maps.xk_h[cur] : q.mode == kPoly ? &maps.ak_h : &maps.bk_h;
          const CUtensorMap *am = q.mode == kPoly ? &maps.am_h : &maps.bm_h;
          operand(st, ak, am, row, mn_a);
          operand(st + kOperand * (SPLIT ? 2u : 1u), ak, q.mode == kUpdate ? &maps.xm_h[cur] : am, col, mn_b);
          if (SPLIT) {
            const CUtensorMap *akl = q.mode == kGram ? &maps.xk_l[cur] : q.mode == kPoly ? &maps.ak_l : &maps.bk_l;
            const CUtensorMap *aml = q.mode == kPoly ? &maps.am_l : &maps.bm_l;
            operand(st + kOperand, akl, aml, row, mn_a);
            operand(st + 3u * kOperand, akl, q.mode == kUpdate ? &maps.xm_l[cur] : aml, col, mn_b);
          }
          if (++s == kStagesN) {
            s = 0;
            ++pass;
          }
        }
        if (*abort_flag) break;
      }
      // Waits (bounded) until every copy that was issued has arrived, whatever made the other roles stop.
      // (The pair's first CTA sees the copies of both.)
      volatile unsigned ignore = 0u;
      for (int k = 0; k < kStagesN && rank == 0; ++k) {
        if (pass == 0 && k >= s) continue;                  // never filled
        mbar_wait(full + 8u * k, (k < s ? pass : pass - 1) & 1u, &ignore, p.timeout_cycles);
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ---- products ----------------------------------------------------------------------------------
    // instruction descriptor: fp32 accumulator (bit 4), fp16 operands, MN-major operands (bits 15, 16),
    // N / 8 at bit 17, M / 16 at bit 24
    const uint32_t idesc0 = (1u << 4) | (static_cast<uint32_t>(BN >> 3) << 17) | (static_cast<uint32_t>(CG * kBM >> 4) << 24);
    // Operand descriptors in units of 16 bytes (version 1 at bit 46, swizzle at bits 61-63).
    // K-major: the k-block is one swizzled row (128 bytes; 64 with split operands), 8-row groups (stride offset)
    // 1024 (512) bytes apart, 16 values of k are 32 bytes.
    // MN-major, 128-byte swizzle: 64-column blocks of kBK * 128 bytes (leading offset), groups of 8 values of k
    // 1024 bytes apart (stride offset), 16 values of k are 2048 bytes.
    const uint64_t desc_k = (1ull << 46) | (1ull << 16) | (SPLIT ? (32ull << 32) | (4ull << 61) : (64ull << 32) | (2ull << 61));
    const uint64_t desc_mn = (1ull << 46) | (64ull << 32) | (2ull << 61) | (static_cast<uint64_t>(kBK * 8) << 16);
    int s = 0;
    uint32_t pass = 0, it = 0, acc = 0;                      // tiles, accumulators of the main products used so far
    for (long long t = first; t < p.tiles; t += step, ++it) {
      const Tile q = tile_of(p, t);
      const int K = q.mode == kGram ? p.n : p.m, n_kb = (K + kBK - 1) / kBK;
      if (SPLIT && it >= 2) mbar_wait(crossempty + 8u * (it & 1u), ((it >> 1) - 1) & 1u, abort_flag, p.timeout_cycles);
      const uint32_t cross = tmem + (2u + (it & 1u)) * BN;   // split operands only
      for (int kb = 0; kb < n_kb; ++kb) {
        const int in_fold = SPLIT ? kb % kFold : kb;
        const uint32_t buf = acc & 1u, use = acc >> 1;
        if (in_fold == 0 && use > 0) mbar_wait(accempty + 8u * buf, (use - 1) & 1u, abort_flag, p.timeout_cycles);
        const uint32_t d = tmem + buf * BN;
        mbar_wait(full + 8u * s, pass & 1u, abort_flag, p.timeout_cycles);
        tcn_after();
        const uint32_t base = ((ring + static_cast<uint32_t>(s) * kStageN) & 0x3ffffu) >> 4;
        const bool mn_a = a_is_mn(q, kb * kBK, BN), mn_b = b_is_mn(q, kb * kBK, BN);
        const uint32_t idesc = idesc0 | (mn_a ? 1u << 15 : 0u) | (mn_b ? 1u << 16 : 0u);
        const uint64_t desc_a = mn_a ? desc_mn : desc_k, desc_b = mn_b ? desc_mn : desc_k;
        const uint32_t step_a = mn_a ? 128u : 2u, step_b = mn_b ? 128u : 2u;
        const bool last = kb == n_kb - 1 || (SPLIT && in_fold == kFold - 1);
        if (elect_one_n()) {
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) {
            constexpr uint32_t op = kOperand >> 4;
            const uint64_t a_h = desc_a | static_cast<uint64_t>(base + step_a * k);
            if constexpr (SPLIT) {
              const uint64_t a_l = desc_a | static_cast<uint64_t>(base + op + step_a * k);
              const uint64_t b_h = desc_b | static_cast<uint64_t>(base + 2u * op + step_b * k);
              const uint64_t b_l = desc_b | static_cast<uint64_t>(base + 3u * op + step_b * k);
              umma_f16<CG>(d, a_h, b_h, idesc, (in_fold | k) ? 1u : 0u);
              // 2^-11 of the main term: an accumulator of their own for the whole of K, read once
              umma_f16<CG>(cross, a_l, b_h, idesc, (kb | k) ? 1u : 0u);
              umma_f16<CG>(cross, a_h, b_l, idesc, 1u);
            } else {
              const uint64_t b_h = desc_b | static_cast<uint64_t>(base + op + step_b * k);
              umma_f16<CG>(d, a_h, b_h, idesc, (in_fold | k) ? 1u : 0u);
            }
          }
          umma_commit_n<CG>(empty + 8u * s);
          if (last) umma_commit_n<CG>(accfull + 8u * buf);
        }
        __syncwarp();
        if (last) ++acc;
        if (++s == kStagesN) {
          s = 0;
          ++pass;
        }
      }
      if (__any_sync(0xffffffffu, *abort_flag != 0u)) break;
    }
    if (elect_one_n()) umma_commit_n<CG>(done);
    __syncwarp();
    volatile unsigned ignore = 0u;
    mbar_wait(done, 0u, &ignore, p.timeout_cycles);           // no product in flight when tensor memory is freed
  } else if (warp == 2) {
    // ---- loads of the units that the coefficients apply to --------------------------------------------
    if (elect_one_n()) {
      uint32_t it = 0, n = 0;                                  // n: units of each half so far
      bool ok = true;
      for (long long t = first; t < p.tiles && ok && !p.drop_loads; t += step, ++it) {
        const Tile q = tile_of(p, t);
        const int cur = q.step & 1, row = q.i * BN + row_in_tile;
        const bool x = q.mode == kUpdate, low = SPLIT || x;    // low: values and remainders
        const CUtensorMap* m_h = x ? &maps.xu_h[cur] : &maps.au_h;
        const CUtensorMap* m_l = x ? &maps.xu_l[SPLIT ? cur : 0] : &maps.au_l;      // remainders of X stay in place, unless operands
        ok = mbar_wait(inputs + 8u * (it & 1u), (it >> 1) & 1u, abort_flag, p.timeout_cycles);
        if (!ok) break;
        mbar_arrive(taken + 8u * (it & 1u));
        for (int u = 0; u < kUnits && ok; ++u, ++n) {
          const uint32_t place = n % kPlaces;
          for (uint32_t half = 0; half < 2; ++half) {
            const uint32_t k = half * kPlaces + place, at = epi_at + k * 2u * kUnitBytes, bar = ready + 8u * k;
            if (n >= kPlaces) ok = mbar_wait(freed + 8u * k, (n / kPlaces - 1u) & 1u, abort_flag, p.timeout_cycles);
            if (!ok) break;
            if (q.mode == kGram) {
              mbar_arrive(bar);
            } else {
              const int c = q.j * BN + static_cast<int>(half) * (BN / 2) + u * kUnitCols;
              mbar_expect_tx(bar, low ? 2u * kUnitBytes : kUnitBytes);
              tma_load_3d(at, m_h, c, row, q.z, bar);
              if (low) tma_load_3d(at + kUnitBytes, m_l, c, row, q.z, bar);
            }
          }
          if (!ok) break;
        }
      }
      if (!ok) {                                               // no load in flight when the CTA exits
        volatile unsigned ignore = 0u;
        for (uint32_t k = n > kPlaces ? n - kPlaces : 0u; k < n; ++k)
          for (uint32_t half = 0; half < 2; ++half)
            mbar_wait(ready + 8u * (half * kPlaces + k % kPlaces), (k / kPlaces) & 1u, &ignore, p.timeout_cycles);
        mbar_wait(ready + 8u * (n % kPlaces), (n / kPlaces) & 1u, &ignore, 100000);      // (the first half's, if it was asked for)
      }
    }
    __syncwarp();
  } else if (warp == 3 || warp == kLookout + 1) {
    // ---- stores of one half's units, announcements ----------------------------------------------------
    if (elect_one_n()) {
      const uint32_t half = warp == 3 ? 0u : 1u;
      uint32_t n = 0;
      bool ok = true;
      for (long long t = first; t < p.tiles && ok; t += step) {
        const Tile q = tile_of(p, t);
        const int nxt = (q.step & 1) ^ 1, row = q.i * BN + row_in_tile, col = q.j * BN + static_cast<int>(half) * (BN / 2);
        const bool x = q.mode == kUpdate, low = SPLIT || x;
        const CUtensorMap* o_h = q.mode == kGram ? &maps.au_h : q.mode == kPoly ? &maps.bu_h : &maps.xu_h[nxt];
        const CUtensorMap* o_l = q.mode == kGram ? &maps.au_l : q.mode == kPoly ? &maps.bu_l : &maps.xu_l[SPLIT ? nxt : 0];
        for (int u = 0; u < kUnits; ++u, ++n) {
          const uint32_t k = half * kPlaces + n % kPlaces, at = epi_at + k * 2u * kUnitBytes;
          ok = mbar_wait(filled + 8u * k, (n / kPlaces) & 1u, abort_flag, p.timeout_cycles);
          if (!ok) break;
          const int c = col + u * kUnitCols;
          tma_store_3d(o_h, at, c, row, q.z);
          if (low) tma_store_3d(o_l, at + kUnitBytes, c, row, q.z);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          mbar_arrive(freed + 8u * k);
        }
        if (!ok) break;
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        asm volatile("fence.acq_rel.gpu;" ::: "memory");       // the half tile, before its announcement
        unsigned* base = p.progress + static_cast<long long>(q.z) * 3 * p.row_blocks;
        if (x) {
          announce(base + q.i);
        } else {
          unsigned* c = base + (q.mode == kGram ? 1 : 2) * p.row_blocks;
          announce(c + q.i);
          if (q.j < q.i) announce(c + q.j);
        }
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
  } else if (warp == kLookout) {
    // ---- waits for the inputs of the tile after the one that is being loaded -----------------------------
    if (elect_one_n()) {
      uint32_t it = 0;
      for (long long t = first; t < p.tiles && !p.drop_loads; t += step, ++it) {
        const Tile q = tile_of(p, t);
        if (it >= 2 && !mbar_wait(taken + 8u * (it & 1u), ((it >> 1) - 1) & 1u, abort_flag, p.timeout_cycles)) break;
        if (!wait_inputs<CG>(p, q, abort_flag)) break;
        mbar_arrive(inputs + 8u * (it & 1u));
      }
    }
    __syncwarp();
  } else if (warp >= kFirstEpi && warp < kLookout) {        // (warp 1 of a pair's second CTA has nothing to do)
    // ---- epilogue: a thread owns a row of the tile and 32 columns of it at a time -----------------------
    const int q4 = warp & 3;
    const uint32_t half = static_cast<uint32_t>(warp - kFirstEpi) >> 2;
    const uint32_t row = static_cast<uint32_t>(q4 * 32 + lane);
    const uint32_t sw64 = (row >> 1) & 3u;                     // swizzle of rows of 64 bytes
    const uint32_t t_row = tmem + half * (BN / 2) + (static_cast<uint32_t>(q4 * 32) << 16);
    const uint32_t accempty0 = CG == 2 ? map_to_rank(accempty, 0) : accempty;
    auto hand_back = [&](uint32_t buf) {                      // this warp has read its part of the accumulator
      tcn_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2) mbar_arrive_cluster(accempty0 + 8u * buf);
        else mbar_arrive(accempty + 8u * buf);
      }
    };
    uint32_t it = 0, acc = 0, n = 0;                          // n: units so far
    bool ok = true;
    for (long long t = first; t < p.tiles && ok; t += step, ++it) {
      const Tile q = tile_of(p, t);
      const NsCoef coef = p.coef[q.step][q.mode];
      const uint64_t c_in = pack_f32x2(coef.in, coef.in), c_acc = pack_f32x2(coef.acc, coef.acc);
      uint32_t r[2][32];                                      // accumulator columns: this unit's and the next one's
      float sum[SPLIT ? kUnits : 1][32];
      if constexpr (SPLIT) {
        const int K = q.mode == kGram ? p.n : p.m, n_kb = (K + kBK - 1) / kBK, folds = (n_kb + kFold - 1) / kFold;
#pragma unroll
        for (int k = 0; k < kUnits; ++k)
#pragma unroll
          for (int e = 0; e < 32; ++e) sum[k][e] = 0.f;
        for (int f = 0; f <= folds && ok; ++f) {              // the last round adds the cross terms
          const bool main = f < folds;
          if (main) {
            ok = __all_sync(0xffffffffu, mbar_wait(accfull + 8u * (acc & 1u), (acc >> 1) & 1u, abort_flag, p.timeout_cycles));
            if (!ok) break;
            tcn_after();
          }
          const uint32_t at = t_row + (main ? acc & 1u : 2u + (it & 1u)) * BN;
#pragma unroll
          for (int k = 0; k < kUnits; ++k) tmem_ld32(at + k * kUnitCols, r[k]);
#pragma unroll
          for (int k = 0; k < kUnits; ++k) {
            tmem_wait(r[k]);
#pragma unroll
            for (int e = 0; e < 32; ++e) sum[k][e] += __uint_as_float(r[k][e]);
          }
          if (main) {
            hand_back(acc & 1u);
            ++acc;
          } else {
            tcn_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(crossempty + 8u * (it & 1u));
          }
        }
        if (!ok) break;
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait(accfull + 8u * (it & 1u), (it >> 1) & 1u, abort_flag, p.timeout_cycles));
        if (!ok) break;
        tcn_after();
        tmem_ld32(t_row + (it & 1u) * BN, r[0]);
      }
      const bool low = SPLIT || q.mode == kUpdate;            // values and remainders
#pragma unroll
      for (int u = 0; u < kUnits; ++u, ++n) {
        const uint32_t place = half * kPlaces + n % kPlaces, h_at = epi_at + place * 2u * kUnitBytes + row * 64u;
        ok = ok && __all_sync(0xffffffffu, mbar_wait(ready + 8u * place, (n / kPlaces) & 1u, abort_flag, p.timeout_cycles));
        uint64_t v[16];                                       // pairs of results
        if constexpr (!SPLIT) tmem_wait(r[u & 1]);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (SPLIT) v[e] = mul_f32x2(c_acc, pack_f32x2(sum[u][2 * e], sum[u][2 * e + 1]));
          else v[e] = mul_f32x2(c_acc, pack_f32x2(__uint_as_float(r[u & 1][2 * e]), __uint_as_float(r[u & 1][2 * e + 1])));
        }
        if constexpr (!SPLIT) {
          if (u + 1 < kUnits) tmem_ld32(t_row + (it & 1u) * BN + (u + 1) * kUnitCols, r[(u + 1) & 1]);
          else hand_back(it & 1u);
        }
        if (q.mode != kGram) {
          uint4 h4[4], l4[4];
#pragma unroll
          for (uint32_t c = 0; c < 4; ++c) h4[c] = lds128(h_at + ((c ^ sw64) << 4));
          if (low) {
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) l4[c] = lds128(h_at + kUnitBytes + ((c ^ sw64) << 4));
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint4 l = l4[e >> 2];
              const float2 y = unpack_half2((e & 3) == 0 ? l.x : (e & 3) == 1 ? l.y : (e & 3) == 2 ? l.z : l.w);
              v[e] = fma_f32x2(c_in, pack_f32x2(y.x, y.y), v[e]);
            }
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint4 h = h4[e >> 2];
            const float2 x = unpack_half2((e & 3) == 0 ? h.x : (e & 3) == 1 ? h.y : (e & 3) == 2 ? h.z : h.w);
            v[e] = fma_f32x2(c_in, pack_f32x2(x.x, x.y), v[e]);
          }
        }
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 w = unpack_f32x2(v[4 * c + e]);
            h[e] = pack_half2(w.x, w.y);
          }
          sts128_n(h_at + ((c ^ sw64) << 4), h);
          if (low) {
            uint32_t l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 w = unpack_f32x2(v[4 * c + e]), f = unpack_half2(h[e]);
              l[e] = pack_half2(w.x - f.x, w.y - f.y);
            }
            sts128_n(h_at + kUnitBytes + ((c ^ sw64) << 4), l);
          }
        }
        fence_async_n();
        __syncwarp();
        if (lane == 0) mbar_arrive(filled + 8u * place);
      }
    }
  }
  __syncwarp();
  tcn_before();
  __syncthreads();
  if (tid == 0 && *abort_flag) atomicOr(p.flag, 1u);
  // neither CTA of a pair leaves while the other may still use its barriers or tensor memory
  if constexpr (CG == 2) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  if (warp == 1) {
    tcn_after();
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------------------
// [Z][rows][cols] fp16 matrices with boxes of [box_rows][box_cols]; what lies outside reads as zero and is not written.
bool encode_half_map(const __half* base, int Z, int rows, int cols, long long ld, int box_rows, int box_cols,
                     CUtensorMapSwizzle swizzle, CUtensorMap* map) {
  const cuuint64_t gdim[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(Z)};
  const cuuint64_t gstr[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * 2 * rows};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 1u};
  const cuuint32_t estr[3] = {1u, 1u, 1u};
  return encode_tiled_fn()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), gdim, gstr, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, bool SPLIT>
int launch_steps(abs_ctx* ctx, const NsBuffers& w, NsStepsParams& p, cudaStream_t st) {
  constexpr int bk = SPLIT ? 32 : 64;
  const CUtensorMapSwizzle sk = SPLIT ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
  const CUtensorMapSwizzle s128 = CU_TENSOR_MAP_SWIZZLE_128B, s64 = CU_TENSOR_MAP_SWIZZLE_64B;
  NsMaps maps;
  bool ok = true;
  for (int k = 0; k < 2; ++k) {
    ok = ok && encode_half_map(w.xh[k], w.Z, w.m, w.n, w.ldx, kBM, bk, sk, &maps.xk_h[k]);
    ok = ok && encode_half_map(w.xh[k], w.Z, w.m, w.n, w.ldx, bk, 64, s128, &maps.xm_h[k]);
    ok = ok && encode_half_map(w.xh[k], w.Z, w.m, w.n, w.ldx, kBM, kUnitCols, s64, &maps.xu_h[k]);
    if (SPLIT) {
      ok = ok && encode_half_map(w.xl[k], w.Z, w.m, w.n, w.ldx, kBM, bk, sk, &maps.xk_l[k]);
      ok = ok && encode_half_map(w.xl[k], w.Z, w.m, w.n, w.ldx, bk, 64, s128, &maps.xm_l[k]);
    }
    if (SPLIT || k == 0) ok = ok && encode_half_map(w.xl[k], w.Z, w.m, w.n, w.ldx, kBM, kUnitCols, s64, &maps.xu_l[k]);
  }
  for (int k = 0; k < (SPLIT ? 2 : 1); ++k) {
    const __half *A = k ? w.al : w.ah, *B = k ? w.bl : w.bh;
    ok = ok && encode_half_map(A, w.Z, w.m, w.m, w.ldm, kBM, bk, sk, k ? &maps.ak_l : &maps.ak_h);
    ok = ok && encode_half_map(B, w.Z, w.m, w.m, w.ldm, kBM, bk, sk, k ? &maps.bk_l : &maps.bk_h);
    ok = ok && encode_half_map(A, w.Z, w.m, w.m, w.ldm, bk, 64, s128, k ? &maps.am_l : &maps.am_h);
    ok = ok && encode_half_map(B, w.Z, w.m, w.m, w.ldm, bk, 64, s128, k ? &maps.bm_l : &maps.bm_h);
    ok = ok && encode_half_map(A, w.Z, w.m, w.m, w.ldm, kBM, kUnitCols, s64, k ? &maps.au_l : &maps.au_h);
    ok = ok && encode_half_map(B, w.Z, w.m, w.m, w.ldm, kBM, kUnitCols, s64, k ? &maps.bu_l : &maps.bu_h);
  }
  if (!ok) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled (matrices of %d x %d) failed", w.m, w.n);
  constexpr int side = 128 * CG;
  p.row_blocks = (w.m + side - 1) / side;
  p.col_tiles = (w.n + side - 1) / side;
  p.tri = p.row_blocks * (p.row_blocks + 1) / 2;
  p.per_step = static_cast<long long>(w.Z) * (2ll * p.tri + static_cast<long long>(p.row_blocks) * p.col_tiles);
  p.tiles = p.per_step * p.steps;

  const size_t smem = kSmemN;
  auto kern = ns_steps_kernel<CG, SPLIT>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  const long long widest = static_cast<long long>(w.Z) * p.row_blocks * (p.row_blocks > p.col_tiles ? p.row_blocks : p.col_tiles);
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeCooperative;
  attrs[0].val.cooperative = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = CG;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  lc.blockDim = dim3(kThreadsN);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  lc.attrs = attrs;
  lc.numAttrs = CG == 2 ? 2 : 1;
  long long resident = ctx->sm_count / CG;
  if (CG == 2) {
    const void* f = reinterpret_cast<const void*>(kern);
    const int slot = ctx->fn_cache.slot(f);
    if (slot >= 0 && ctx->fn_cache.max_clusters[slot] > 0) {
      resident = ctx->fn_cache.max_clusters[slot];
    } else {
      lc.gridDim = dim3(static_cast<unsigned>(resident) * CG);
      int clusters = 0;
      ABS_CUDA_TRY(ctx, cudaOccupancyMaxActiveClusters(&clusters, f, &lc));
      if (clusters < 1) return set_error(ctx, ABS_ERR_UNSUPPORTED, "the device cannot hold a pair of CTAs");
      if (clusters < resident) resident = clusters;
      if (slot >= 0) ctx->fn_cache.max_clusters[slot] = static_cast<int>(resident);
    }
  }
  const long long grid = widest < resident ? widest : resident;
  lc.gridDim = dim3(static_cast<unsigned>(grid) * CG);
  ABS_CUDA_TRY(ctx, cudaLaunchKernelEx(&lc, kern, maps, p));
  return ABS_OK;
}

}  // namespace

int launch_ns_steps(abs_ctx* ctx, const NsBuffers& w, int steps, float a, float b, float c, const NsScales& sc, bool split,
                    cudaStream_t st) {
  if (encode_tiled_fn() == nullptr) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  NsStepsParams p = {};
  p.Z = w.Z; p.m = w.m; p.n = w.n; p.steps = steps;
  p.progress = w.progress;
  p.flag = ctx->flags + kNsFlagWord;
  p.timeout_cycles = ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles;
  p.drop_loads = ctx->tuning.stats_fault_drop_loads ? 1 : 0;
  for (int k = 0; k < steps; ++k) ns_coefs(p.coef[k], a, b, c, sc, k);
  if (split) return launch_steps<1, true>(ctx, w, p, st);
  // Single CTAs or pairs.  A pair's 256 x 256 tile takes about as long as a single CTA's 128 x 128 (each is bound by
  // what its SMs fetch), so a step of T1 or T2 tiles takes T1 / 148 or T2 / 74 of that time: pairs are up to twice as fast, less
  // what the last row and column blocks pad.  A larger tile has the longer epilogue, which counts where matrices are small
  // or few.  us a step, pairs and single CTAs (T1 / T2): 4096 x 4096 221, 353 (3.94); 2000 x 1500 40, 50 (3.87); 8 of
  // 1024 x 1024 38, 48 (3.78); 14 of 768 x 768 33, 39 (3.71); 24 of 256 x 1024 24, 22 and of 200 x 1000 25, 22 (3.67);
  // 16 of 512 x 512 25, 24 (3.6); 8 of 784 x 1024 44, 43 (3.1); 64 of 300 x 520 54, 38 (2.25); and with fewer tiles than pairs
  // 1024 x 1024 40, 29.
  // The limit of 3.7 is right for a few waves of tiles.  With many, pairs are better below it too, the more so the longer the
  // products are, and this rule, which knows neither, gives these to single CTAs: 112 of 256 x 1024 61, 64, of 512 x 512 96, 117 and
  // 24 of 784 x 1024 88, 135.
  auto tiles = [&](long long side) {
    const long long rb = (w.m + side - 1) / side, cb = (w.n + side - 1) / side;
    return w.Z * (rb * (rb + 1) + rb * cb);
  };
  const long long t1 = tiles(128), t2 = tiles(256);
  const bool pairs = ctx->tuning.ns_pair_tiles ? ctx->tuning.ns_pair_tiles == 2 : 10 * t1 > 37 * t2 && 2 * t2 >= ctx->sm_count;
  return pairs ? launch_steps<2, false>(ctx, w, p, st) : launch_steps<1, false>(ctx, w, p, st);
}

}  // namespace absk
