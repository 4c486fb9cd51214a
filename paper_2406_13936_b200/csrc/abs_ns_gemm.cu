// The three products of a Newton-Schulz step on the tcgen05 tensor cores, batched over matrices:
//   kGram    A = X X'                      both operands K-major rows of X, result symmetric
//   kPoly    B = b A + c A A               both operands K-major rows of A (A = A'), result symmetric
//   kUpdate  X <- a X + B X                B K-major, X MN-major (its rows are the k index)
// Symmetric results are computed for tiles on and below the diagonal and written to both places.
//
// CTA: warp 0 loads tiles by TMA (128-byte swizzle) into a ring of stages, warp 1 issues the
// products (M = 128, fp32 accumulators in tensor memory, two of them so that the next tile's products
// run while this one is read back), warps 4-11 read back, apply the step's coefficients and store.
// A persistent grid walks the tiles.  All waits are bounded; one that runs out raises the CTA's abort
// flag, every role falls through, tensor memory is freed and the context's time-out word is set.
#include "abs_ns.cuh"
#include "abs_pipeline.cuh"

namespace absk {
namespace {

enum { kGram = 0, kPoly = 1, kUpdate = 2 };

constexpr int kBM = 128;                     // tile rows
constexpr int kBK = 64;                      // k-block: 64 fp16 = one 128-byte swizzled row
constexpr int kEpiWarpsN = 8;
constexpr int kFirstEpi = 4;
constexpr int kThreadsN = (kFirstEpi + kEpiWarpsN) * 32;   // 384
constexpr uint32_t kABytes = kBM * 128;

struct NsGemmParams {
  int mode;
  int Z, m, n;                // n: columns of the result (m for the symmetric products)
  int K;
  long long tiles;            // tiles in all
  int row_tiles, col_tiles, tiles_per_matrix;
  const __half* in_h;         // the matrix that the epilogue reads: A (kPoly), X (kUpdate)
  const __half* in_l;
  __half* out_h;
  __half* out_l;
  long long ld;               // of in and out
  long long zs;               // elements from one matrix of in / out to the next
  float c_in, c_acc;          // out = c_in * in + c_acc * accumulator
  unsigned* flag;
  long long timeout_cycles;
  int drop_loads;             // test hook: nothing is loaded, so every wait must run out
};

__device__ __forceinline__ void fence_async_n() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_n(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// Waits (bounded) until every copy that was issued has arrived, so that none is in flight when the CTA
// exits, whatever made the other roles stop.  (s, pass): the stage that would have been filled next.
__device__ __forceinline__ void drain_loads(uint32_t full, int stages, int s, uint32_t pass, long long limit) {
  volatile unsigned ignore = 0u;
  for (int k = 0; k < stages; ++k) {
    const int stage = k;
    if (pass == 0 && stage >= s) continue;                      // never filled
    const uint32_t last = stage < s ? pass : pass - 1;           // the pass that filled it last
    mbar_wait(full + 8u * stage, last & 1u, &ignore, limit);
  }
}

// Tile t of one matrix: symmetric results number the tiles on and below the diagonal row by row.
__device__ __forceinline__ void tile_of(const NsGemmParams& p, long long t, int bn, int& z, int& i, int& j) {
  z = static_cast<int>(t / p.tiles_per_matrix);
  int r = static_cast<int>(t - static_cast<long long>(z) * p.tiles_per_matrix);
  if (p.mode == kUpdate) {
    i = r / p.col_tiles;
    j = r - i * p.col_tiles;
    return;
  }
  i = 0;
  for (;;) {                                    // at most m / 128 rounds
    const int in_row = i * kBM / bn + 1;        // column tiles that start at or left of the diagonal block
    if (r < in_row) break;
    r -= in_row;
    ++i;
  }
  j = r;
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// Stores 8 results of row r from column c on, as fp16 values and, where out_l is given, remainders.
__device__ __forceinline__ void store8(const NsGemmParams& p, __half* oh, __half* ol, const float* v) {
  uint32_t h[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) h[q] = pack_half2(v[2 * q], v[2 * q + 1]);
  *reinterpret_cast<uint4*>(oh) = make_uint4(h[0], h[1], h[2], h[3]);
  if (ol != nullptr) {
    uint32_t l[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 f = unpack_half2(h[q]);
      l[q] = pack_half2(v[2 * q] - f.x, v[2 * q + 1] - f.y);
    }
    *reinterpret_cast<uint4*>(ol) = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// 32 accumulator values of row r, columns c .. c + 31 of matrix z: coefficients, stores, mirror.
template <bool SPLIT>
__device__ __forceinline__ void finish32(const NsGemmParams& p, int z, int r, int c, float (&v)[32], bool mirror) {
  const int cols = p.n;
  const bool symmetric = p.mode != kUpdate;
  const long long off = z * p.zs + static_cast<long long>(r) * p.ld + c;
  const bool live = r < p.m;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (!live || c + 8 * q >= cols) continue;            // ld is a multiple of 8: a piece never leaves its row
    float* w = v + 8 * q;
    if (p.mode == kGram) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] *= p.c_acc;
    } else {
      const uint4 h = *reinterpret_cast<const uint4*>(p.in_h + off + 8 * q);
      const uint32_t hh[4] = {h.x, h.y, h.z, h.w};
      uint32_t ll[4] = {0u, 0u, 0u, 0u};
      if (SPLIT || p.mode == kUpdate) {
        const uint4 l = *reinterpret_cast<const uint4*>(p.in_l + off + 8 * q);
        ll[0] = l.x; ll[1] = l.y; ll[2] = l.z; ll[3] = l.w;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 a = unpack_half2(hh[e]), b = unpack_half2(ll[e]);
        w[2 * e] = fmaf(p.c_acc, w[2 * e], p.c_in * (a.x + b.x));
        w[2 * e + 1] = fmaf(p.c_acc, w[2 * e + 1], p.c_in * (a.y + b.y));
      }
    }
    store8(p, p.out_h + off + 8 * q, (SPLIT || p.mode == kUpdate) ? p.out_l + off + 8 * q : nullptr, w);
  }
  if (symmetric && mirror && live) {
    __half* th = p.out_h + z * p.zs + r;
    __half* tl = SPLIT ? p.out_l + z * p.zs + r : nullptr;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      if (c + e >= cols) continue;
      const __half h = __float2half_rn(v[e]);
      th[static_cast<long long>(c + e) * p.ld] = h;
      if (SPLIT) tl[static_cast<long long>(c + e) * p.ld] = __float2half_rn(v[e] - __half2float(h));
    }
  }
}

// The epilogue works through a tile in pieces of 32 columns: kPieces buffers of 16 KB in shared memory,
// each two halves of 8 KB: what is read and written in place (fp16 values; remainders for kUpdate) or,
// for a symmetric result, the values and their mirror image.  One thread of warp 2 moves the pieces by
// TMA: it stores a finished piece, waits until the store has read the buffer, and loads the piece that
// takes its place.
constexpr int kPieces = 4;
constexpr int kPieceCols = 32;
constexpr uint32_t kHalfPiece = kBM * kPieceCols * 2;      // 8 KB
constexpr uint32_t kPieceBytes = 2 * kHalfPiece;

struct NsMaps {
  CUtensorMap a, b;            // operands
  CUtensorMap in_h, in_l;      // pieces of the matrix that the epilogue reads, 64-byte swizzle
  CUtensorMap out_h, out_l;    // pieces of the result, 64-byte swizzle
  CUtensorMap mirror;          // transposed pieces of a symmetric result, no swizzle
};

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src),
               "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void sts128_n(uint32_t addr, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void sts16_n(uint32_t addr, __half h) {
  asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"(__half_as_ushort(h)) : "memory");
}

// BN: tile columns.  B_MN: the second operand is MN-major (kUpdate).
template <int BN, int MODE>
__global__ void __launch_bounds__(kThreadsN, 1)
ns_gemm_kernel(const __grid_constant__ NsMaps maps, const NsGemmParams p) {
  constexpr bool B_MN = MODE == kUpdate;
  constexpr uint32_t kBBytes = BN * 128;
  constexpr uint32_t kStage = kABytes + kBBytes;
  constexpr int kStages = BN == 256 ? 3 : 5;
  constexpr int kTilePieces = BN / kPieceCols;
  extern __shared__ unsigned char smem_dyn[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = smem_u32(smem_dyn), ring = (raw + 1023u) & ~1023u;
  const uint32_t pieces = ring + kStages * kStage;
  unsigned char* tail = smem_dyn + (ring - raw) + static_cast<size_t>(kStages) * kStage + kPieces * kPieceBytes;
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(tail);
  constexpr int kBars = 2 * kStages + 5 + 2 * kPieces;
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + kBars);
  unsigned* tmem_slot = const_cast<unsigned*>(abort_flag) + 1;
  const uint32_t full = smem_u32(bars), empty = full + 8u * kStages, accfull = empty + 8u * kStages,
                 accempty = accfull + 16u, done = accempty + 16u, ready = done + 8u, filled = ready + 8u * kPieces;
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8u * s, 1);
      mbar_init(empty + 8u * s, 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(accfull + 8u * k, 1);
      mbar_init(accempty + 8u * k, kEpiWarpsN * 32);
    }
    mbar_init(done, 1);
    for (int k = 0; k < kPieces; ++k) {
      mbar_init(ready + 8u * k, 1);                      // the buffer is loaded (or free)
      mbar_init(filled + 8u * k, kEpiWarpsN * 32);       // the piece is finished
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(static_cast<uint32_t>(2 * BN))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcn_before();
  __syncthreads();
  tcn_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();
  const int n_kb = (p.K + kBK - 1) / kBK;
  const long long step = gridDim.x;

  if (warp == 0) {
    // ---- operand loads ---------------------------------------------------------------------------
    if (elect_one_n()) {
      int s = 0;
      uint32_t pass = 0;
      for (long long t = blockIdx.x; t < p.tiles && !p.drop_loads; t += step) {
        int z, i, j;
        tile_of(p, t, BN, z, i, j);
        for (int kb = 0; kb < n_kb; ++kb) {
          if (pass > 0 && !mbar_wait(empty + 8u * s, (pass - 1) & 1u, abort_flag, p.timeout_cycles)) break;
          const uint32_t st = ring + static_cast<uint32_t>(s) * kStage;
          mbar_expect_tx(full + 8u * s, kStage);
          tma_load_3d(st, &maps.a, kb * kBK, i * kBM, z, full + 8u * s);
          if (B_MN) {
#pragma unroll
            for (int q = 0; q < BN / 64; ++q)      // blocks of [64 values of k] x [64 columns]
              tma_load_3d(st + kABytes + q * 8192u, &maps.b, j * BN + q * 64, kb * kBK, z, full + 8u * s);
          } else {
            tma_load_3d(st + kABytes, &maps.b, kb * kBK, j * BN, z, full + 8u * s);
          }
          if (++s == kStages) {
            s = 0;
            ++pass;
          }
        }
        if (*abort_flag) break;
      }
      drain_loads(full, kStages, s, pass, p.timeout_cycles);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- products ----------------------------------------------------------------------------------
    const uint32_t idesc = (1u << 4) | (B_MN ? (1u << 16) : 0u) | (static_cast<uint32_t>(BN >> 3) << 17) |
                           (static_cast<uint32_t>(kBM >> 4) << 24);
    // K-major, 128-byte swizzle: 8-row groups 1024 bytes apart, 16 values of k are 32 bytes.
    // MN-major, 128-byte swizzle: 64-column blocks 8192 bytes apart (leading offset), groups of 8
    // values of k 1024 bytes apart (stride offset), 16 values of k are 2048 bytes.
    const uint64_t desc_k = (64ull << 32) | (1ull << 46) | (2ull << 61) | (1ull << 16);
    const uint64_t desc_mn = (64ull << 32) | (1ull << 46) | (2ull << 61) | (512ull << 16);
    int s = 0;
    uint32_t pass = 0, it = 0;
    for (long long t = blockIdx.x; t < p.tiles; t += step, ++it) {
      const uint32_t buf = it & 1u, use = it >> 1;
      if (use > 0) mbar_wait(accempty + 8u * buf, (use - 1) & 1u, abort_flag, p.timeout_cycles);
      tcn_after();
      const uint32_t d = tmem + buf * BN;
      for (int kb = 0; kb < n_kb; ++kb) {
        mbar_wait(full + 8u * s, pass & 1u, abort_flag, p.timeout_cycles);
        tcn_after();
        const uint32_t base = ((ring + static_cast<uint32_t>(s) * kStage) & 0x3ffffu) >> 4;
        if (elect_one_n()) {
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) {
            const uint64_t da = desc_k | static_cast<uint64_t>(base + 2u * k);
            const uint64_t db = B_MN ? desc_mn | static_cast<uint64_t>(base + (kABytes >> 4) + 128u * k)
                                     : desc_k | static_cast<uint64_t>(base + (kABytes >> 4) + 2u * k);
            umma_f16(d, da, db, idesc, (kb | k) ? 1u : 0u);
          }
          umma_commit_n(empty + 8u * s);
          if (kb == n_kb - 1) umma_commit_n(accfull + 8u * buf);
        }
        __syncwarp();
        if (++s == kStages) {
          s = 0;
          ++pass;
        }
      }
      if (__any_sync(0xffffffffu, *abort_flag != 0u)) break;
    }
    if (elect_one_n()) umma_commit_n(done);
    __syncwarp();
    volatile unsigned ignore = 0u;
    mbar_wait(done, 0u, &ignore, p.timeout_cycles);           // no product in flight when tensor memory is freed
  } else if (warp == 2) {
    // ---- pieces of the epilogue: store the finished one, load the one that takes its buffer ---------
    if (elect_one_n()) {
      long long t_in = blockIdx.x;                             // the piece that is loaded next
      int piece_in = 0;
      uint32_t issued = 0;
      auto load_next = [&](uint32_t b) {
        if (t_in >= p.tiles) return;
        int z, i, j;
        tile_of(p, t_in, BN, z, i, j);
        const uint32_t at = pieces + b * kPieceBytes, bar = ready + 8u * b;
        const int c = j * BN + piece_in * kPieceCols;
        if (MODE == kGram || p.drop_loads) {
          mbar_arrive(bar);
        } else {
          mbar_expect_tx(bar, MODE == kUpdate ? kPieceBytes : kHalfPiece);
          tma_load_3d(at, &maps.in_h, c, i * kBM, z, bar);
          if (MODE == kUpdate) tma_load_3d(at + kHalfPiece, &maps.in_l, c, i * kBM, z, bar);
        }
        ++issued;
        if (++piece_in == kTilePieces) {
          piece_in = 0;
          t_in += step;
        }
      };
      for (uint32_t b = 0; b < kPieces; ++b) load_next(b);
      uint32_t n = 0;                                          // pieces stored so far
      for (long long t = blockIdx.x; t < p.tiles; t += step) {
        int z, i, j;
        tile_of(p, t, BN, z, i, j);
        bool ok = true;
        for (int piece = 0; piece < kTilePieces && ok; ++piece, ++n) {
          const uint32_t b = n % kPieces;
          ok = mbar_wait(filled + 8u * b, (n / kPieces) & 1u, abort_flag, p.timeout_cycles);
          if (!ok) break;
          const uint32_t at = pieces + b * kPieceBytes;
          const int c = j * BN + piece * kPieceCols;
          tma_store_3d(&maps.out_h, at, c, i * kBM, z);
          if (MODE == kUpdate) tma_store_3d(&maps.out_l, at + kHalfPiece, c, i * kBM, z);
          else if (c / kBM < i) tma_store_3d(&maps.mirror, at + kHalfPiece, i * kBM, c, z);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          load_next(b);
        }
        if (!ok) break;
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      // no load in flight when the CTA exits (buffers are loaded in turn)
      volatile unsigned ignore = 0u;
      for (uint32_t b = 0; b < kPieces && b < issued; ++b) {
        const uint32_t last = (issued - 1 - b) / kPieces;      // passes of buffer b, minus one
        mbar_wait(ready + 8u * b, last & 1u, &ignore, p.timeout_cycles);
      }
    }
    __syncwarp();
  } else if (warp >= kFirstEpi) {
    // ---- epilogue: lanes are rows; the two warps of a quarter take 16 of a piece's 32 columns each ---
    const int q = warp & 3, part = (warp - kFirstEpi) >> 2;
    const uint32_t row = static_cast<uint32_t>(q * 32 + lane), sw = (row >> 1) & 3u;
    uint32_t it = 0, n = 0;
    bool ok = true;
    for (long long t = blockIdx.x; t < p.tiles && ok; t += step, ++it) {
      const uint32_t buf = it & 1u, use = it >> 1;
      ok = __all_sync(0xffffffffu, mbar_wait(accfull + 8u * buf, use & 1u, abort_flag, p.timeout_cycles));
      if (!ok) break;
      tcn_after();
      const uint32_t taddr = tmem + buf * BN + static_cast<uint32_t>(part * 16) + (static_cast<uint32_t>(q * 32) << 16);
#pragma unroll 1
      for (int piece = 0; piece < kTilePieces; ++piece, ++n) {
        const uint32_t b = n % kPieces;
        float v[16];
        tmem_ld16(taddr + static_cast<uint32_t>(piece * kPieceCols), v);
        if (piece == kTilePieces - 1) {                        // the accumulator is in registers: hand it back
          tcn_before();
          mbar_arrive(accempty + 8u * buf);
        }
        ok = __all_sync(0xffffffffu, mbar_wait(ready + 8u * b, (n / kPieces) & 1u, abort_flag, p.timeout_cycles));
        if (!ok) break;
        const uint32_t at = pieces + b * kPieceBytes;
#pragma unroll
        for (int g = 0; g < 2; ++g) {                          // 8 columns: one 16-byte chunk
          const uint32_t chunk = static_cast<uint32_t>(part * 2 + g);
          const uint32_t addr = at + row * 64u + ((chunk ^ sw) << 4);
          float* w = v + 8 * g;
          if (MODE == kGram) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] *= p.c_acc;
          } else {
            const uint4 h = lds128(addr);
            const uint32_t hh[4] = {h.x, h.y, h.z, h.w};
            uint4 l = make_uint4(0u, 0u, 0u, 0u);
            if (MODE == kUpdate) l = lds128(addr + kHalfPiece);
            const uint32_t ll[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 x = unpack_half2(hh[e]), y = unpack_half2(ll[e]);
              w[2 * e] = fmaf(p.c_acc, w[2 * e], p.c_in * (x.x + y.x));
              w[2 * e + 1] = fmaf(p.c_acc, w[2 * e + 1], p.c_in * (x.y + y.y));
            }
          }
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = pack_half2(w[2 * e], w[2 * e + 1]);
          sts128_n(addr, h);
          if (MODE == kUpdate) {
            uint32_t l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = unpack_half2(h[e]);
              l[e] = pack_half2(w[2 * e] - f.x, w[2 * e + 1] - f.y);
            }
            sts128_n(addr + kHalfPiece, l);
          } else {                                             // mirror image: row = column, 256 bytes a row
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t base = at + kHalfPiece + (chunk * 8u + 2u * e) * 256u + row * 2u;
              const __half2 hv = *reinterpret_cast<const __half2*>(&h[e]);
              sts16_n(base, __low2half(hv));
              sts16_n(base + 256u, __high2half(hv));
            }
          }
        }
        fence_async_n();
        mbar_arrive(filled + 8u * b);
      }
    }
  }
  tcn_before();
  __syncthreads();
  if (warp == 1) {
    tcn_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(static_cast<uint32_t>(2 * BN))
                 : "memory");
  }
  if (tid == 0 && *abort_flag) atomicOr(p.flag, 1u);
}

// ---- split operands: hi hi + hi lo + lo hi ------------------------------------------------------
// One 128 x 128 tile per CTA.  The tensor core adds without rounding to nearest, so an accumulator of
// the main products takes kFold k-blocks (4 kFold additions) before the epilogue warps add it, rounded to nearest, to running sums in registers; two of them alternate.
// The cross terms (2^-11 of the main one) have an accumulator of their own for the whole of K.
constexpr int kFold = 4;
constexpr int kSplitStages = 3;
constexpr uint32_t kSplitStage = 4 * kABytes;

template <bool B_MN>
__global__ void __launch_bounds__(kThreadsN, 1)
ns_gemm_split_kernel(const __grid_constant__ CUtensorMap map_ah, const __grid_constant__ CUtensorMap map_al,
                     const __grid_constant__ CUtensorMap map_bh, const __grid_constant__ CUtensorMap map_bl,
                     const NsGemmParams p) {
  constexpr int BN = 128;
  extern __shared__ unsigned char smem_dyn[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = smem_u32(smem_dyn), ring = (raw + 1023u) & ~1023u;
  unsigned char* tail = smem_dyn + (ring - raw) + static_cast<size_t>(kSplitStages) * kSplitStage;
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(tail);
  volatile unsigned* abort_flag = reinterpret_cast<volatile unsigned*>(bars + 2 * kSplitStages + 5);
  unsigned* tmem_slot = const_cast<unsigned*>(abort_flag) + 1;
  const uint32_t full = smem_u32(bars), empty = full + 8u * kSplitStages, accfull = empty + 8u * kSplitStages,
                 accempty = accfull + 16u, done = accempty + 16u;
  if (tid == 0) {
    for (int s = 0; s < kSplitStages; ++s) {
      mbar_init(full + 8u * s, 1);
      mbar_init(empty + 8u * s, 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(accfull + 8u * k, 1);
      mbar_init(accempty + 8u * k, kEpiWarpsN * 32);
    }
    mbar_init(done, 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcn_before();
  __syncthreads();
  tcn_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();
  const int n_kb = (p.K + kBK - 1) / kBK;
  const int n_fold = (n_kb + kFold - 1) / kFold;
  int z, i, j;
  tile_of(p, blockIdx.x, BN, z, i, j);

  if (warp == 0) {
    if (elect_one_n()) {
      int kb = 0;
      for (; kb < n_kb && !p.drop_loads; ++kb) {
        const int s = kb % kSplitStages;
        const uint32_t pass = static_cast<uint32_t>(kb / kSplitStages);
        if (pass > 0 && !mbar_wait(empty + 8u * s, (pass - 1) & 1u, abort_flag, p.timeout_cycles)) break;
        const uint32_t st = ring + static_cast<uint32_t>(s) * kSplitStage, bar = full + 8u * s;
        mbar_expect_tx(bar, kSplitStage);
        tma_load_3d(st, &map_ah, kb * kBK, i * kBM, z, bar);
        tma_load_3d(st + kABytes, &map_al, kb * kBK, i * kBM, z, bar);
        if (B_MN) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            tma_load_3d(st + 2 * kABytes + q * 8192u, &map_bh, j * BN + q * 64, kb * kBK, z, bar);
            tma_load_3d(st + 3 * kABytes + q * 8192u, &map_bl, j * BN + q * 64, kb * kBK, z, bar);
          }
        } else {
          tma_load_3d(st + 2 * kABytes, &map_bh, kb * kBK, j * BN, z, bar);
          tma_load_3d(st + 3 * kABytes, &map_bl, kb * kBK, j * BN, z, bar);
        }
      }
      drain_loads(full, kSplitStages, kb % kSplitStages, static_cast<uint32_t>(kb / kSplitStages), p.timeout_cycles);
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t idesc = (1u << 4) | (B_MN ? (1u << 16) : 0u) | (static_cast<uint32_t>(BN >> 3) << 17) |
                           (static_cast<uint32_t>(kBM >> 4) << 24);
    const uint64_t desc_k = (64ull << 32) | (1ull << 46) | (2ull << 61) | (1ull << 16);
    const uint64_t desc_mn = (64ull << 32) | (1ull << 46) | (2ull << 61) | (512ull << 16);
    const uint64_t desc_b = B_MN ? desc_mn : desc_k;
    const uint32_t step_b = B_MN ? 128u : 2u, op16 = kABytes >> 4;
    for (int kb = 0; kb < n_kb; ++kb) {
      const uint32_t fold = static_cast<uint32_t>(kb / kFold), buf = fold & 1u, use = fold >> 1;
      if (kb % kFold == 0 && use > 0) mbar_wait(accempty + 8u * buf, (use - 1) & 1u, abort_flag, p.timeout_cycles);
      const int s = kb % kSplitStages;
      mbar_wait(full + 8u * s, static_cast<uint32_t>(kb / kSplitStages) & 1u, abort_flag, p.timeout_cycles);
      tcn_after();
      const uint32_t base = ((ring + static_cast<uint32_t>(s) * kSplitStage) & 0x3ffffu) >> 4;
      const uint32_t d_main = tmem + buf * BN, d_cross = tmem + 2 * BN;
      if (elect_one_n()) {
#pragma unroll
        for (int k = 0; k < kBK / 16; ++k) {
          const uint64_t a_h = desc_k | static_cast<uint64_t>(base + 2u * k);
          const uint64_t a_l = desc_k | static_cast<uint64_t>(base + op16 + 2u * k);
          const uint64_t b_h = desc_b | static_cast<uint64_t>(base + 2u * op16 + step_b * k);
          const uint64_t b_l = desc_b | static_cast<uint64_t>(base + 3u * op16 + step_b * k);
          umma_f16(d_main, a_h, b_h, idesc, (kb % kFold == 0 && k == 0) ? 0u : 1u);
          umma_f16(d_cross, a_l, b_h, idesc, (kb | k) ? 1u : 0u);
          umma_f16(d_cross, a_h, b_l, idesc, 1u);
        }
        umma_commit_n(empty + 8u * s);
        if (kb % kFold == kFold - 1 || kb == n_kb - 1) umma_commit_n(accfull + 8u * buf);
      }
      __syncwarp();
    }
    if (elect_one_n()) umma_commit_n(done);
    __syncwarp();
    volatile unsigned ignore = 0u;
    mbar_wait(done, 0u, &ignore, p.timeout_cycles);
  } else if (warp >= kFirstEpi) {
    constexpr int kCols = BN / 2;
    const int q = warp & 3, part = (warp - kFirstEpi) >> 2;
    const int r = i * kBM + q * 32 + lane;
    const uint32_t t_row = tmem + static_cast<uint32_t>(part * kCols) + (static_cast<uint32_t>(q * 32) << 16);
    float acc[2][32];
#pragma unroll
    for (int e = 0; e < 32; ++e) acc[0][e] = acc[1][e] = 0.f;
    for (int f = 0; f < n_fold; ++f) {
      const uint32_t buf = static_cast<uint32_t>(f) & 1u, use = static_cast<uint32_t>(f) >> 1;
      mbar_wait(accfull + 8u * buf, use & 1u, abort_flag, p.timeout_cycles);
      tcn_after();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[32];
        tmem_ld32(t_row + buf * BN + 32u * h, v);
#pragma unroll
        for (int e = 0; e < 32; ++e) acc[h][e] += v[e];
      }
      tcn_before();
      mbar_arrive(accempty + 8u * buf);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[32];
      tmem_ld32(t_row + 2 * BN + 32u * h, v);
#pragma unroll
      for (int e = 0; e < 32; ++e) acc[h][e] += v[e];
      const int c = j * BN + part * kCols + 32 * h;
      if (c < p.n) finish32<true>(p, z, r, c, acc[h], j < i);
    }
  }
  tcn_before();
  __syncthreads();
  if (warp == 1) {
    tcn_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (tid == 0 && *abort_flag) atomicOr(p.flag, 1u);
}

// ---- host ------------------------------------------------------------------------------------------
// [Z][rows][cols] fp16 matrix with boxes of [box_rows][box_cols]; what lies outside reads as zero and is not written.
int encode_half_map(abs_ctx* ctx, const __half* base, int Z, int rows, int cols, long long ld, int box_rows,
                    CUtensorMap* map, int box_cols = 64, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  const cuuint64_t gdim[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(Z)};
  const cuuint64_t gstr[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * 2 * rows};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 1u};
  const cuuint32_t estr[3] = {1u, 1u, 1u};
  const CUresult r = encode_tiled_fn()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), gdim, gstr, box,
                                       estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS)
    return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled (matrix) failed with code %d", static_cast<int>(r));
  return ABS_OK;
}

void count_tiles(NsGemmParams& p, int bn) {
  p.row_tiles = (p.m + kBM - 1) / kBM;
  p.col_tiles = (p.n + bn - 1) / bn;
  if (p.mode == kUpdate) {
    p.tiles_per_matrix = p.row_tiles * p.col_tiles;
  } else {
    p.tiles_per_matrix = 0;
    for (int i = 0; i < p.row_tiles; ++i) p.tiles_per_matrix += i * kBM / bn + 1;
  }
  p.tiles = static_cast<long long>(p.tiles_per_matrix) * p.Z;
}

constexpr size_t ns_smem(int stages, uint32_t stage_bytes) { return static_cast<size_t>(stages) * stage_bytes + 1024 + 256; }

template <int BN, int MODE>
int launch_plain(abs_ctx* ctx, NsGemmParams p, const __half* a, int a_rows, int a_cols, long long a_ld, const __half* b,
                 int b_rows, int b_cols, long long b_ld, cudaStream_t st) {
  p.mode = MODE;
  NsMaps maps;
  const __half* in_h = MODE == kGram ? p.out_h : p.in_h;        // unused maps are given a valid matrix
  const __half* in_l = MODE == kUpdate ? p.in_l : in_h;
  const __half* out_l = MODE == kUpdate ? p.out_l : p.out_h;
  const CUtensorMapSwizzle s64 = CU_TENSOR_MAP_SWIZZLE_64B;
  int rc = encode_half_map(ctx, a, p.Z, a_rows, a_cols, a_ld, kBM, &maps.a);
  if (rc == ABS_OK) rc = encode_half_map(ctx, b, p.Z, b_rows, b_cols, b_ld, MODE == kUpdate ? 64 : BN, &maps.b);
  if (rc == ABS_OK) rc = encode_half_map(ctx, in_h, p.Z, p.m, p.n, p.ld, kBM, &maps.in_h, kPieceCols, s64);
  if (rc == ABS_OK) rc = encode_half_map(ctx, in_l, p.Z, p.m, p.n, p.ld, kBM, &maps.in_l, kPieceCols, s64);
  if (rc == ABS_OK) rc = encode_half_map(ctx, p.out_h, p.Z, p.m, p.n, p.ld, kBM, &maps.out_h, kPieceCols, s64);
  if (rc == ABS_OK) rc = encode_half_map(ctx, out_l, p.Z, p.m, p.n, p.ld, kBM, &maps.out_l, kPieceCols, s64);
  if (rc == ABS_OK)
    rc = encode_half_map(ctx, p.out_h, p.Z, p.m, p.n, p.ld, kPieceCols, &maps.mirror, kBM, CU_TENSOR_MAP_SWIZZLE_NONE);
  if (rc != ABS_OK) return rc;
  count_tiles(p, BN);
  const size_t smem = ns_smem(BN == 256 ? 3 : 5, kABytes + BN * 128) + kPieces * kPieceBytes;
  auto kern = ns_gemm_kernel<BN, MODE>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  const unsigned grid = static_cast<unsigned>(p.tiles < ctx->sm_count ? p.tiles : ctx->sm_count);
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(grid), dim3(kThreadsN), smem, st, maps, p));
  return ABS_OK;
}

template <bool B_MN>
int launch_split(abs_ctx* ctx, NsGemmParams p, const __half* ah, const __half* al, int a_rows, int a_cols, long long a_ld,
                 const __half* bh, const __half* bl, int b_rows, int b_cols, long long b_ld, cudaStream_t st) {
  CUtensorMap mah, mal, mbh, mbl;
  int rc = encode_half_map(ctx, ah, p.Z, a_rows, a_cols, a_ld, kBM, &mah);
  if (rc == ABS_OK) rc = encode_half_map(ctx, al, p.Z, a_rows, a_cols, a_ld, kBM, &mal);
  if (rc == ABS_OK) rc = encode_half_map(ctx, bh, p.Z, b_rows, b_cols, b_ld, B_MN ? 64 : 128, &mbh);
  if (rc == ABS_OK) rc = encode_half_map(ctx, bl, p.Z, b_rows, b_cols, b_ld, B_MN ? 64 : 128, &mbl);
  if (rc != ABS_OK) return rc;
  count_tiles(p, 128);
  const size_t smem = ns_smem(kSplitStages, kSplitStage);
  auto kern = ns_gemm_split_kernel<B_MN>;
  ABS_CUDA_TRY(ctx, ensure_dynamic_smem(ctx, kern, smem));
  ABS_CUDA_TRY(ctx, launch_dependent(kern, dim3(static_cast<unsigned>(p.tiles)), dim3(kThreadsN), smem, st, mah, mal, mbh,
                                     mbl, p));
  return ABS_OK;
}

}  // namespace

int launch_ns_step(abs_ctx* ctx, const NsBuffers& w, int cur, float a, float b, float c, float sx, float ta, float tb,
                   float sx_next, bool split, cudaStream_t st) {
  if (encode_tiled_fn() == nullptr) return set_error(ctx, ABS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  const __half *xh = w.xh[cur], *xl = w.xl[cur];
  NsGemmParams p = {};
  p.Z = w.Z;
  p.flag = ctx->flags + kNsFlagWord;
  p.drop_loads = ctx->tuning.stats_fault_drop_loads ? 1 : 0;
  p.timeout_cycles = ctx->tuning.stats_timeout_cycles ? ctx->tuning.stats_timeout_cycles : kDefaultTimeoutCycles;
  p.m = p.n = w.m;
  p.ld = w.ldm;
  p.zs = w.ldm * w.m;
  // A = X X'
  p.mode = kGram;
  p.K = w.n;
  p.c_acc = ta / (sx * sx);
  p.out_h = w.ah; p.out_l = w.al;
  int rc = split ? launch_split<false>(ctx, p, xh, xl, w.m, w.n, w.ldx, xh, xl, w.m, w.n, w.ldx, st)
                 : launch_plain<128, kGram>(ctx, p, xh, w.m, w.n, w.ldx, xh, w.m, w.n, w.ldx, st);
  if (rc != ABS_OK) return rc;
  // B = b A + c A A
  p.mode = kPoly;
  p.K = w.m;
  p.in_h = w.ah; p.in_l = w.al;
  p.out_h = w.bh; p.out_l = w.bl;
  p.c_in = b * (tb / ta);
  p.c_acc = c * (tb / (ta * ta));
  rc = split ? launch_split<false>(ctx, p, w.ah, w.al, w.m, w.m, w.ldm, w.ah, w.al, w.m, w.m, w.ldm, st)
             : launch_plain<128, kPoly>(ctx, p, w.ah, w.m, w.m, w.ldm, w.ah, w.m, w.m, w.ldm, st);
  if (rc != ABS_OK) return rc;
  // X <- a X + B X
  p.mode = kUpdate;
  p.n = w.n;
  p.ld = w.ldx;
  p.zs = w.ldx * w.m;
  p.in_h = xh; p.in_l = xl;
  p.out_h = w.xh[cur ^ 1]; p.out_l = w.xl[cur ^ 1];
  p.c_in = a * (sx_next / sx);
  p.c_acc = sx_next / (tb * sx);
  if (split) return launch_split<true>(ctx, p, w.bh, w.bl, w.m, w.m, w.ldm, xh, xl, w.m, w.n, w.ldx, st);
  return launch_plain<256, kUpdate>(ctx, p, w.bh, w.m, w.m, w.ldm, xh, w.m, w.n, w.ldx, st);
}

}  // namespace absk
