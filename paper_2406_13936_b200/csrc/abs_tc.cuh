// tcgen05, tensor-memory and packed-arithmetic wrappers of the attention kernels.
#pragma once

#include "abs_pipeline.cuh"

namespace absk {

#ifdef __CUDACC__
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool elect_lane() {
  uint32_t is_leader;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(is_leader));
  return is_leader != 0;
}
// d (tensor memory, fp32) (+)= A B, bf16: both operands in shared memory, or A in tensor memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives on the barrier when the products issued so far are complete.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_alloc_all(uint32_t slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_all(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// 32 columns of this thread's lane; the values may be used after tmem_loaded on the same registers.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_loaded(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
        "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
        "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
        "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      :
      : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
        "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Pairs of fp32.
__device__ __forceinline__ uint64_t pack2f(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2f(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t fma2f(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2f(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2f(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {          // within 2 ulp; results below 2^-126 are zero
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
  const float2 v = unpack2f(x);
  return pack2f(exp2_approx(v.x), exp2_approx(v.y));
}
// 2^x of a pair on the FMA pipe, for some of the exponentials where the other unit (16 a clock and SM) is what bounds: x = n + f with n
// the nearest whole number (Cody and Waite's reduction, exact for base 2), 2^f by a polynomial of degree 5 whose relative error is the
// least possible on [-1/2, 1/2] (7.5e-8, found by Remez's exchange; 2.1e-7 with its roundings), and 2^n from its bits: adding 1.5 2^23 + 127
// leaves n + 127 in the lowest bits, which are shifted into the exponent.  Below -126.5 zero; NaN stays NaN.
__device__ __forceinline__ uint64_t exp2_pair_fma(uint64_t x) {
  constexpr float kShift = 12582912.f + 127.f;
  float2 v = unpack2f(x);
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(v.x) : "f"(-127.f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(v.y) : "f"(-127.f));
  x = pack2f(v.x, v.y);
  const uint64_t t = add2f(x, pack2f(kShift, kShift));
  const uint64_t n = add2f(t, pack2f(-kShift, -kShift)), f = fma2f(n, pack2f(-1.f, -1.f), x);
  uint64_t p = fma2f(pack2f(1.3276472454890609e-3f, 1.3276472454890609e-3f), f, pack2f(9.675540961325169e-3f, 9.675540961325169e-3f));
  p = fma2f(p, f, pack2f(5.550713092088699e-2f, 5.550713092088699e-2f));
  p = fma2f(p, f, pack2f(0.24022120237350464f, 0.24022120237350464f));
  p = fma2f(p, f, pack2f(0.6931469440460205f, 0.6931469440460205f));
  p = fma2f(p, f, pack2f(1.0000001192092896f, 1.0000001192092896f));
  const float2 b = unpack2f(t);
  return mul2f(p, pack2f(__uint_as_float(__float_as_uint(b.x) << 23), __uint_as_float(__float_as_uint(b.y) << 23)));
}
__device__ __forceinline__ float max3f(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// A wait of a whole warp, the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile unsigned* abort_flag, long long limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit));
}

// The same for copies that were issued: no other role's abort ends it, since they write to shared memory that must still be this CTA's.  One
// that does run out raises the abort flag.
__device__ __forceinline__ bool warp_arrival(uint32_t bar, uint32_t parity, volatile unsigned* abort_flag, long long limit) {
  bool here = mbar_try_wait(bar, parity);
  for (const long long t0 = clock64(); !here && clock64() - t0 <= limit;) here = mbar_try_wait(bar, parity);
  here = __all_sync(0xffffffffu, here);
  if (!here) *abort_flag = 1u;
  return here;
}

// Operand descriptors without the address (in units of 16 bytes): 128-byte swizzled rows, version 1 (bit 46), swizzle mode 2 (bits
// 61-63).  K-major: a row is 64 values of k, groups of 8 rows 1024 bytes apart; 16 values of k are 32 bytes.  MN-major: a row is
// 64 columns at one value of k, groups of 8 values of k 1024 bytes apart (stride offset), further blocks of 64 columns `block`
// bytes apart (leading offset); 16 values of k are 2048 bytes.
constexpr uint64_t kDescK = (64ull << 32) | (1ull << 46) | (2ull << 61) | (1ull << 16);
__host__ __device__ constexpr uint64_t desc_mn(uint32_t block) { return (64ull << 32) | (1ull << 46) | (2ull << 61) | (static_cast<uint64_t>(block >> 4) << 16); }
__device__ __forceinline__ uint32_t desc_at(uint32_t smem) { return (smem & 0x3ffffu) >> 4; }
// fp32 accumulator, bf16 operands, MN-major ones, M x N
__host__ __device__ constexpr uint32_t mma_idesc(int m, int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
         (static_cast<uint32_t>(m >> 4) << 24);
}
#endif

// 32 columns of a thread's row times `by` as bf16 (NaN if not valid), of which the first `columns` exist, a multiple of 8; of a row's
// length and place multiples of 16 (sectors) whole sectors of 32 bytes: a warp's rows lie far apart, and the backward pass of 16 x 1024 tokens,
// 12 heads of 128, took 340 us with 16 bytes at a time and takes 323.
__device__ __forceinline__ void store_row32(__nv_bfloat16* out, const uint32_t* x, float by, bool valid, int columns, bool sectors) {
#pragma unroll
  for (int c = 0; c < 32; c += 16) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      w[i] = valid ? bf16_pair(__uint_as_float(x[c + 2 * i]) * by, __uint_as_float(x[c + 2 * i + 1]) * by) : 0x7fc07fc0u;
    if (sectors) {
      if (c < columns)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + c), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                     "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
      if (c < columns) *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
      if (c + 8 < columns) *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}

}  // namespace absk
