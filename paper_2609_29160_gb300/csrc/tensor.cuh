// What the kernels on the tensor cores share: barriers in shared memory, tensor memory,
// products (tcgen05) of tiles of 128 rows, tensor copies.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"

namespace tre {

constexpr long long kWaitClocks = 4000000000ll, kDrainClocks = 40000000ll;

__device__ __forceinline__ uint32_t smem_of(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(smem_of(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(smem_of(b)) : "memory");
}
// One arrival for a warp whose lanes are all done.
__device__ __forceinline__ void bar_arrive_warp(uint64_t* b) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) bar_arrive(b);
}
__device__ __forceinline__ bool bar_poll(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2; selp.b32 %0, 1, 0, p; }"
      : "=r"(ok)
      : "r"(smem_of(b)), "r"(parity)
      : "memory");
  return ok;
}
// Waits. False when the barrier did not come in about two seconds, here or in another warp:
// then there is no more work, and every warp meets at the end. (A thread for itself; a warp.)
__device__ __forceinline__ bool bar_wait_one(uint64_t* b, uint32_t parity, volatile int* dead) {
  bool ok = bar_poll(b, parity);
  if (!ok) {
    const long long from = clock64();
    while (!(ok = bar_poll(b, parity))) {
      if (*dead) break;
      if (clock64() - from > kWaitClocks) {
        *dead = 1;
        break;
      }
    }
  }
  return ok;
}
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* dead) {
  return __all_sync(0xffffffffu, bar_wait_one(b, parity, dead));
}

__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(at)
      : "memory");
}
// (names the registers, so that nothing reads them before)
__device__ __forceinline__ void tmem_wait_ld(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                 "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
  asm volatile(""
               : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                 "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                   smem_of(b))
               : "memory");
}
// One lane of a warp, in a way that lets the compiler keep what it computes in the
// warp's shared registers: the operands of a product come from those, and moving
// them there one by one takes longer than the product.
__device__ __forceinline__ bool one_lane() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.b32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}
// D (TMEM) = or += A * B, both operands in shared memory / A in TMEM. Operands of
// shared memory by the low half of their description (see operand).
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       bool add) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 x, y; setp.ne.b32 p, %4, 0; mov.b64 x, {%1, %5}; "
      "mov.b64 y, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "n"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                       bool add) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 y; setp.ne.b32 p, %4, 0; mov.b64 y, {%2, %5};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "n"(kOperandHigh)
      : "memory");
}

// Two floats at a time
__device__ __forceinline__ uint64_t two(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(uint64_t v, uint32_t* x) {
  asm("mov.b64 {%0, %1}, %2;" : "=r"(x[0]), "=r"(x[1]) : "l"(v));
}
__device__ __forceinline__ uint64_t two(const uint32_t* x) {
  return two(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ void fma2(uint32_t* x, float f, float plus) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(two(x)), "l"(two(f, f)), "l"(two(plus, plus)));
  split(r, x);
}
__device__ __forceinline__ void fma2(uint32_t* x, float f, float plus, float plus1) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(two(x)), "l"(two(f, f)), "l"(two(plus, plus1)));
  split(r, x);
}
__device__ __forceinline__ void mul2(uint32_t* x, float f, float g) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(two(x)), "l"(two(f, g)));
  split(r, x);
}
__device__ __forceinline__ uint64_t sum2(uint64_t s, float a, float b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(s), "l"(two(a, b)));
  return r;
}
__device__ __forceinline__ float halves_sum(uint64_t a, uint64_t b) {
  uint32_t x[2], y[2];
  split(a, x);
  split(b, y);
  return (__uint_as_float(x[0]) + __uint_as_float(y[0])) +
         (__uint_as_float(x[1]) + __uint_as_float(y[1]));
}

// Low half of the description of an operand in shared memory, in rows of 128 bytes with
// the 16-byte pieces of row r at piece ^ (r & 7): its address and `lead`, the bytes to
// the next 64 elements along the dense axis (where that axis is not the one summed
// over). The high half (kOperandHigh) says 1024 bytes to the next eight rows and that
// order of pieces.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t lead) {
  return ((at >> 4) & 0x3fff) | (lead >> 4) << 16;
}
template <class T> __host__ __device__ constexpr uint32_t idesc_of(int n, bool b_turned) {
  const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (b_turned ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 |
         (uint32_t)(128 >> 4) << 24;
}

__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(smem_of(b)), "r"(bytes)
               : "memory");
}

// The driver's encoder of tensor maps, looked up once (it is not part of the runtime).
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                            const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline Encode encoder() {
  static const Encode fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<Encode>(p);
  }();
  return fn;
}

}  // namespace tre
