// What the replica's kernels share: element types, the paged cache's addressing
// and the search for a row's sequence.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace tre {

enum class Code { kNone, kHalf, kE4m3, kI8 };   // what a cache holds: nothing, 16 bits, 8 bits

__device__ __forceinline__ void unpack(uint32_t v, float& lo, float& hi, __nv_bfloat16) {
  lo = __uint_as_float(v << 16);
  hi = __uint_as_float(v & 0xffff0000u);
}
__device__ __forceinline__ void unpack(uint32_t v, float& lo, float& hi, __half) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
  lo = f.x;
  hi = f.y;
}
template <class T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 16 bytes of T as floats, and back
template <class T> struct Vec {
  static constexpr int N = 16 / sizeof(T);
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    unpack(v.x, x[0], x[1], T());
    unpack(v.y, x[2], x[3], T());
    unpack(v.z, x[4], x[5], T());
    unpack(v.w, x[6], x[7], T());
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(pack<T>(x[0], x[1]), pack<T>(x[2], x[3]), pack<T>(x[4], x[5]),
                      pack<T>(x[6], x[7]));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
  }
};

// Two 8-bit codes (the low 16 bits of w) as a pair of halves, which hold both kinds exactly.
template <Code CODE> __device__ __forceinline__ uint32_t halves(uint32_t w) {
  if constexpr (CODE == Code::kE4m3) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    // 0x6400 + u is the half 1024 + u; u = code + 128
    const uint32_t u = __byte_perm(w ^ 0x8080u, 0x6464u, 0x4140);
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

// four 8-bit codes as floats
template <Code CODE> __device__ __forceinline__ void codes4(uint32_t v, float* x) {
  unpack(halves<CODE>(v), x[0], x[1], __half());
  unpack(halves<CODE>(v >> 16), x[2], x[3], __half());
}

// A paged cache as the kernels see it (strides in elements).
struct CacheArgs {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int64_t s_page, s_token, s_head;      // of codes
  int64_t c_page, c_token, c_head;      // of scales
  int32_t n_pages, page, heads;
  FastDiv31 by_page;
};
struct BatchArgs {
  const int32_t *pages, *ctx_len, *q_start;
  int64_t pages_row;
  int32_t n_seq, n_rows, max_pages;
};

// Page of a position of sequence i, -1 where the table holds none.
__device__ __forceinline__ int page_of(const CacheArgs& c, const BatchArgs& b, int i, int pos,
                                       int& slot) {
  if (pos < 0) return -1;
  const int q = (int)c.by_page.div((uint32_t)pos);
  slot = pos - q * c.page;
  if (q >= b.max_pages) return -1;
  const int id = b.pages[(int64_t)i * b.pages_row + q];
  return id >= 0 && id < c.n_pages ? id : -1;
}

// The sequence that row t belongs to (-1: none): the last one that starts at or
// before t. The whole warp searches, 32 probes a step.
__device__ __forceinline__ int find_seq(const BatchArgs& b, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = b.n_seq + 1;
  while (true) {
    const int step = (len + 31) >> 5;
    const int at = lane * step;
    const bool below = at < len && b.q_start[lo + at] <= t;
    const int c = __popc(__ballot_sync(0xffffffffu, below));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    len = min(step, len - (c - 1) * step);
    if (step == 1) break;
  }
  return lo < b.n_seq ? lo : -1;
}

// host side, kvcache.cu: checks and the kernels' form of the C structs
bool cache_args(const tre_kv_cache* c, CacheArgs& a);
bool batch_args(const tre_kv_batch* b, BatchArgs& a);

}  // namespace tre
