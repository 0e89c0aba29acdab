// Rows of heads on their way into a paged cache and out of it.
//
// k_heads: y = x * w / sqrt(mean x^2 + eps), then the rotation of the row's
// position, then either a rounding to the input's type or a cache code: scale
// amax|y| / Q (Q = 448 for e4m3, 127 for int8), code = round(y / scale). A row of
// 64 or 128 elements is read once and stays in the registers of 8 or 16 lanes, each
// with four elements and the four that they turn with, so only its sum and maximum go
// between lanes; everything is 32-bit until the one rounding at the end, and the
// division is the exact one, so codes do not depend on how a row is reached. A warp
// takes a whole token where there are many: its place in the cache, cosines and sines
// are fetched once for all heads. Bound by HBM when rows are many and wide: 40,013 tokens
// of 32 heads of 64 floats 106 us, 6.2 TB/s; of bfloat16, half the bytes, 63 us, 5.3 TB/s;
// 12 chunks of up to 4,001 tokens, 48 heads of 64, f16 into an f16 cache 51 us, 5.5 TB/s.
// Into codes the instructions bind: the same chunks into int8 68 us, 3.5 TB/s, three of
// four issue slots taken (exact divisions, packing). By the chain q_start ->
// lengths -> page -> store when there are few: one token of 64 requests is a few us on
// the device, less than what its call costs the host.
//
// k_read: codes (and scales) of whole tokens back to rows of a model's type, bound by
// HBM: 16 contexts of up to 50,000 tokens, e4m3 to bf16, 138 us, 6.6 TB/s (159 us with
// 16-byte stores; 32-byte ones where the outputs' boundaries allow). The 12 chunks above
// out of codes 27 us, 5.3 TB/s, out of f16 34 us, 5.6.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "kvcache.cuh"

namespace tre {
namespace {

constexpr int kThreads = 256;

struct HeadsArgs {
  const uint8_t* in[3];           // q, k, v
  int64_t row[3], head[3];        // bytes
  uint8_t* out[2];
  int64_t orow[2], ohead[2];      // bytes
  const void* weight[2];
  const float* cos_sin;
  int64_t cs_row;
  const int32_t* positions;       // without a cache
  int32_t heads[3];
  int32_t n_rows, n_pos, rot;
  float eps;
  bool interleaved, weight_f32;
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

template <int W> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int W> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Four elements of T
template <class T> struct Four {
  using Raw = uint2;
  static __device__ __forceinline__ Raw zero() { return make_uint2(0, 0); }
  static __device__ __forceinline__ void get(const Raw& v, float* x) {
    unpack(v.x, x[0], x[1], T());
    unpack(v.y, x[2], x[3], T());
  }
  static __device__ __forceinline__ Raw put(const float* x) {
    return make_uint2(pack<T>(x[0], x[1]), pack<T>(x[2], x[3]));
  }
};
template <> struct Four<float> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ void get(const Raw& v, float* x) { Vec<float>::get(v, x); }
  static __device__ __forceinline__ Raw put(const float* x) { return Vec<float>::put(x); }
};

// x / d correctly rounded, given y = 1 / d correctly rounded: a product, its exact
// remainder and one correction (P. Markstein, "Computation of elementary functions on
// the IBM RISC System/6000 processor", 1990). For d in [2^-100, 2^100] and |x| <= 512 d;
// a quotient so small that its remainder underflows rounds to a code of zero either way.
__device__ __forceinline__ float quotient(float x, float d, float y) {
  const float q = __fmul_rn(x, y);
  return __fmaf_rn(__fmaf_rn(-q, d, x), y, q);
}

// Four codes of x / by
template <Code CODE> __device__ __forceinline__ uint32_t codes_of(const float* q) {
  if constexpr (CODE == Code::kE4m3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(q[0], q[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(q[2], q[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  } else {
    // |q| <= 127 (see where it is taken): in q + 1.5 * 2^23 the last byte is q rounded to nearest even
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(__fadd_rn(q[j], 12582912.f));
    return __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
  }
}

// A warp takes `its` steps of RPW rows of a token's q, k and v heads; `groups` warps
// share a token.
template <class T, Code CODE, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 3 : 4)
k_heads(HeadsArgs a, BatchArgs b, CacheArgs c, int groups, int its, tre_diag* diag) {
  using F = Four<T>;
  constexpr int LPR = D / 8, RPW = 32 / LPR, U = sizeof(T) == 4 ? 2 : 4, EL = sizeof(T);
  const int lane = threadIdx.x & 31, sub = lane / LPR, u = lane % LPR;
  const uint32_t w =
      __shfl_sync(0xffffffffu, blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), 0);
  const int t = (int)(w / groups), grp = (int)(w - (uint32_t)t * groups);
  if (t >= a.n_rows) return;
  // steps of q, of k, of v: a step's rows are of one kind
  const int first_k = (a.heads[0] + RPW - 1) / RPW;
  const int first_v = first_k + (a.heads[1] + RPW - 1) / RPW;
  const int n_steps = first_v + (a.heads[2] + RPW - 1) / RPW;
  const int end_step = min((grp + 1) * its, n_steps);
  // this lane's elements: ea .. ea + 3 and those they turn with, eb .. eb + 3 (a row's
  // unturned tail is halved in the same way)
  const int half = a.rot >> 1;
  const bool turns = 4 * u < half;
  const int ea = a.interleaved ? 8 * u : turns ? 4 * u : half + 4 * u;
  const int eb = ea + (a.interleaved ? 4 : turns ? half : (D - a.rot) >> 1);

  typename F::Raw raw[U][2];
  // the first rows: they depend on nothing
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int st = grp * its + k, s = st < first_k ? 0 : st < first_v ? 1 : 2;
    const int h = (st - (s == 0 ? 0 : s == 1 ? first_k : first_v)) * RPW + sub;
    raw[k][0] = raw[k][1] = F::zero();
    if (st < end_step && h < a.heads[s]) {
      const uint8_t* p = a.in[s] + t * a.row[s] + h * a.head[s];
      raw[k][0] = *reinterpret_cast<const typename F::Raw*>(p + ea * EL);
      raw[k][1] = *reinterpret_cast<const typename F::Raw*>(p + eb * EL);
    }
  }

  // where the token stands
  int pos, page = 0, slot = 0;
  bool ok = true, counted = true;
  if (CODE == Code::kNone) {
    pos = a.positions ? a.positions[t] : 0;
  } else {
    const int i = find_seq(b, t);
    pos = 0;
    ok = counted = false;
    if (i >= 0) {
      const int end = b.q_start[i + 1];
      if (t < end) {
        counted = true;
        pos = b.ctx_len[i] - (end - t);
        page = page_of(c, b, i, pos, slot);
        ok = page >= 0;
      }
    }
  }
  if (a.cos_sin && (pos < 0 || pos >= a.n_pos)) ok = false;
  if (!ok && counted && diag && grp == 0 && lane == 0)
    atomicAdd((unsigned long long*)&diag->dropped_range, 1ull);

  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.cos_sin && turns && ok) {
    const float* p = a.cos_sin + pos * a.cs_row + 4 * u;
    const float4 y = *reinterpret_cast<const float4*>(p);
    const float4 z = *reinterpret_cast<const float4*>(p + half);
    cs[0] = y.x; cs[1] = y.y; cs[2] = y.z; cs[3] = y.w;
    sn[0] = z.x; sn[1] = z.y; sn[2] = z.z; sn[3] = z.w;
  }
  const int64_t at = page * c.s_page + slot * c.s_token;

  auto part = [&](auto kind) {
    constexpr int s = decltype(kind)::value;
    constexpr bool stored = CODE != Code::kNone && s >= 1;
    const int from = s == 0 ? 0 : s == 1 ? first_k : first_v;
    const int upto = min(end_step, s == 0 ? first_k : s == 1 ? first_v : n_steps);
    int it = max(grp * its, from);
    if (it >= upto) return;
    bool have = it == grp * its;
    const uint8_t* in = a.in[s] + t * a.row[s];
    const int64_t in_head = a.head[s];
    uint8_t* out;
    int64_t out_head;
    if constexpr (stored) {
      out = (s == 1 ? c.k : c.v) + at * (CODE == Code::kHalf ? EL : 1);
      out_head = c.s_head * (CODE == Code::kHalf ? EL : 1);
    } else {
      out = a.out[s & 1] + t * a.orow[s & 1];
      out_head = a.ohead[s & 1];
    }
    float g[8];
    const void* wt = s < 2 ? a.weight[s & 1] : nullptr;
    if (wt) {
      if (a.weight_f32) {
        Four<float>::get(*reinterpret_cast<const uint4*>(static_cast<const float*>(wt) + ea), g);
        Four<float>::get(*reinterpret_cast<const uint4*>(static_cast<const float*>(wt) + eb), g + 4);
      } else {
        F::get(*reinterpret_cast<const typename F::Raw*>(static_cast<const T*>(wt) + ea), g);
        F::get(*reinterpret_cast<const typename F::Raw*>(static_cast<const T*>(wt) + eb), g + 4);
      }
    }
    for (; it < upto; it += U) {
      if (!have) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int h = (it + k - from) * RPW + sub;
          raw[k][0] = raw[k][1] = F::zero();
          if (it + k < upto && h < a.heads[s]) {
            const uint8_t* p = in + h * in_head;
            raw[k][0] = *reinterpret_cast<const typename F::Raw*>(p + ea * EL);
            raw[k][1] = *reinterpret_cast<const typename F::Raw*>(p + eb * EL);
          }
        }
      }
      have = false;
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (it + k >= upto) break;
        const int h = (it + k - from) * RPW + sub;
        const bool there = h < a.heads[s];
        float x[8];
        F::get(raw[k][0], x);
        F::get(raw[k][1], x + 4);
        if (wt) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = __fmaf_rn(x[e], x[e], ss);
          const float r = rsqrtf(__fmaf_rn(group_sum<LPR>(ss), 1.f / D, a.eps));
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * r * g[e];
        }
        if (s < 2 && a.cos_sin && turns) {
          if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = x[2 * e], q = x[2 * e + 1];
              x[2 * e] = __fmaf_rn(p, cs[e], -(q * sn[e]));
              x[2 * e + 1] = __fmaf_rn(q, cs[e], p * sn[e]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = x[e], q = x[e + 4];
              x[e] = __fmaf_rn(p, cs[e], -(q * sn[e]));
              x[e + 4] = __fmaf_rn(q, cs[e], p * sn[e]);
            }
          }
        }
        uint8_t* p = out + h * out_head;
        if constexpr (!stored || CODE == Code::kHalf) {
          if (!stored && !ok) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
          }
          if (there && (!stored || ok)) {
            *reinterpret_cast<typename F::Raw*>(p + ea * EL) = F::put(x);
            *reinterpret_cast<typename F::Raw*>(p + eb * EL) = F::put(x + 4);
          }
        } else {
          float m = fabsf(x[0]);
#pragma unroll
          for (int e = 1; e < 8; ++e) m = max_nan(m, fabsf(x[e]));
          m = group_max<LPR>(m);
          if (ok && there) {
            constexpr float Q = CODE == Code::kE4m3 ? 448.f : 127.f;
            const bool plain = m > 0x1p-90f && m < 0x1p90f;
            // (an infinite maximum leaves a scale that is no number)
            const float sc = plain ? quotient(m, Q, 1.f / Q) : div_rn(m, Q) + 0.f * m;
            const float by = sc == 0.f ? 1.f : sc, r = __frcp_rn(by);
            float q[8];
            if (plain) {
#pragma unroll
              for (int e = 0; e < 8; ++e) q[e] = quotient(x[e], by, r);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                // (a scale that is a subnormal of few bits may be well below max|x| / Q)
                q[e] = div_rn(x[e], by);
                if constexpr (CODE == Code::kI8) q[e] = fminf(fmaxf(q[e], -Q), Q);
              }
            }
            *reinterpret_cast<uint32_t*>(p + ea) = codes_of<CODE>(q);
            *reinterpret_cast<uint32_t*>(p + eb) = codes_of<CODE>(q + 4);
            if (u == 0)
              (s == 1 ? c.k_scale : c.v_scale)[page * c.c_page + slot * c.c_token + h * c.c_head] = sc;
          }
        }
      }
    }
  };
  part(std::integral_constant<int, 0>());
  part(std::integral_constant<int, 1>());
  if constexpr (CODE != Code::kNone) part(std::integral_constant<int, 2>());
}

struct ReadOut {
  uint8_t *k, *v;
  int64_t row, head;             // elements
  bool wide;                     // on 32-byte boundaries
};

// One warp takes one token's keys and values, 16 bytes of the cache a lane, the
// token's place once.
template <class T, class OUT, Code CODE, int D>
__global__ void __launch_bounds__(kThreads)
k_read(BatchArgs b, CacheArgs c, ReadOut o, tre_diag* diag) {
  constexpr int CB = CODE == Code::kHalf ? 2 : 1;       // bytes of an element in the cache
  constexpr int N = 16 / CB, LPR = D / N, RPW = 32 / LPR, OV = Vec<OUT>::N;
  const int lane = threadIdx.x & 31, sub = lane / LPR, e0 = (lane % LPR) * N;
  const int64_t t64 = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t64 >= b.n_rows) return;
  const int t = (int)t64, i = find_seq(b, t);
  int page = -1, slot = 0;
  if (i >= 0) {
    const int end = b.q_start[i + 1];
    if (t < end) {
      page = page_of(c, b, i, b.ctx_len[i] - (end - t), slot);
      if (page < 0 && diag && lane == 0)
        atomicAdd((unsigned long long*)&diag->dropped_range, 1ull);
    }
  }
  const int64_t at = page * c.s_page + slot * c.s_token, sat = page * c.c_page + slot * c.c_token;
  const int rows = 2 * c.heads;
  constexpr int U = 4;
  for (int r0 = sub; r0 < rows; r0 += U * RPW) {
    uint4 raw[U];
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * RPW;
      raw[u] = make_uint4(0, 0, 0, 0);
      sc[u] = 0.f;
      if (r < rows && page >= 0) {
        const bool val = r >= c.heads;
        const int h = val ? r - c.heads : r;
        raw[u] = *reinterpret_cast<const uint4*>((val ? c.v : c.k) + (at + h * c.s_head + e0) * CB);
        if (CB == 1) sc[u] = (val ? c.v_scale : c.k_scale)[sat + h * c.c_head];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * RPW;
      if (r >= rows) continue;
      const bool val = r >= c.heads;
      const int h = val ? r - c.heads : r;
      float x[N];
      if constexpr (CB == 2) {
        Vec<T>::get(raw[u], x);
      } else {
        const uint32_t q[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) codes4<CODE>(q[j], x + 4 * j);
        if (page >= 0) {
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = mul_rn(x[e], sc[u]);
        }
      }
      OUT* dst = reinterpret_cast<OUT*>(val ? o.v : o.k) + t * o.row + h * o.head + e0;
      if (o.wide && N > OV) {
        // 32 bytes a store: whole sectors
#pragma unroll
        for (int e = 0; e + OV < N; e += 2 * OV) {
          const uint4 y = Vec<OUT>::put(x + e), z = Vec<OUT>::put(x + e + OV);
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + e),
                       "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w), "r"(z.x), "r"(z.y), "r"(z.z), "r"(z.w)
                       : "memory");
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; e += OV) *reinterpret_cast<uint4*>(dst + e) = Vec<OUT>::put(x + e);
      }
    }
  }
}

bool mult16(int64_t elements, int size) { return elements * size % 16 == 0; }
bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int type_size(int d) {
  switch (d) {
    case TRE_F32: return 4;
    case TRE_BF16: case TRE_F16: return 2;
    case TRE_E4M3: case TRE_I8: return 1;
  }
  return 0;
}

// Fills `a` from the caller's struct; false for what no kernel takes.
bool heads_args(const tre_heads* h, bool keys_out, HeadsArgs& a) {
  if (!h || (h->dim != 64 && h->dim != 128) || h->n_rows < 0 || h->q_heads < 0 || h->k_heads < 0)
    return false;
  const int el = type_size(h->dtype);
  if (el < 2 || h->q_heads > 65536 || h->k_heads > 65536) return false;
  if (!(h->eps >= 0.f) || h->eps > 3e38f) return false;
  if ((h->q_weight || h->k_weight) &&
      (h->weight_dtype != h->dtype && h->weight_dtype != TRE_F32))
    return false;
  if ((h->q_weight && !at16(h->q_weight)) || (h->k_weight && !at16(h->k_weight))) return false;
  if (h->cos_sin) {
    if (h->rot < 16 || h->rot > h->dim || h->rot % 16 || h->n_pos < 1 || !at16(h->cos_sin) ||
        !mult16(h->cos_sin_row, 4))
      return false;
  }
  const void* in[2] = {h->q, h->k};
  void* out[2] = {h->q_out, h->k_out};
  const int64_t row[2] = {h->q_row, h->k_row}, head[2] = {h->q_head, h->k_head};
  const int64_t orow[2] = {h->q_out_row, h->k_out_row}, ohead[2] = {h->q_out_head, h->k_out_head};
  for (int s = 0; s < 2; ++s) {
    const int n = s ? h->k_heads : h->q_heads;
    a.heads[s] = n;
    a.in[s] = static_cast<const uint8_t*>(in[s]);
    a.out[s] = static_cast<uint8_t*>(out[s]);
    a.row[s] = row[s] * el;
    a.head[s] = head[s] * el;
    a.orow[s] = orow[s] * el;
    a.ohead[s] = ohead[s] * el;
    if (n == 0 || h->n_rows == 0) continue;
    if (!in[s] || !at16(in[s]) || !mult16(row[s], el) || !mult16(head[s], el)) return false;
    if (s == 1 && !keys_out) continue;
    if (!out[s] || !at16(out[s]) || !mult16(orow[s], el) || !mult16(ohead[s], el)) return false;
  }
  a.heads[2] = 0;
  a.in[2] = nullptr;
  a.row[2] = a.head[2] = 0;
  a.weight[0] = h->q_weight;
  a.weight[1] = h->k_weight;
  a.weight_f32 = h->weight_dtype == TRE_F32;
  a.cos_sin = h->cos_sin;
  a.cs_row = h->cos_sin_row;
  a.positions = nullptr;
  a.n_rows = h->n_rows;
  a.n_pos = h->n_pos;
  a.rot = h->cos_sin ? h->rot : 0;
  a.eps = h->eps;
  a.interleaved = h->interleaved != 0;
  return true;
}

// A warp takes a whole token's heads when that leaves every SM 32 warps (its place and
// its rotation are then fetched once for all of them), else as few as still does. One step
// a warp took 184 us for 40,013 tokens of 32 heads (106 so) and 178 for appending the
// f16 -> int8 chunks above and reading them back (93); whole tokens always are the same
// there and 39.0 against 36.4 us for both calls of one token of 64 requests.
template <class T, Code CODE, int D>
cudaError_t launch_heads(const HeadsArgs& a, const BatchArgs& b, const CacheArgs& c,
                         tre_diag* diag, cudaStream_t s) {
  constexpr int RPW = 32 / (D / 8);
  if (a.heads[0] + a.heads[1] + a.heads[2] == 0 || a.n_rows == 0) return cudaSuccess;
  int64_t steps = 0;
  for (int x = 0; x < 3; ++x) steps += (a.heads[x] + RPW - 1) / RPW;
  const int64_t warps = (int64_t)device_sm_count() * 32;
  const int64_t its = std::min(steps, std::max<int64_t>(1, a.n_rows * steps / warps));
  const int64_t groups = (steps + its - 1) / its;
  constexpr int64_t per = kThreads / 32;
  const int64_t blocks = ((int64_t)a.n_rows * groups + per - 1) / per;
  if (blocks > 2147483647) return cudaErrorInvalidValue;
  k_heads<T, CODE, D><<<(unsigned)blocks, kThreads, 0, s>>>(a, b, c, (int)groups, (int)its, diag);
  return cudaGetLastError();
}

template <class T, Code CODE>
cudaError_t heads_by_dim(int dim, const HeadsArgs& a, const BatchArgs& b, const CacheArgs& c,
                         tre_diag* diag, cudaStream_t s) {
  return dim == 64 ? launch_heads<T, CODE, 64>(a, b, c, diag, s)
                   : launch_heads<T, CODE, 128>(a, b, c, diag, s);
}

template <class T>
cudaError_t append_by_code(int code, int dim, const HeadsArgs& a, const BatchArgs& b,
                           const CacheArgs& c, tre_diag* diag, cudaStream_t s) {
  if (code == TRE_E4M3) return heads_by_dim<T, Code::kE4m3>(dim, a, b, c, diag, s);
  if (code == TRE_I8) return heads_by_dim<T, Code::kI8>(dim, a, b, c, diag, s);
  return heads_by_dim<T, Code::kHalf>(dim, a, b, c, diag, s);
}

template <class T, class OUT, Code CODE>
cudaError_t launch_read(int dim, const BatchArgs& b, const CacheArgs& c, const ReadOut& o,
                        tre_diag* diag, cudaStream_t s) {
  constexpr int64_t per = kThreads / 32;
  const unsigned blocks = (unsigned)(((int64_t)b.n_rows + per - 1) / per);
  if (dim == 64) k_read<T, OUT, CODE, 64><<<blocks, kThreads, 0, s>>>(b, c, o, diag);
  else k_read<T, OUT, CODE, 128><<<blocks, kThreads, 0, s>>>(b, c, o, diag);
  return cudaGetLastError();
}

template <class OUT>
cudaError_t read_by_code(int code, int dim, const BatchArgs& b, const CacheArgs& c,
                         const ReadOut& o, tre_diag* diag, cudaStream_t s) {
  switch (code) {
    case TRE_BF16: return launch_read<__nv_bfloat16, OUT, Code::kHalf>(dim, b, c, o, diag, s);
    case TRE_F16: return launch_read<__half, OUT, Code::kHalf>(dim, b, c, o, diag, s);
    case TRE_E4M3: return launch_read<__half, OUT, Code::kE4m3>(dim, b, c, o, diag, s);
    default: return launch_read<__half, OUT, Code::kI8>(dim, b, c, o, diag, s);
  }
}

}  // namespace

bool cache_args(const tre_kv_cache* c, CacheArgs& a) {
  if (!c || (c->dim != 64 && c->dim != 128) || c->page < 1 || c->heads < 1 || c->heads > 65535 ||
      c->n_pages < 0)
    return false;
  const bool coded = c->dtype == TRE_E4M3 || c->dtype == TRE_I8;
  if (!coded && c->dtype != TRE_BF16 && c->dtype != TRE_F16) return false;
  const int el = type_size(c->dtype);
  if (c->n_pages > 0) {
    if (!c->k || !c->v || !at16(c->k) || !at16(c->v)) return false;
    if (coded && (!c->k_scale || !c->v_scale)) return false;
  }
  if (!mult16(c->page_stride, el) || !mult16(c->token_stride, el) || !mult16(c->head_stride, el))
    return false;
  a.k = static_cast<uint8_t*>(c->k);
  a.v = static_cast<uint8_t*>(c->v);
  a.k_scale = coded ? c->k_scale : nullptr;
  a.v_scale = coded ? c->v_scale : nullptr;
  a.s_page = c->page_stride;
  a.s_token = c->token_stride;
  a.s_head = c->head_stride;
  a.c_page = c->scale_page_stride;
  a.c_token = c->scale_token_stride;
  a.c_head = c->scale_head_stride;
  a.n_pages = c->n_pages;
  a.page = c->page;
  a.heads = c->heads;
  a.by_page = FastDiv31((uint32_t)c->page);
  return true;
}

bool batch_args(const tre_kv_batch* b, BatchArgs& a) {
  if (!b || b->n_seq < 0 || b->n_rows < 0 || b->max_pages < 0 || b->max_new < 0 || b->max_ctx < 0)
    return false;
  if (b->n_seq > 0 && (!b->ctx_len || !b->q_start)) return false;
  if (b->n_seq > 0 && b->max_pages > 0 && !b->pages) return false;
  a.pages = b->pages;
  a.ctx_len = b->ctx_len;
  a.q_start = b->q_start;
  a.pages_row = b->pages_row;
  a.n_seq = b->n_seq;
  a.n_rows = b->n_rows;
  a.max_pages = b->max_pages;
  return true;
}

}  // namespace tre

using namespace tre;

extern "C" {

tre_status tre_qk_norm_rope(const tre_heads* heads, const int32_t* positions, tre_diag* diag,
                            tre_stream stream) {
  HeadsArgs a;
  if (!heads_args(heads, true, a) || (heads->cos_sin && heads->n_rows > 0 && !positions))
    return TRE_EINVAL;
  a.positions = positions;
  BatchArgs b{};
  CacheArgs c{};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (heads->dtype == TRE_F32) e = heads_by_dim<float, Code::kNone>(heads->dim, a, b, c, diag, s);
  else if (heads->dtype == TRE_BF16)
    e = heads_by_dim<__nv_bfloat16, Code::kNone>(heads->dim, a, b, c, diag, s);
  else e = heads_by_dim<__half, Code::kNone>(heads->dim, a, b, c, diag, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

tre_status tre_kv_append(const tre_kv_cache* cache, const tre_kv_batch* batch,
                         const tre_heads* heads, const void* v, int64_t v_row, int64_t v_head,
                         tre_diag* diag, tre_stream stream) {
  HeadsArgs a;
  BatchArgs b;
  CacheArgs c;
  if (!heads_args(heads, false, a) || !batch_args(batch, b) || !cache_args(cache, c))
    return TRE_EINVAL;
  if (heads->dtype != TRE_BF16 && heads->dtype != TRE_F16) return TRE_EINVAL;
  if (cache->dtype != heads->dtype && cache->dtype != TRE_E4M3 && cache->dtype != TRE_I8)
    return TRE_EINVAL;
  if (heads->k_heads != cache->heads || heads->dim != cache->dim || heads->n_rows != batch->n_rows)
    return TRE_EINVAL;
  if (heads->n_rows == 0) return TRE_OK;
  if (!v || !at16(v) || !mult16(v_row, 2) || !mult16(v_head, 2)) return TRE_EINVAL;
  if (batch->n_seq == 0) return TRE_EINVAL;
  a.heads[2] = cache->heads;
  a.in[2] = static_cast<const uint8_t*>(v);
  a.row[2] = v_row * 2;
  a.head[2] = v_head * 2;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      heads->dtype == TRE_BF16
          ? append_by_code<__nv_bfloat16>(cache->dtype, heads->dim, a, b, c, diag, s)
          : append_by_code<__half>(cache->dtype, heads->dim, a, b, c, diag, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

tre_status tre_kv_read(const tre_kv_cache* cache, const tre_kv_batch* batch, tre_dtype out_dtype,
                       void* k_out, void* v_out, int64_t out_row, int64_t out_head,
                       tre_diag* diag, tre_stream stream) {
  BatchArgs b;
  CacheArgs c;
  if (!batch_args(batch, b) || !cache_args(cache, c)) return TRE_EINVAL;
  const int el = type_size(out_dtype);
  if (el < 2) return TRE_EINVAL;
  if (batch->n_rows == 0) return TRE_OK;
  if (batch->n_seq == 0) return TRE_EINVAL;
  if (!k_out || !v_out || !at16(k_out) || !at16(v_out) || !mult16(out_row, el) ||
      !mult16(out_head, el))
    return TRE_EINVAL;
  const bool wide = !((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 31) &&
                    out_row * el % 32 == 0 && out_head * el % 32 == 0;
  ReadOut o{static_cast<uint8_t*>(k_out), static_cast<uint8_t*>(v_out), out_row, out_head, wide};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (out_dtype == TRE_F32) e = read_by_code<float>(cache->dtype, cache->dim, b, c, o, diag, s);
  else if (out_dtype == TRE_BF16)
    e = read_by_code<__nv_bfloat16>(cache->dtype, cache->dim, b, c, o, diag, s);
  else e = read_by_code<__half>(cache->dtype, cache->dim, b, c, o, diag, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

}  // extern "C"
