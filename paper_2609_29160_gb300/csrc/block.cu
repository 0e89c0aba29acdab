// The rows between two blocks of a layer: residual, gate, norms; and the choice of
// experts.
#include <algorithm>

#include "internal.h"
#include "kvcache.cuh"

namespace tre {
namespace {

// ---------------------------------------------------------------------------
// Norms around a block.
//
// One pass: a row's elements of y and of the residual stay in registers between the two
// sums (mean of squares of y, where there is a post norm, and of r), so that each input is
// read once and each output written once; 8, 16 or 32 elements a thread: a warp has rows of up to 1,024,
// a block of up to 512 threads the others. Bound by HBM where there are rows enough: 20,011 rows of 5,120, bfloat16 beside a 32-bit
// stream, both norms and a gate: 193 us for 1.18 GB, 6.1 TB/s.
// ---------------------------------------------------------------------------
struct BlockArgs {
  const uint8_t *residual, *y, *post_weight, *gate, *weight;
  uint8_t *residual_out, *out;
  int64_t residual_row, y_row, gate_row, gate_col, residual_out_row, out_row;
  int32_t n_rows, dim, per_row;        // per_row: threads of a row
  float scale, eps;
  bool weight_f32, y_f32, out_f32;
};

template <class T> __device__ __forceinline__ void get8(const T* p, float* x) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    Vec<T>::get(*reinterpret_cast<const uint4*>(p), x);
  }
}
template <class T> __device__ __forceinline__ void put8(T* p, const float* x) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = Vec<T>::put(x);
  }
}

// A thread's elements of a row: V times eight, next to each other with WIDE, else a row's
// threads apart: `per_row`, or STEP of them where that is known, so that 32 elements' addresses are one
// and constants. (Kept in registers they went past 128 and to memory: 20,000 rows of 1,001 bfloat16
// 109 us, 51 so; 4,000 of 16,383 444, 230 so.)
template <int V, bool WIDE, int STEP> struct Mine {
  int t, per_row, dim;
  __device__ __forceinline__ int at(int v, int e) const {
    const int step = STEP ? STEP : per_row;
    return WIDE ? (v * step + t) * 8 + e : (v * 8 + e) * step + t;
  }
  template <class T> __device__ __forceinline__ void get(const T* p, float* x) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (WIDE) {
        if (at(v, 0) < dim) get8(p + at(v, 0), x + 8 * v);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) x[8 * v + e] = 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[8 * v + e] = at(v, e) < dim ? (float)p[at(v, e)] : 0.f;
      }
    }
  }
  template <class T> __device__ __forceinline__ void put(T* p, const float* x) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (WIDE) {
        if (at(v, 0) < dim) put8(p + at(v, 0), x + 8 * v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at(v, e) < dim) p[at(v, e)] = T(x[8 * v + e]);
      }
    }
  }
};

// Sum over a row's threads (a warp, or the whole block). `part`: a warp's place each.
__device__ __forceinline__ float row_sum(float x, bool block, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (!block) return x;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  x = lane < warps ? part[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

template <class T, int N, class M>
__device__ __forceinline__ void times_weight(const BlockArgs& a, const uint8_t* w, const M& mine,
                                             float by, float* x) {
  float f[N];
  if (std::is_same<T, float>::value || a.weight_f32) mine.get(reinterpret_cast<const float*>(w), f);
  else mine.get(reinterpret_cast<const T*>(w), f);
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = x[e] * by * f[e];
}

template <class T, class S, int V, bool WIDE, int STEP>
__global__ void __launch_bounds__(512) k_block_norm(const __grid_constant__ BlockArgs a) {
  constexpr int N = 8 * V;
  __shared__ float part[2][32];
  const bool block = a.per_row > 32;
  const int64_t row = block ? blockIdx.x : (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (row >= a.n_rows) return;                       // (whole warps, of rows of their own)
  const Mine<V, WIDE, STEP> mine{block ? (int)threadIdx.x : (int)(threadIdx.x & 31), a.per_row, a.dim};
  float r[N];
  mine.get(reinterpret_cast<const S*>(a.residual) + row * a.residual_row, r);
  if (a.y) {
    float y[N];
    if (std::is_same<T, float>::value || a.y_f32) mine.get(reinterpret_cast<const float*>(a.y) + row * a.y_row, y);
    else mine.get(reinterpret_cast<const T*>(a.y) + row * a.y_row, y);
    if (a.post_weight) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) sum = fmaf(y[e], y[e], sum);
      sum = row_sum(sum, block, part[0]);
      times_weight<T, N>(a, a.post_weight, mine, rsqrtf(sum / a.dim + a.eps), y);
    }
    if (a.gate) {
      const T* g = reinterpret_cast<const T*>(a.gate) + row * a.gate_row;
      if (a.gate_col) {
        float f[N];
        mine.get(g, f);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= f[e];
      } else {
        const float f = (float)*g;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= f;
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = fmaf(a.scale, y[e], r[e]);
  }
  if (a.residual_out) mine.put(reinterpret_cast<S*>(a.residual_out) + row * a.residual_out_row, r);
  if (!a.out) return;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) sum = fmaf(r[e], r[e], sum);
  sum = row_sum(sum, block, part[1]);
  times_weight<T, N>(a, a.weight, mine, rsqrtf(sum / a.dim + a.eps), r);
  if (std::is_same<T, float>::value || a.out_f32) mine.put(reinterpret_cast<float*>(a.out) + row * a.out_row, r);
  else mine.put(reinterpret_cast<T*>(a.out) + row * a.out_row, r);
}

constexpr int kMaxDim = 16384;

template <class T, class S, bool WIDE>
cudaError_t launch_norm(BlockArgs a, cudaStream_t s) {
  const int eights = (a.dim + 7) / 8;
  const int v = eights <= 32 ? 1 : eights <= 64 ? 2 : eights <= 128 ? 4 : eights <= 512 ? 1 : eights <= 1024 ? 2 : 4;
  a.per_row = ((eights + v - 1) / v + 31) / 32 * 32;
  if (!WIDE && v == 4 && a.per_row > 32) a.per_row = 512;
  const bool block = a.per_row > 32;
  const int threads = block ? a.per_row : 128;
  const int64_t blocks = block ? a.n_rows : ((int64_t)a.n_rows + 3) / 4;
  const unsigned grid = (unsigned)blocks;
  if (v == 1) k_block_norm<T, S, 1, WIDE, 0><<<grid, threads, 0, s>>>(a);
  else if (v == 2) k_block_norm<T, S, 2, WIDE, 0><<<grid, threads, 0, s>>>(a);
  else if (block) k_block_norm<T, S, 4, WIDE, WIDE ? 0 : 512><<<grid, threads, 0, s>>>(a);
  else k_block_norm<T, S, 4, WIDE, WIDE ? 0 : 32><<<grid, threads, 0, s>>>(a);
  return cudaGetLastError();
}

template <class T, class S>
cudaError_t launch_norm(const BlockArgs& a, bool wide, cudaStream_t s) {
  return wide ? launch_norm<T, S, true>(a, s) : launch_norm<T, S, false>(a, s);
}

int float_size(int d) { return d == TRE_F32 ? 4 : d == TRE_BF16 || d == TRE_F16 ? 2 : 0; }
bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// ---------------------------------------------------------------------------
// Routing.
//
// A warp a token, a lane every 32nd expert. Choices have to be those of the formulas, not of
// their rounding, because one other expert is another answer. Where c grows with the logit
// (no bias) the logits themselves are compared: scores that 64 bits round to the same number
// are not equal. Else, and for sums of groups, c is computed in 32 bits. Where
// two that follow each other in the choice are closer than 32 bits can tell (one row in some
// hundred of 256 sigmoid scores), the candidates get theirs in 64 bits, a lane each, and are put in
// that order; where a kept group is that close to one that is not (one row in 100,000), or there
// are too many candidates, the whole row's groups or choice are done in 64 bits, whose pipe is some
// sixty times slower.
//
// Candidates: the top-th largest of the lanes' own maxima is not above the top-th largest of all,
// so that what is not below it (some ten to fifteen of 256 for the best eight) has the chosen in
// it. They go to a lane each, which counts how many come before. Taking the best out one after
// the other took 100 instructions each, 1.45 us for 16,384 rows. Where they are more than the lanes
// (one row in some hundred at the best 16, one in five at 20, nearly all from 24 on) a higher bound is
// looked for by halves. Bound by instructions, some 900 for a row of 256 sigmoid scores with a bias in
// groups: 16,384 rows 19 us, 11 without bias and groups, 32 for the best 32 with a bias.
// ---------------------------------------------------------------------------
struct RouteArgs {
  const uint8_t* logits;
  const float* bias;
  int32_t* ids;
  float* weights;
  int64_t row;
  int32_t dtype, n_rows, experts, top, groups, per, top_groups, group_best;
  FastDiv31 by_per;
  float scale;
  bool softmax, renorm, raw;          // raw: choices by the logits
};

constexpr int kRouteWarps = 8, kWideRouteWarps = 4;      // with more than 512 experts (their room)

// NaN is not there, +inf the largest float.
__device__ __forceinline__ float sane(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e38f); }
template <class T> __device__ __forceinline__ const T* logits_of(const RouteArgs& a, int64_t row) {
  return reinterpret_cast<const T*>(a.logits) + row * a.row;
}
__device__ __forceinline__ float logit(const RouteArgs& a, int64_t row, int e) {
  if (a.dtype == TRE_F32) return sane(logits_of<float>(a, row)[e]);
  if (a.dtype == TRE_BF16) return sane((float)logits_of<__nv_bfloat16>(a, row)[e]);
  return sane((float)logits_of<__half>(a, row)[e]);
}
// A lane's logits of a row, as they are (all loads before any is looked at).
template <int NV> __device__ __forceinline__ void row_logits(const RouteArgs& a, int64_t row, float* l) {
  const int lane = threadIdx.x & 31;
  auto all = [&](const auto* p) {
#pragma unroll
    for (int j = 0; j < NV; ++j) l[j] = j * 32 + lane < a.experts ? (float)p[j * 32 + lane] : -INFINITY;
  };
  if (a.dtype == TRE_F32) all(logits_of<float>(a, row));
  else if (a.dtype == TRE_BF16) all(logits_of<__nv_bfloat16>(a, row));
  else all(logits_of<__half>(a, row));
}

// Largest of the lanes (none is NaN)
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Larger floats have larger keys; -inf is the least of those used.
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Largest value of the lanes, and the least index that has it.
__device__ __forceinline__ float warp_best(float x, int& at) {
  const uint32_t key = order(x + 0.f);                // (-0 counts as 0)
  const uint32_t top = __reduce_max_sync(0xffffffffu, key);
  at = (int)__reduce_min_sync(0xffffffffu, key == top ? (uint32_t)at : 0x7fffffffu);
  return value_of(top);
}
// The same of doubles by their keys: comparisons of doubles would go through their slow pipe.
__device__ __forceinline__ uint64_t order(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t key) {
  return __longlong_as_double((long long)(key >> 63 ? key & ~(1ull << 63) : ~key));
}
__device__ __forceinline__ uint64_t warp_best(uint64_t key, int& at) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32));
  const bool in = (uint32_t)(key >> 32) == hi;
  const uint32_t lo = __reduce_max_sync(0xffffffffu, in ? (uint32_t)key : 0u);
  at = (int)__reduce_min_sync(0xffffffffu, in && (uint32_t)key == lo ? (uint32_t)at : 0x7fffffffu);
  return (uint64_t)hi << 32 | lo;
}
template <class F> __device__ __forceinline__ F warp_sum(F x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

// 1 / (1 + exp(-x)), e^x
__device__ __forceinline__ float sigmoid_of(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
__device__ __forceinline__ double sigmoid_of(double x) { return 1.0 / (1.0 + exp(-x)); }

// How far a c in 32 bits may be off, both sides of a comparison. The quick exponential is off by
// (2 + 1.2 |x|) units of 2^-23 of itself, which reach a sigmoid by s (1 - s): less than 1e-7 in
// all; its sum and quotient add 3 units of 2^-24 of s, the bias half a unit of c. A softmax's sum
// of up to 1,024 terms adds a unit for each of its 10 levels. A group's sum of two is off by twice
// that and, as each c and the sum are rounded, by a unit of 2^-23 of what both c are in size.
constexpr float kOffSigmoid = 7e-7f, kOffSoftmax = 3e-6f, kOffBias = 2.5e-7f;

// c of expert j * 32 + lane
template <class F>
__device__ __forceinline__ F score(const RouteArgs& a, float l, float most, F total, int e) {
  const F none = -(F)INFINITY;
  if (!(l > -INFINITY)) return none;
  if (a.raw) return (F)l + (F)0;                     // (-0 counts as 0)
  F c = a.softmax ? exp_of((F)l - (F)most) / total : sigmoid_of((F)l);
  if (a.bias) c += (F)a.bias[e];
  return c > none ? c : none;
}

// Those of a lane's experts (the cases outside the loop: a branch an expert costs more than c).
template <class F, int NV>
__device__ __forceinline__ void all_scores(const RouteArgs& a, const float* l, float most, F total, F* c) {
  const int lane = threadIdx.x & 31;
  const F none = -(F)INFINITY;
  if (a.raw) {
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = (F)l[j] + (F)0;
    return;
  }
  if (a.softmax) {
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = exp_of((F)l[j] - (F)most) / total;
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = sigmoid_of((F)l[j]);
  }
  if (a.bias) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * 32 + lane < a.experts) c[j] += (F)a.bias[j * 32 + lane];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) c[j] = l[j] > -INFINITY && c[j] > none ? c[j] : none;
}

// The two largest of a lane's
template <class F> __device__ __forceinline__ void keep_two(F x, F& first, F& second) {
  if (x > first) {
    second = first;
    first = x;
  } else if (x > second) {
    second = x;
  }
}

// Lane g's return: what group g counts as. size: of what that is the sum of (its error is theirs,
// which may be far larger than the sum).
template <int NV>
__device__ __forceinline__ float group_scores(const RouteArgs& a, const float* c, float* room, float& size) {
  const int lane = threadIdx.x & 31;
  const float none = -INFINITY;
  float first = none, second = none, best = none, next = none;   // best, next: of this lane's group
  auto take = [&](int g, float x, float y) {
    if (lane == g) {
      best = x;
      next = y;
    }
  };
  if (a.per == 32) {                                 // a group a register
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const float x = warp_max(c[j]);
      float y = none;
      if (a.group_best == 2) {
        const int who = __ffs(__ballot_sync(0xffffffffu, c[j] == x)) - 1;
        y = warp_max(lane == who ? none : c[j]);
      }
      take(j, x, y);                                 // (registers past the last group have -inf)
    }
  } else if (a.per % 32 == 0) {                      // groups of whole registers
    const int regs = a.per / 32;
    int left = regs, g = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      keep_two(c[j], first, second);
      if (--left == 0) {
        const float x = warp_max(first);
        float y = none;
        if (a.group_best == 2) {
          const int who = __ffs(__ballot_sync(0xffffffffu, first == x)) - 1;
          y = warp_max(lane == who ? second : first);
        }
        take(g, x, y);
        ++g;
        left = regs;
        first = second = none;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * 32 + lane < a.experts) room[j * 32 + lane] = c[j];
    __syncwarp();
    if (lane < a.groups) {
      int i = lane % a.per;                          // (lanes start apart: their banks)
      for (int n = 0; n < a.per; ++n) {
        keep_two(room[lane * a.per + i], best, next);
        if (++i == a.per) i = 0;
      }
      if (a.group_best == 1) next = none;
    }
    __syncwarp();
  }
  size = best > none ? fabsf(best) : 0.f;
  if (next > none) {
    best += next;
    size += fabsf(next);
  }
  return best;
}
// The same in 64 bits, of keys.
__device__ __forceinline__ uint64_t group_scores(const RouteArgs& a, const uint64_t* room) {
  const int lane = threadIdx.x & 31;
  const uint64_t none = order(-(double)INFINITY);
  if (lane >= a.groups) return none;
  uint64_t first = none, second = none;
  int i = lane % a.per;
  for (int n = 0; n < a.per; ++n) {
    keep_two(room[lane * a.per + i], first, second);
    if (++i == a.per) i = 0;
  }
  if (a.group_best == 1 || second == none) return first;
  return order(value_of(first) + value_of(second));
}

// The groups that stay, by lanes' scores of them, and how far the last of them is from the next.
__device__ __forceinline__ unsigned kept_groups(const RouteArgs& a, float mine, float& last, float& next) {
  unsigned kept = 0;
  for (int k = 0; k < a.top_groups; ++k) {
    last = warp_max(mine);
    const int who = __ffs(__ballot_sync(0xffffffffu, mine == last)) - 1;
    kept |= 1u << who;                               // (of what is left, none of them -inf: any)
    if ((threadIdx.x & 31) == who) mine = -INFINITY;
  }
  next = warp_max(mine);
  return kept;
}
__device__ __forceinline__ unsigned kept_groups(const RouteArgs& a, uint64_t mine) {
  const int lane = threadIdx.x & 31;
  int better = 0;
  for (int g = 0; g < a.groups; ++g) {
    const uint64_t x = __shfl_sync(0xffffffffu, mine, g);
    if (x > mine || (x == mine && g < lane)) ++better;
  }
  return __ballot_sync(0xffffffffu, lane < a.groups && better < a.top_groups);
}
template <int NV, class K>
__device__ __forceinline__ void only_kept(const RouteArgs& a, unsigned kept, K none, K* c) {
  const int lane = threadIdx.x & 31;
  if (a.per == 32) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (!(kept >> j & 1)) c[j] = none;
  } else if (a.per % 32 == 0) {
    const int regs = a.per / 32;
    int left = regs;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (!(kept & 1)) c[j] = none;
      if (--left == 0) {
        kept >>= 1;
        left = regs;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * 32 + lane < a.experts && !(kept >> a.by_per.div(j * 32 + lane) & 1)) c[j] = none;
  }
}

// The largest c and its expert, which is taken out.
template <int NV, class K> __device__ __forceinline__ K take_best(K* c, K none, int& at) {
  const int lane = threadIdx.x & 31;
  K best = none;
  at = 0x7fffffff;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (c[j] > best) {
      best = c[j];
      at = j * 32 + lane;
    }
  best = warp_best(best, at);
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j * 32 + lane == at) c[j] = none;
  return best;
}

template <class F, int NV>
__device__ __forceinline__ F softmax_total(const float* l, float most) {
  F sum = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) sum += l[j] > -INFINITY ? exp_of((F)l[j] - (F)most) : (F)0;
  return warp_sum(sum);
}

// A lane's c of the whole row in 64 bits, by their keys.
template <int NV>
__device__ __forceinline__ void double_scores(const RouteArgs& a, int64_t row, float most, uint64_t* c) {
  const int lane = threadIdx.x & 31;
  const uint64_t none = order(-(double)INFINITY);
  float l[NV];
  row_logits<NV>(a, row, l);
#pragma unroll
  for (int j = 0; j < NV; ++j) l[j] = sane(l[j]);
  const double total = a.softmax ? softmax_total<double, NV>(l, most) : 1.0;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    c[j] = j * 32 + lane < a.experts ? order(score(a, l[j], most, total, j * 32 + lane)) : none;
}
// The groups that stay, by them.
template <int NV>
__device__ __noinline__ unsigned kept_double(const RouteArgs& a, int64_t row, float most, uint64_t* room) {
  const int lane = threadIdx.x & 31;
  uint64_t c[NV];
  double_scores<NV>(a, row, most, c);
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j * 32 + lane < a.experts) room[j * 32 + lane] = c[j];
  __syncwarp();
  const unsigned kept = kept_groups(a, group_scores(a, room));
  __syncwarp();
  return kept;
}
// Lane i's return is the i-th expert of the groups that stay (-1: none).
template <int NV>
__device__ __noinline__ int choose_double(const RouteArgs& a, int64_t row, float most, unsigned kept) {
  const int lane = threadIdx.x & 31;
  const uint64_t none = order(-(double)INFINITY);
  uint64_t c[NV];
  double_scores<NV>(a, row, most, c);
  if (a.groups > 1) only_kept<NV>(a, kept, none, c);
  int mine = -1;
  for (int k = 0; k < a.top; ++k) {
    int at;
    if (take_best<NV>(c, none, at) == none) break;
    if (lane == k) mine = at;
  }
  return mine;
}

// What a lane has of the choice: an expert and its place in the order (past `top`: not chosen).
struct Choice {
  int expert, place;
};

// The same in 32 bits where they can tell. near: the warp's room for candidates.
struct Near {
  float c[32];
  int expert[32];
};
template <int NV>
__device__ __forceinline__ Choice choose(const RouteArgs& a, int64_t row, const float* l, float most, uint64_t* room,
                                         Near& near) {
  const int lane = threadIdx.x & 31;
  float c[NV];
  const float total = a.softmax && !a.raw ? softmax_total<float, NV>(l, most) : 1.f;
  all_scores<float, NV>(a, l, most, total, c);
  float off = a.raw ? 0.f : a.softmax ? kOffSoftmax : kOffSigmoid, rel = a.raw ? 0.f : kOffBias;
  unsigned kept = 0;
  if (a.groups > 1) {
    float last = 0.f, next = 0.f, size;
    const float value = group_scores<NV>(a, c, reinterpret_cast<float*>(room), size);
    kept = kept_groups(a, value, last, next);
    // (of the largest group: others than these two may be further off than they are apart)
    const bool unsure = next > -INFINITY && !(last - next > 2.f * off + rel * warp_max(size));
    if (off > 0.f && unsure) kept = kept_double<NV>(a, row, most, room);
    if (!a.bias && !a.raw) {                         // in the groups that stay it is the logits
#pragma unroll
      for (int j = 0; j < NV; ++j) c[j] = l[j] + 0.f;
      off = rel = 0.f;
    }
    only_kept<NV>(a, kept, (float)-INFINITY, c);
  }
  // the top-th largest of the lanes' maxima, and what 32 bits cannot tell from it
  constexpr float kLeast = -3.402823466e38f;
  float own = c[0];
#pragma unroll
  for (int j = 1; j < NV; ++j) own = fmaxf(own, c[j]);
  float bound = -INFINITY, best = own;
  for (int k = 0; k < a.top; ++k) {
    bound = warp_max(own);
    if (own == bound) own = -INFINITY;               // (all that are equal: the bound is then lower)
  }
  bound = fmaxf(bound, kLeast);
  auto below = [&](float x) {
    const float least = x - (off + rel * fabsf(x));
    return least > kLeast ? least : kLeast;          // (also what infinities make of it)
  };
  // Those not below it (not -inf), a place each of the first 32; how many
  auto list = [&](float least) {
    int count = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const bool in = c[j] >= least;
      const unsigned all = __ballot_sync(0xffffffffu, in);
      const int at = count + __popc(all & ((1u << lane) - 1));
      if (in && at < 32) {
        near.c[at] = c[j];
        near.expert[at] = j * 32 + lane;
      }
      count += __popc(all);
    }
    __syncwarp();
    return count;
  };
  int count = list(below(bound));
  Choice mine{-1, 32};
  if (count > 32) {
    // more than lanes (`top` near their number, or many equal ones): a higher bound that has `top` of
    // them not below it, by halves between this one and the largest
    auto many = [&](float least) {
      int n = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) n += c[j] >= least;
      return (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
    };
    best = warp_max(best);
    uint32_t low = order(bound), high = order(best) + 1;
    while (high - low > 1) {
      const uint32_t mid = low + (high - low) / 2;
      const float x = value_of(mid);
      if (many(x) < a.top) {
        high = mid;
        continue;
      }
      low = mid;
      if (many(below(x)) <= 32) break;
    }
    count = list(below(value_of(low)));
  }
  if (count > 32) {                                  // many equal ones, or closer than 32 bits tell
    if (off > 0.f) return Choice{choose_double<NV>(a, row, most, kept), lane};
    for (int k = 0; k < a.top; ++k) {
      int at;
      if (!(take_best<NV>(c, (float)-INFINITY, at) > -INFINITY)) break;
      if (lane == k) mine = Choice{at, k};
    }
    return mine;
  }
  // (candidates stand in the order of experts, which decides between equal ones)
  const float x = lane < count ? near.c[lane] : -INFINITY;
  if (lane < count) mine.expert = near.expert[lane];
  __syncwarp();
  int before = 0;
  float under = -INFINITY;                           // the largest that comes after
  for (int k = 0; k < count; ++k) {
    const float y = __shfl_sync(0xffffffffu, x, k);
    if (y > x || (y == x && k < lane)) ++before;
    else if (k != lane) under = fmaxf(under, y);
  }
  if (lane < count) mine.place = before;
  const bool unsure = off > 0.f && lane < count && before < a.top && under > -INFINITY &&
                      !(x - under > off + rel * fabsf(x));
  if (!__any_sync(0xffffffffu, unsure)) return mine;
  const double sum = a.softmax ? softmax_total<double, NV>(l, most) : 1.0;
  double z = -(double)INFINITY;
  if (mine.expert >= 0) z = score(a, logit(a, row, mine.expert), most, sum, mine.expert);
  before = 0;
  for (int k = 0; k < count; ++k) {
    const double y = __shfl_sync(0xffffffffu, z, k);
    if (y > z || (y == z && k < lane)) ++before;
  }
  if (lane < count) mine.place = before;
  return mine;
}

template <int NV> constexpr int route_warps = NV > 16 ? kWideRouteWarps : kRouteWarps;
template <int NV>
__global__ void __launch_bounds__(route_warps<NV> * 32) k_route(const __grid_constant__ RouteArgs a) {
  extern __shared__ uint64_t room_all[];               // [warps][experts], with groups
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ Near near[kRouteWarps];
  uint64_t* room = room_all + warp * a.experts;
  const int64_t row = (int64_t)blockIdx.x * route_warps<NV> + warp;
  if (row >= a.n_rows) return;
  float l[NV], most = -INFINITY;
  row_logits<NV>(a, row, l);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    l[j] = sane(l[j]);
    most = fmaxf(most, l[j]);
  }
  most = warp_max(most);
  const Choice mine = choose<NV>(a, row, l, most, room, near[warp]);
  const bool chosen = mine.expert >= 0 && mine.place < a.top;
  const float x = chosen ? logit(a, row, mine.expert) : -INFINITY;
  // Weights; with their sum divided out a sigmoid's are kept from running out of exponent
  // by the largest of them.
  float w = 0.f;
  if (a.renorm) {
    const float top = warp_max(x);
    if (chosen) {
      if (a.softmax) w = expf(x - top);
      else w = x >= 0.f ? 1.f / (1.f + expf(-x)) : expf(x - fminf(top, 0.f)) / (1.f + expf(x));
    }
    const float sum = warp_sum(w);
    if (chosen) w = w / sum * a.scale;
  } else if (a.softmax) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) sum += l[j] > -INFINITY ? expf(l[j] - most) : 0.f;
    sum = warp_sum(sum);
    if (chosen) w = expf(x - most) / sum * a.scale;
  } else if (chosen) {
    w = 1.f / (1.f + expf(-x)) * a.scale;
  }
  if (chosen) {
    a.ids[row * a.top + mine.place] = mine.expert;
    a.weights[row * a.top + mine.place] = w;
  }
  const int found = __popc(__ballot_sync(0xffffffffu, chosen));
  if (lane >= found && lane < a.top) {
    a.ids[row * a.top + lane] = -1;
    a.weights[row * a.top + lane] = 0.f;
  }
}

template <int NV> cudaError_t launch_route(const RouteArgs& a, cudaStream_t s) {
  constexpr int warps = route_warps<NV>;
  const int64_t blocks = ((int64_t)a.n_rows + warps - 1) / warps;
  const size_t room = a.groups > 1 ? sizeof(uint64_t) * warps * a.experts : 0;
  k_route<NV><<<(unsigned)blocks, warps * 32, room, s>>>(a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace tre

using namespace tre;

extern "C" {

tre_status tre_block_norm(const tre_block_rows* b, tre_stream stream) {
  if (!b || b->n_rows < 0 || b->dim < 1 || b->dim > kMaxDim) return TRE_EINVAL;
  const int el = float_size(b->dtype), st = float_size(b->stream_dtype);
  const int yt = float_size(b->y_dtype), ot = float_size(b->out_dtype), wt = float_size(b->weight_dtype);
  if (!el) return TRE_EINVAL;
  for (tre_dtype d : {b->stream_dtype, b->y_dtype, b->out_dtype, b->weight_dtype})
    if (d != TRE_F32 && d != b->dtype) return TRE_EINVAL;
  if (!(b->eps >= 0.f) || b->eps > 3e38f || !(b->scale >= -3e38f && b->scale <= 3e38f))
    return TRE_EINVAL;
  if (b->gate_col != 0 && b->gate_col != 1) return TRE_EINVAL;
  if (!b->y && (b->post_weight || b->gate)) return TRE_EINVAL;
  if ((b->out && !b->weight) || (!b->out && !b->residual_out)) return TRE_EINVAL;
  if (!on(b->residual, st) || !on(b->residual_out, st) || !on(b->y, yt) || !on(b->gate, el) ||
      !on(b->out, ot) || !on(b->post_weight, wt) || !on(b->weight, wt))
    return TRE_EINVAL;
  if (b->n_rows == 0) return TRE_OK;
  if (!b->residual) return TRE_EINVAL;
  BlockArgs a;
  a.residual = static_cast<const uint8_t*>(b->residual);
  a.y = static_cast<const uint8_t*>(b->y);
  a.post_weight = static_cast<const uint8_t*>(b->post_weight);
  a.gate = static_cast<const uint8_t*>(b->gate);
  a.weight = static_cast<const uint8_t*>(b->weight);
  a.residual_out = static_cast<uint8_t*>(b->residual_out);
  a.out = static_cast<uint8_t*>(b->out);
  a.residual_row = b->residual_row;
  a.y_row = b->y_row;
  a.gate_row = b->gate_row;
  a.gate_col = b->gate_col;
  a.residual_out_row = b->residual_out_row;
  a.out_row = b->out_row;
  a.n_rows = b->n_rows;
  a.dim = b->dim;
  a.scale = b->scale;
  a.eps = b->eps;
  a.weight_f32 = b->weight_dtype == TRE_F32;
  a.y_f32 = b->y_dtype == TRE_F32;
  a.out_f32 = b->out_dtype == TRE_F32;
  const bool wide =
      b->dim % 8 == 0 && on(b->residual, 16) && on(b->y, 16) && on(b->residual_out, 16) &&
      on(b->out, 16) && on(b->post_weight, 16) && on(b->weight, 16) &&
      b->residual_row * st % 16 == 0 && (!b->y || b->y_row * yt % 16 == 0) &&
      (!b->residual_out || b->residual_out_row * st % 16 == 0) &&
      (!b->out || b->out_row * ot % 16 == 0) &&
      (!b->gate || !b->gate_col || (on(b->gate, 16) && b->gate_row * el % 16 == 0));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (b->dtype == TRE_F32) e = launch_norm<float, float>(a, wide, s);
  else if (b->dtype == TRE_BF16)
    e = b->stream_dtype == TRE_F32 ? launch_norm<__nv_bfloat16, float>(a, wide, s)
                                   : launch_norm<__nv_bfloat16, __nv_bfloat16>(a, wide, s);
  else
    e = b->stream_dtype == TRE_F32 ? launch_norm<__half, float>(a, wide, s)
                                   : launch_norm<__half, __half>(a, wide, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

tre_status tre_route(const tre_router* r, tre_stream stream) {
  if (!r || r->n_rows < 0 || r->experts < 1 || r->experts > 1024) return TRE_EINVAL;
  const int el = float_size(r->dtype);
  if (!el || !on(r->logits, el)) return TRE_EINVAL;
  if (r->top < 1 || r->top > 32 || r->top > r->experts) return TRE_EINVAL;
  if (r->scores != TRE_SOFTMAX && r->scores != TRE_SIGMOID) return TRE_EINVAL;
  if (r->groups < 1 || r->groups > 32 || r->experts % r->groups || r->top_groups < 1 ||
      r->top_groups > r->groups || r->group_best < 1 || r->group_best > 2)
    return TRE_EINVAL;
  if (!(r->scale >= -3e38f && r->scale <= 3e38f)) return TRE_EINVAL;
  if (r->n_rows == 0) return TRE_OK;
  if (!r->logits || !r->ids || !r->weights) return TRE_EINVAL;
  if (!on(r->ids, 4) || !on(r->weights, 4) || !on(r->bias, 4)) return TRE_EINVAL;
  RouteArgs a;
  a.logits = static_cast<const uint8_t*>(r->logits);
  a.bias = r->bias;
  a.ids = r->ids;
  a.weights = r->weights;
  a.row = r->logits_row;
  a.dtype = r->dtype;
  a.n_rows = r->n_rows;
  a.experts = r->experts;
  a.top = r->top;
  a.groups = r->top_groups == r->groups ? 1 : r->groups;      // (all stay)
  a.per = r->experts / r->groups;
  a.top_groups = r->top_groups;
  a.group_best = r->group_best;
  a.by_per = FastDiv31((uint32_t)a.per);
  a.scale = r->scale;
  a.softmax = r->scores == TRE_SOFTMAX;
  a.renorm = r->renorm != 0;
  a.raw = !r->bias && (a.groups == 1 || r->group_best == 1);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int nv = (r->experts + 31) / 32;
  const cudaError_t e = nv <= 1   ? launch_route<1>(a, s)
                        : nv <= 2 ? launch_route<2>(a, s)
                        : nv <= 4 ? launch_route<4>(a, s)
                        : nv <= 8 ? launch_route<8>(a, s)
                        : nv <= 16 ? launch_route<16>(a, s)
                                   : launch_route<32>(a, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

}  // extern "C"
