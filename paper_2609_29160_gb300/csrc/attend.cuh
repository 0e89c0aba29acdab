// What the attention kernels share: the call's arguments, the range of positions
// that a tile of rows sees, and the output of rows whose masked values are no number.
#pragma once

#include "kvcache.cuh"

namespace tre {

constexpr float kLn2 = 0.693147180559945309f;

struct AttendArgs {
  const uint8_t* q;
  uint8_t* out;
  float* lse;                     // [n_rows][heads], may be null
  int32_t q_row, q_head, o_row, o_head;   // elements
  int32_t heads, group;           // query heads, query heads of one cache head
  FastDiv31 by_group;
  float scale2;                   // scale * log2(e): scores are kept in powers of two
  int32_t window;                 // 0: none
  int32_t parts, split;           // parts of a context, and the shortest part
  int32_t row_tiles;              // k_attend: blocks along a sequence's rows
  int32_t few;                    // rows of a sequence that k_attend takes
  // Sums, maxima and weights of parts, for the join: [parts][part_rows * heads][dim], [..][2].
  // tokens > 0: row r of sequence i stands at part row i * tokens + r (only sequences
  // of few rows have any), else at its own.
  float *part_o, *part_ml;
  int64_t part_rows;
  int32_t tokens;
  float2* done;                   // the other kernel's part_ml: rows that are not its
  // k_attend_tc: `parts` is the most there is room for; how many it takes is seen on the
  // device, where the rows of each sequence are known, and left here for the join
  int32_t* parts_taken;
  uint32_t* next;                 // k_attend_tc: units taken past the first of each block, or null
  int32_t sms;
  bool wide;                      // outputs on 32-byte boundaries
  bool beside;                    // k_attend: launched beside k_attend_tc
};

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// New rows of sequence i and the positions it holds.
struct Seq {
  int start, n, ctx;
};
__device__ __forceinline__ Seq seq_of(const BatchArgs& b, int i) {
  Seq s;
  const int a = min(max(b.q_start[i], 0), b.n_rows);
  s.start = a;
  s.n = min(max(b.q_start[i + 1], a), b.n_rows) - a;
  s.ctx = b.ctx_len[i];
  return s;
}

// Positions [lo, hi) that rows of tokens t0..t1 of a sequence may see; lo is a
// multiple of STEP.
template <int STEP>
__device__ __forceinline__ void range_of(const Seq& s, const CacheArgs& c, const BatchArgs& b,
                                         int window, int t0, int t1, int& lo, int& hi) {
  const int base = s.ctx - s.n;
  const int64_t cap = (int64_t)b.max_pages * c.page;
  const int64_t h = min64((int64_t)base + t1 + 1, cap);
  hi = (int)(h > 0 ? h : 0);
  int64_t l = window > 0 ? (int64_t)base + t0 - window + 1 : 0;
  lo = (int)(l > 0 ? l : 0) / STEP * STEP;
}

// Part sp of a range: contexts longer than the host expected get longer parts.
// STEP: tokens that a kernel takes at a time.
template <int STEP>
__device__ __forceinline__ void part_of(const AttendArgs& a, int sp, int& lo, int& hi) {
  const int len = hi - lo;
  if (len <= 0) return;
  int chunk = max(a.split, (len + a.parts - 1) / a.parts);
  chunk = (chunk + STEP - 1) / STEP * STEP;
  const int64_t from = (int64_t)lo + (int64_t)sp * chunk;
  const int to = (int)min64(hi, from + chunk);
  lo = (int)min64(from, hi);
  hi = to;
}

// k_attend_tc's time, in positions, with contexts of up to `len` in n parts each: whole
// rounds of one unit an SM, a round takes its part and about 900 more (a unit's start and
// end); a split costs what a row's partial sums cost to write and read, about 400 a part,
// spread over all SMs, and some 1,500 for the join.
__host__ __device__ __forceinline__ float parts_time(int64_t n, int64_t units, int64_t len,
                                                     int64_t sms) {
  return (float)((units * n + sms - 1) / sms) * ((float)len / n + 900.f) +
         (n > 1 ? 400.f * n * units / sms + 1500.f : 0.f);
}

// Whether a row saw no position (scores that are no number leave m alone, not l).
__device__ __forceinline__ bool saw_nothing(float m, float l) { return m == -INFINITY && l == l; }

// What a block leaves beside a row's sum: for its part of the join, or (one part)
// the row's logarithm, and for the other kernel's join that the row is not its (a weight
// below zero).
__device__ __forceinline__ void row_state(const AttendArgs& a, int sp, int64_t row,
                                          int64_t part_row, int head, float m, float l) {
  if (a.parts > 1)
    reinterpret_cast<float2*>(a.part_ml)[(sp * a.part_rows + part_row) * a.heads + head] =
        make_float2(m, l);
  else if (a.lse)
    a.lse[row * a.heads + head] = saw_nothing(m, l) ? -INFINITY : (m + log2f(l)) * kLn2;
  if (a.done && sp == 0) a.done[row * a.heads + head] = make_float2(0.f, -1.f);
}

// The power of two of a value's scale, which counts in its weight: with m the
// largest s + exponent, a weight exp2(s - m) * scale stays below two whatever the
// scales are. (Bounded, so that a scale of zero leaves m finite.)
__device__ __forceinline__ float weight_exponent(float scale) {
  return fminf(fmaxf(__log2f(fabsf(scale)), -100.f), 100.f);
}

// DIM/32 elements of one cached row, as floats (without the scale).
template <class T, Code CODE, int DIM>
__device__ __forceinline__ void cached(const uint8_t* base, int64_t off, int lane, float* x) {
  constexpr int N = DIM / 32;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int64_t at = off + lane * N + e;
    if constexpr (CODE == Code::kHalf) {
      float hi;
      unpack(reinterpret_cast<const uint16_t*>(base)[at], x[e], hi, T());
    } else {
      float y[4];
      codes4<CODE>(base[at], y);
      x[e] = y[0];
    }
  }
}

// One row's sum of exp2(s_j - m) v_j over the positions of [lo, hi) that it sees,
// by one warp, DIM/32 elements a lane. The tiled kernels multiply masked values by
// zero, which leaves NaN where a masked value is infinite or no number: a row that
// comes out that way is done again here, where masked values are not touched.
template <class T, Code CODE, int DIM>
__device__ void row_again(const AttendArgs& a, const BatchArgs& b, const CacheArgs& c, int i,
                          int kvh, const T* q, int pos, int lo, int hi, float m, float* acc) {
  constexpr int N = DIM / 32;
  const int lane = threadIdx.x & 31;
  float x[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    x[e] = (float)q[lane * N + e];
    acc[e] = 0.f;
  }
  if (a.window > 0) lo = max(lo, pos - a.window + 1);
  hi = min(hi, pos + 1);
  for (int j = lo; j < hi; ++j) {
    int slot = 0;
    const int page = page_of(c, b, i, j, slot);
    if (page < 0) continue;
    const int64_t off = page * c.s_page + slot * c.s_token + kvh * c.s_head;
    const int64_t soff = page * c.c_page + slot * c.c_token + kvh * c.c_head;
    float y[N], s = 0.f;
    cached<T, CODE, DIM>(c.k, off, lane, y);
#pragma unroll
    for (int e = 0; e < N; ++e) s = __fmaf_rn(x[e], y[e], s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= a.scale2;
    if (CODE != Code::kHalf) s *= c.k_scale[soff];
    float p = exp2_fast(s - m);
    if (CODE != Code::kHalf) p = mul_rn(p, c.v_scale[soff]);
    cached<T, CODE, DIM>(c.v, off, lane, y);
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = __fmaf_rn(p, y[e], acc[e]);
  }
}

// Rows of no sequence (before the first, after the last): zeros, no weight. One
// block of every launch does them; usually there are none.
template <class T, int DIM>
__device__ void loose_rows(const AttendArgs& a, const BatchArgs& b) {
  const int first = min(max(b.q_start[0], 0), b.n_rows);
  const int last = min(max(b.q_start[b.n_seq], first), b.n_rows);
  const int loose = first + b.n_rows - last;
  for (int64_t r = threadIdx.x; r < (int64_t)loose * a.heads; r += blockDim.x) {
    const int k = (int)(r / a.heads), h = (int)(r - (int64_t)k * a.heads);
    const int64_t t = k < first ? k : last + (k - first);
    T* o = reinterpret_cast<T*>(a.out) + t * a.o_row + (int64_t)h * a.o_head;
    for (int e = 0; e < DIM; ++e) o[e] = T(0.f);
    if (a.lse) a.lse[t * a.heads + h] = -INFINITY;
    if (a.done) a.done[t * a.heads + h] = make_float2(0.f, -1.f);
    if (a.parts > 1 && a.tokens == 0)
      reinterpret_cast<float2*>(a.part_ml)[t * a.heads + h] = make_float2(0.f, -1.f);
  }
}

}  // namespace tre
