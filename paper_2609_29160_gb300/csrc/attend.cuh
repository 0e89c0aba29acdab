// What the attention kernels share: the call's arguments, the range of positions
// that a tile of rows sees, and what masked values that are no numbers are kept from.
#pragma once

#include <type_traits>

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

// Words of a tile with elements that are no finite numbers as zeros. Products multiply
// masked values by weights of zero, which such a value would turn into NaN: in tiles that
// some row sees and another does not they are left out, and rows that see them get them
// back from add_seen.
template <class T, Code CODE> __device__ __forceinline__ uint32_t finite(uint32_t x) {
  if constexpr (CODE == Code::kHalf) {
    constexpr uint32_t top = std::is_same<T, __nv_bfloat16>::value ? 0x7f807f80u : 0x7c007c00u;
    return x & ~__vcmpeq2(x & top, top);
  } else if constexpr (CODE == Code::kE4m3) {
    return x & ~__vcmpeq4(x & 0x7f7f7f7fu, 0x7f7f7f7fu);
  }
  return x;
}
template <class T, Code CODE> __device__ __forceinline__ uint4 finite(const uint4& v) {
  return make_uint4(finite<T, CODE>(v.x), finite<T, CODE>(v.y), finite<T, CODE>(v.z),
                    finite<T, CODE>(v.w));
}
__device__ __forceinline__ bool differ(const uint4& a, const uint4& b) {
  return ((a.x ^ b.x) | (a.y ^ b.y) | (a.z ^ b.z) | (a.w ^ b.w)) != 0;
}

// The tiles of STEP positions of [lo, hi) (lo a multiple of STEP) that not every row sees,
// with rows between positions p0 and p1: those below `behind` and from `ahead` on.
struct Edges {
  int behind, ahead;
};
template <int STEP>
__device__ __forceinline__ Edges edges_of(int window, int p0, int p1, int lo, int hi) {
  const int64_t w = window > 0 ? (int64_t)p1 - window + 1 : 0;      // the last row sees from here on
  Edges e;
  e.behind = w > lo ? (int)min64(hi, (w + STEP - 1) / STEP * STEP) : lo;
  e.ahead = p0 + 1 < hi ? max(e.behind, max(lo, p0 + 1) / STEP * STEP) : hi;
  return e;
}

// Adds to one row's sum, by one warp and DIM/32 elements a lane, the elements that are no
// finite numbers of the edges' positions that it sees. Weights do not matter to them: any
// that is above zero leaves an infinity or NaN as it is.
template <class T, Code CODE, int DIM>
__device__ __forceinline__ void add_seen(const BatchArgs& b, const CacheArgs& c, int window, int i,
                                         int kvh, int pos, int lo, const Edges& edge, int hi,
                                         float* acc) {
  constexpr int N = DIM / 32;
  if (window > 0) lo = max(lo, pos - window + 1);
#pragma unroll 1
  for (int j = lo; j < hi; ++j) {
    if (j >= edge.behind && j < edge.ahead) j = edge.ahead;
    if (j > pos || j >= hi) break;
    int slot = 0;
    const int page = page_of(c, b, i, j, slot);
    if (page < 0) continue;
    float y[N];
    cached<T, CODE, DIM>(c.v, page * c.s_page + slot * c.s_token + kvh * c.s_head,
                         threadIdx.x & 31, y);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (!(fabsf(y[e]) < INFINITY)) acc[e] += y[e];
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
