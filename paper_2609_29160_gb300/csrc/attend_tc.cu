// Attention of many new tokens (chunks of prompts) over a paged cache, on the
// tensor cores with their accumulators in tensor memory.
//
// The same sum as k_attend (attend.cu), for sequences with more rows (new tokens x
// query heads of a cache head) than its tiles of 8 or 16 rows serve well: these calls are
// bound by the products, 4 * dim operations a (row, position). One CTA takes two
// tiles of 128 rows against a part of the context, 128 positions at a time:
//
//   S = Q K^T       both operands in shared memory, S (128 x 128, float) in TMEM
//   P = exp2(S - m) S out of TMEM, P back over it in 16 bits (a product's operand has no
//                   more; a second one for the rest would be half of the products again)
//   O += P V        P from TMEM, V from shared memory, O (128 x dim, float) in TMEM
//
// While one tile's warps take exponentials the tensor cores multiply for the other.
// O is only rescaled when a row's maximum has grown by more than 2^8 since the last
// time (weights then reach 256, far inside either 16-bit type's range; m and l are
// exact in any case), so the pass over O is rare.
//
// Whole tiles of 16-bit elements come by tensor copies, a box a page; the last tile of a
// range, and every tile of pages that 8 does not divide, by 16-byte pieces, which leave
// zeros past the range's end.
//
// Warps 0-3, 4-7: a tile's rows, a thread a row with its 128 scores in registers. Warps
// 8-10: copies, through pages, of keys and values into a ring of 128-token tiles (codes
// come into a ring of their own and are widened to halves there, in which both kinds are
// exact; the scales go into the scores and weights instead). Warp 11 issues the products.
//
// 4,096 new tokens after 32,000, 32 heads on 8 of 128, bf16: 1.39 ms in a loop, 1.6
// PFLOP/s; the tensor pipe is busy three quarters of the time, the rest are its operands'
// reads from shared memory and the start of each unit. Dim 64 has half the products for
// the same exponentials: there the chain of a row binds (scores out of TMEM, maximum,
// 128 exponentials, weights back: some 2,600 cycles a tile, and 6,000 to start and end a
// unit): 24 prompts of up to 2,000, 16 heads, f16, 123 us. Two threads a row spill at the
// registers that are then left and took twice the time. Over codes the copy warps' lookups
// and widening bind: 2,048 tokens after 8,000, 32 heads on 8 of 128, 209 us over bf16, 460
// over e4m3, 525 over int8.
#include <cuda.h>

#include <algorithm>
#include <cstring>
#include <numeric>

#include "attend.cuh"
#include "attend_tc.h"
#include "internal.h"

namespace tre {
namespace {

constexpr int kRows = 128, kTok = 128;
constexpr int kRowWarps = 8, kCopyWarp = kRowWarps, kCopyWarps = 3;
constexpr int kMmaWarp = kCopyWarp + kCopyWarps;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr int kUnits = 4;          // units that the copies may be ahead
constexpr int kMarked = 64;        // units that a pass may mark (see Passes)
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
// A whole warp waits. False when the barrier did not come in about two seconds, here
// or in another warp: the warp then does no more work, and every warp meets at the end.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* dead) {
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
  return __all_sync(0xffffffffu, ok);
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
         (uint32_t)(kRows >> 4) << 24;
}

// Keys and values as tensors of (element, slot, head, page), read in boxes of `box`
// slots and 64 elements; box 0: not to be read that way.
struct Maps {
  CUtensorMap k, v;
  int32_t box;
};
__device__ __forceinline__ void box_load(uint32_t dst, const CUtensorMap* map, int x, int slot,
                                         int head, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(smem_of(bar))
      : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(smem_of(b)), "r"(bytes)
               : "memory");
}

// A position's page, asked for now and looked at later.
struct Ask {
  int id = -1, slot = 0;
  __device__ __forceinline__ void at(const CacheArgs& c, const BatchArgs& b, int i, int j,
                                     int end) {
    const int q = (int)c.by_page.div((uint32_t)j);
    slot = j - q * c.page;
    id = j < end && q < b.max_pages ? b.pages[(int64_t)i * b.pages_row + q] : -1;
  }
  __device__ __forceinline__ int page(const CacheArgs& c) const {
    return id >= 0 && id < c.n_pages ? id : -1;
  }
};

// Shared memory of a block, all of it: the queries, and as many tiles of keys and values
// as the rest holds; over codes their raw tiles take a part.
template <Code CODE, int DIM> struct Tc {
  static constexpr bool CODED = CODE != Code::kHalf;
  static constexpr int BUF = kTok * DIM * 2;            // a tile of keys or values
  static constexpr int RING = DIM == 128 ? (CODED ? 3 : 5) : (CODED ? 6 : 8);
  static constexpr int RAW = kTok * DIM, RAWS = CODED ? 3 : 0;   // a tile of codes, and how many
  static constexpr int META = DIM == 128 ? 4 : 8;       // tiles whose scales and masks are kept
  static constexpr int Q = 2 * kRows * DIM * 2;
  static constexpr int AT_RING = Q;
  static constexpr int AT_RAW = AT_RING + RING * BUF;
  static constexpr int AT_MASK = AT_RAW + RAWS * RAW;   // uint32 [META][4]
  static constexpr int AT_SCALE = AT_MASK + META * 16;  // float [META][3][kTok]
  static constexpr int AT_BACK = AT_SCALE + (CODED ? META * 3 * kTok * 4 : 0);  // float [2][kRows]
  static constexpr int AT_BAR = AT_BACK + (CODED ? 2 * kRows * 4 : 0);
  static constexpr int BARS = 2 * RING + 2 * RAWS + META + 10 + 2 * kUnits;
  static constexpr int AT_UNIT = (AT_BAR + BARS * 8 + 16 + 63) / 64 * 64;    // Unit [kUnits]
  static constexpr int AT_PASS = AT_UNIT + kUnits * 64;
  static constexpr int SMEM = AT_PASS + (kMarked + 4) * 4;
  static_assert(SMEM <= 227 * 1024, "shared memory of a block");
};

// Row tiles of sequence i, none where it is k_attend's.
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const BatchArgs& b, int i) {
  if (i >= b.n_seq) return 0;
  const int r = seq_of(b, i).n * a.group;
  return r > a.few ? (r + 2 * kRows - 1) / (2 * kRows) : 0;
}

// The number of parts with the least time by parts_time. The whole warp looks.
__device__ __forceinline__ int choose_parts(AttendArgs& a, const BatchArgs& b, int heads) {
  const int lane = threadIdx.x & 31;
  int units = 0, len = 1;
  for (int from = 0; from < b.n_seq; from += 32) {
    const int tiles = tiles_of(a, b, from + lane);
    units += tiles;
    if (tiles > 0) {
      const Seq s = seq_of(b, from + lane);
      const int64_t seen = a.window > 0 ? (int64_t)a.window + s.n + kTok : s.ctx;
      len = max(len, (int)min64(s.ctx, seen));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    units += __shfl_xor_sync(0xffffffffu, units, o);
    len = max(len, __shfl_xor_sync(0xffffffffu, len, o));
  }
  units *= heads;
  float least = 0.f;
  int parts = 1;
  for (int n = 1; n <= a.parts && (n == 1 || len / n >= 512); ++n) {
    const float cost = parts_time(n, units, len, a.sms);
    if (n == 1 || cost < least) {
      least = cost;
      parts = n;
    }
  }
  a.split = max(kTok, (len + parts - 1) / parts);
  return parts;
}

// A block's piece of work: up to 256 rows of a sequence against one part of its context
// for one cache head. Units go through the sequences' row tiles (of those that are not
// k_attend's), each sequence's longest ranges first, heads fastest: heads of a tile read
// neighbouring memory, rows of a head the same.
struct alignas(64) Unit {
  int i, kvh, sp, r0, rows, start, base, lo, hi;
  int n_x[2];                     // 128-token tiles that each half of the rows sees
  uint32_t u;                     // its number
  int marked;                     // (see Passes)
  // The whole warp looks; false past the last unit.
  __device__ __forceinline__ bool find(const AttendArgs& a, const BatchArgs& b,
                                       const CacheArgs& c, uint32_t u) {
    const int lane = threadIdx.x & 31;
    // (blocks that take units in turn) every other round backwards, so that none has the
    // longer end of each
    const uint32_t round = u / gridDim.x;
    if (!a.next && (round & 1)) u = round * gridDim.x + (gridDim.x - 1 - (u - round * gridDim.x));
    kvh = (int)(u % c.heads);
    u /= c.heads;
    sp = (int)(u % a.parts);
    int t = (int)(u / a.parts);
    i = -1;
    int tiles = 0, rt = 0;
    for (int from = 0; from < b.n_seq; from += 32) {
      const int mine = tiles_of(a, b, from + lane);
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, t < upto);
      if (past) {
        const int who = __ffs(past) - 1;
        i = from + who;
        tiles = __shfl_sync(0xffffffffu, mine, who);
        rt = tiles - 1 - (int)(t - (__shfl_sync(0xffffffffu, upto, who) - tiles));
        break;
      }
      t -= __shfl_sync(0xffffffffu, upto, 31);
    }
    if (i < 0) return false;
    const Seq s = seq_of(b, i);
    start = s.start;
    rows = s.n * a.group;
    base = s.ctx - s.n;
    r0 = rt * 2 * kRows;
    const int end = min(r0 + 2 * kRows, rows) - 1;
    range_of<kTok>(s, c, b, a.window, a.by_group.div(r0), a.by_group.div(end), lo, hi);
    part_of<kTok>(a, sp, lo, hi);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int f = r0 + x * kRows, l = min(f + kRows, rows) - 1;
      int l2 = 0, h2 = 0;
      if (f < rows) range_of<kTok>(s, c, b, a.window, a.by_group.div(f), a.by_group.div(l), l2, h2);
      h2 = min(h2, hi);
      n_x[x] = h2 > lo ? (h2 - lo + kTok - 1) / kTok : 0;
    }
    return true;
  }
};

// A block's units go in passes. Where a row comes out as no number, which a value that it
// does not see may have done (zero times infinity), the unit is marked, and after the
// pass the marked ones are done once more with those values left out (a careful pass; the
// rows that do see them get them back at its end, from give_back). A pass ends with the last
// unit, or early where the marked ones fill their list. Healthy values have one pass and
// pay a sum a row for it; values that are none cost a second one, whatever the context's
// length, and no wait takes longer for it.
struct Passes {
  uint32_t unit[kMarked];
  uint32_t marked, done;           // units marked, and of those done again
  int careful, more;               // the pass is one; it ended early
};

// 16 bytes of codes as 16 halves
template <Code CODE> __device__ __forceinline__ void widen(const uint4& v, uint4& lo, uint4& hi) {
  lo = make_uint4(halves<CODE>(v.x), halves<CODE>(v.x >> 16), halves<CODE>(v.y),
                  halves<CODE>(v.y >> 16));
  hi = make_uint4(halves<CODE>(v.z), halves<CODE>(v.z >> 16), halves<CODE>(v.w),
                  halves<CODE>(v.w >> 16));
}

// Which of the 32 positions from j on (below `to`) hold an element that is no finite number:
// a lane looks at one position's values.
template <class T, Code CODE, int DIM>
__device__ unsigned unfinite(const BatchArgs& b, const CacheArgs& c, int i, int kvh, int j, int to) {
  constexpr int CB = CODE == Code::kHalf ? 2 : 1;
  j += threadIdx.x & 31;
  int slot = 0;
  const int page = j < to ? page_of(c, b, i, j, slot) : -1;
  bool any = false;
  if (page >= 0) {
    const uint4* p = reinterpret_cast<const uint4*>(
        c.v + (page * c.s_page + slot * c.s_token + kvh * c.s_head) * CB);
#pragma unroll 2
    for (int k = 0; k < DIM * CB / 16; ++k) {
      const uint4 v = p[k];
      any |= differ(v, finite<T, CODE>(v));
    }
  }
  return __ballot_sync(0xffffffffu, any);
}

// A unit's rows from r0 on, every `step`th, get back by one warp what add_seen (attend.cuh)
// adds to one.
template <class T, Code CODE, int DIM>
__device__ void give_back(const AttendArgs& a, const BatchArgs& b, const CacheArgs& c, const Unit& w,
                          int r0, int step) {
  constexpr int N = DIM / 32;
  const int lane = threadIdx.x & 31;
  const Edges edge = edges_of<kTok>(a.window, w.base + a.by_group.div(w.r0),
                                    w.base + a.by_group.div(min(w.r0 + 2 * kRows, w.rows) - 1),
                                    w.lo, w.hi);
  for (int j0 = w.lo; j0 < w.hi; j0 += 32) {     // (32 divides the first edge)
    if (j0 == edge.behind) j0 = edge.ahead;
    unsigned left = unfinite<T, CODE, DIM>(b, c, w.i, w.kvh, j0, w.hi);
    while (left) {
      const int j = j0 + __ffs(left) - 1;
      left &= left - 1;
      int slot = 0;
      const int page = page_of(c, b, w.i, j, slot);
      float y[N];
      cached<T, CODE, DIM>(c.v, page * c.s_page + slot * c.s_token + w.kvh * c.s_head, lane, y);
#pragma unroll 1
      for (int r = r0; r < min(w.r0 + 2 * kRows, w.rows); r += step) {
        const int t = a.by_group.div(r), pos = w.base + t, h = w.kvh * a.group + (r - t * a.group);
        if (j > pos || (a.window > 0 && j <= pos - a.window)) continue;
        const int64_t row = (int64_t)(w.start + t);
        float* part = a.part_o + (((int64_t)w.sp * a.part_rows + row) * a.heads + h) * DIM + lane * N;
        T* out = reinterpret_cast<T*>(a.out) + row * a.o_row + (int64_t)h * a.o_head + lane * N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (fabsf(y[e]) < INFINITY) continue;
          if (a.parts > 1) part[e] += y[e];
          else out[e] = T((float)out[e] + y[e]);
        }
      }
    }
  }
}

template <class T, Code CODE, int DIM>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(AttendArgs a, BatchArgs b, CacheArgs c, const __grid_constant__ Maps maps,
            tre_diag* diag) {
  using L = Tc<CODE, DIM>;
  // codes are multiplied as halves, and queries and weights with them
  using CT = typename std::conditional<L::CODED, __half, T>::type;
  extern __shared__ __align__(1024) uint8_t sm[];
  const int tid = threadIdx.x, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;");      // k_attend may run beside
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (a.parts > 1) {
    a.parts = choose_parts(a, b, c.heads);
    if (blockIdx.x == 0 && tid == 0) *a.parts_taken = a.parts;
  }
  {
    Unit w;
    if (!w.find(a, b, c, blockIdx.x)) return;
  }

  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + L::AT_BAR);
  uint64_t *full = bars, *empty = bars + L::RING, *meta = empty + L::RING, *s_full = meta + L::META,
           *p_full = s_full + 2, *o_done = p_full + 4, *q_full = o_done + 2,
           *u_full = q_full + 2, *u_empty = u_full + kUnits, *raw_full = u_empty + kUnits,
           *raw_empty = raw_full + L::RAWS;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(bars + L::BARS);
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_at + 1);
  uint32_t* mask_s = reinterpret_cast<uint32_t*>(sm + L::AT_MASK);
  float* scale_s = reinterpret_cast<float*>(sm + L::AT_SCALE);
  float* back_s = reinterpret_cast<float*>(sm + L::AT_BACK);
  const volatile Unit* units = reinterpret_cast<const volatile Unit*>(sm + L::AT_UNIT);
  volatile Passes* passes = reinterpret_cast<volatile Passes*>(sm + L::AT_PASS);

  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     smem_of(tmem_at))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) {
    *dead = 0;
    passes->marked = passes->done = 0;
    passes->careful = passes->more = 0;
    for (int k = 0; k < L::RING; ++k) {
      bar_init(full + k, kCopyWarps);
      bar_init(empty + k, 1);
    }
    for (int k = 0; k < L::META; ++k) bar_init(meta + k, 4);
    for (int x = 0; x < 2; ++x) {
      bar_init(s_full + x, 1);
      bar_init(p_full + 2 * x, kRowWarps / 2);
      bar_init(p_full + 2 * x + 1, kRowWarps / 2);
      bar_init(o_done + x, 1);
      bar_init(q_full + x, kRowWarps / 2);
    }
    for (int k = 0; k < L::RAWS; ++k) {
      bar_init(raw_full + k, kCopyWarps);
      bar_init(raw_empty + k, kCopyWarps);
    }
    for (int k = 0; k < kUnits; ++k) {
      bar_init(u_full + k, 1);
      bar_init(u_empty + k, kRowWarps + kCopyWarps);     // (one copy warp writes it)
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_at, 0);
  // Codes of integers are finite: their units are never marked.
  constexpr bool PASSES = CODE != Code::kI8;
  // The end of a pass, where every warp comes: whether there is another. `last`: what a warp
  // does when the rows of a careful one are written.
  auto next_pass = [&](auto last) {
    const bool was_careful = passes->careful;
    __syncthreads();
    if (!PASSES || *dead) return false;
    const bool again = !was_careful && passes->marked > 0;
    if (was_careful) last();
    if (!again && !passes->more) return false;
    if (tid == 0) passes->careful = again;
    __syncthreads();
    return true;
  };
  auto finish = [&]() {
    // A block that has given up does not know which of its copies and products are still on
    // their way into its shared and tensor memory: it stays some 20 ms, far longer than any
    // takes, before it lets go of them.
    if (*dead) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      const long long from = clock64();
      while (clock64() - from < kDrainClocks) {
      }
      __syncthreads();
    }
    if (warp == kMmaWarp) {
      tmem_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(*tmem_at));
    }
    if (tid == 0 && *dead && diag) diag->err = TRE_ETIMEOUT;
  };

  // Registers move once, from the launch's 3 x 168 (in groups of four warps) to twice
  // 208 for the rows and 88 for copies and products.
  if (warp < kRowWarps) {
    // ---- rows --------------------------------------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // (counted over the block's units: the barriers' phases)
    uint32_t n_tile = 0, n_own = 0, n_unit = 0;
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    bool alive = true;
    // Queries of a unit: 16-byte pieces, neighbouring lanes along a row
    constexpr int PPR = DIM / 8, RPW = 32 / PPR, QS = 32 / RPW;
    const int q_row0 = (warp & 3) * 32 + lane / PPR, q_piece = lane % PPR;
    auto q_load = [&](const volatile Unit* w, uint4* v) {
      const int left = w->rows - w->r0 - x * kRows;      // rows of this tile
      const uint32_t r = w->r0 + x * kRows + q_row0;
      const T* from = reinterpret_cast<const T*>(a.q) + (int64_t)w->start * a.q_row +
                      (int64_t)(w->kvh * a.group) * a.q_head + q_piece * 8;
#pragma unroll
      for (int k = 0; k < QS; ++k) {
        const int t = a.by_group.div(r + k * RPW), g = r + k * RPW - t * a.group;
        const T* p = from + ((int64_t)t * a.q_row + (int64_t)g * a.q_head);
        v[k] = make_uint4(0, 0, 0, 0);
        if (q_row0 + k * RPW < left) v[k] = *reinterpret_cast<const uint4*>(p);
      }
    };
    auto q_store = [&](uint4* v) {
      if constexpr (L::CODED && !std::is_same<T, CT>::value) {
        // bfloat16 queries as halves, each row divided by the power of two of its largest
        // element (what is below 2^-24 of that is cut); its scores get it back
#pragma unroll
        for (int k = 0; k < QS; ++k) {
          float y[8], top = 0.f;
          Vec<T>::get(v[k], y);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(y[e]));
#pragma unroll
          for (int o = PPR / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          const int ex = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
          if (q_piece == 0)
            back_s[x * kRows + q_row0 + k * RPW] = __uint_as_float((uint32_t)ex << 23);
          const float by = __uint_as_float((uint32_t)(254 - ex) << 23);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] *= by;
          v[k] = Vec<CT>::put(y);
        }
      }
      uint8_t* q_s = sm + x * kRows * DIM * 2 + (q_piece >> 3) * (kRows * 128);
#pragma unroll
      for (int k = 0; k < QS; ++k) {
        const int rr = q_row0 + k * RPW;
        *reinterpret_cast<uint4*>(q_s + rr * 128 + (((q_piece & 7) ^ (rr & 7)) << 4)) = v[k];
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bar_arrive_warp(q_full + x);
    };
    uint32_t nu = 0;
    while (true) {
      alive = bar_wait(u_full + nu % kUnits, (nu / kUnits) & 1, dead);
      if (alive && units[nu % kUnits].i >= 0 && units[nu % kUnits].n_x[x] > 0) {
        uint4 v[QS];
        q_load(units + nu % kUnits, v);
        q_store(v);
      }
      while (alive) {
        // (what the tile loop does not need stays in shared memory)
        const volatile Unit* w = units + nu % kUnits;
        if (w->i < 0) break;
        const int n_mine = w->n_x[x], lo = w->lo;
        int pos, first, last;
        {
          const int rows = w->rows, r0 = w->r0 + x * kRows, base = w->base;
          pos = base + a.by_group.div(min(r0 + row, rows - 1));
          first = base + a.by_group.div(r0 < rows ? r0 : 0);
          last = base + a.by_group.div(min(r0 + kRows, rows) - 1);
        }
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + x * kTok, o_at = tmem + lanes + 256 + x * 128;
        const float back =
            L::CODED && !std::is_same<T, CT>::value ? back_s[x * kRows + row] : 1.f;
        float m = -INFINITY, l = 0.f;
#pragma unroll 1
        for (int k = 0; k < n_mine; ++k) {
          const int ms = (n_tile + k) % L::META;
          if (!bar_wait(meta + ms, ((n_tile + k) / L::META) & 1, dead) ||
              !bar_wait(s_full + x, (n_own + k) & 1, dead)) {
            alive = false;
            break;
          }
          tmem_after();
          uint32_t v[kTok];
          tmem_ld32(s_at, v);
          tmem_ld32(s_at + 32, v + 32);
          const int j0 = lo + k * kTok;
          const uint4 held = *reinterpret_cast<const uint4*>(mask_s + ms * 4);
          const bool whole = (held.x & held.y & held.z & held.w) == 0xffffffffu &&
                             j0 + kTok - 1 <= first && (a.window == 0 || j0 > last - a.window);
          const float* meta_s = scale_s + ms * 3 * kTok;
          float t0 = -INFINITY, t1 = -INFINITY, t2 = -INFINITY, t3 = -INFINITY;
          // half of the scores at a time, the other on its way
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            tmem_wait_ld(v + 64 * hf);
            tmem_wait_ld(v + 64 * hf + 32);
            if (hf == 0) {
              tmem_ld32(s_at + 64, v + 64);
              tmem_ld32(s_at + 96, v + 96);
            }
            if constexpr (L::CODED) {
#pragma unroll
              for (int e = 64 * hf; e < 64 * hf + 64; e += 4) {
                const float4 f = *reinterpret_cast<const float4*>(meta_s + e);
                mul2(v + e, f.x, f.y);
                mul2(v + e + 2, f.z, f.w);
              }
            }
            if (!whole) {
              const uint32_t hw[2] = {hf ? held.z : held.x, hf ? held.w : held.y};
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int c0 = 64 * hf + 32 * y;
                const int to = min(max(pos - j0 - c0 + 1, 0), 32);
                const int from = a.window ? min(max(pos - a.window + 1 - j0 - c0, 0), 32) : 0;
                const uint32_t see = hw[y] & (to == 32 ? 0xffffffffu : (1u << to) - 1) &
                                     (from == 32 ? 0u : 0xffffffffu << from);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (!(see >> e & 1)) v[c0 + e] = 0xff800000u;
              }
            }
#pragma unroll
            for (int e = 64 * hf; e < 64 * hf + 64; e += 8) {
              if constexpr (L::CODED) {
                // a value's scale counts in its weight: the largest weight is below one by
                // the scale's power of two
#pragma unroll
                for (int y = 0; y < 8; y += 4) {
                  const float4 f = *reinterpret_cast<const float4*>(meta_s + 2 * kTok + e + y);
                  uint32_t z[4] = {v[e + y], v[e + y + 1], v[e + y + 2], v[e + y + 3]};
                  fma2(z, back, f.x, f.y);
                  fma2(z + 2, back, f.z, f.w);
                  t0 = max3(t0, __uint_as_float(z[0]), __uint_as_float(z[1]));
                  t1 = max3(t1, __uint_as_float(z[2]), __uint_as_float(z[3]));
                }
              } else {
                t0 = max3(t0, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                t1 = max3(t1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
                t2 = max3(t2, __uint_as_float(v[e + 4]), __uint_as_float(v[e + 5]));
                t3 = max3(t3, __uint_as_float(v[e + 6]), __uint_as_float(v[e + 7]));
              }
            }
          }
          float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3));
          if (!L::CODED) top *= a.scale2;
          if (__any_sync(0xffffffffu, top > m + 8.f || (m == -INFINITY && top > m))) {
            const float mn = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.f : exp2_fast(m - mn);
            m = mn;
            l *= f;
            if (k > 0) {
#pragma unroll 1
              for (int h = 0; h < DIM / 16; ++h) {
                uint32_t o[16];
                tmem_ld16(o_at + 16 * h, o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st16(o_at + 16 * h, o);
              }
            }
          }
          const float use = m == -INFINITY ? 0.f : m;
          uint64_t l0 = 0, l1 = 0;                 // pairs of sums
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            uint32_t p[16];
#pragma unroll
            for (int e = 32 * h; e < 32 * h + 32; e += 4) {
              if constexpr (L::CODED) {
                fma2(v + e, back, -use);
                fma2(v + e + 2, back, -use);
              } else {
                fma2(v + e, a.scale2, -use);
                fma2(v + e + 2, a.scale2, -use);
              }
              float y[4];
#pragma unroll
              for (int z = 0; z < 4; ++z) y[z] = exp2_fast(__uint_as_float(v[e + z]));
              l0 = sum2(l0, y[0], y[1]);
              l1 = sum2(l1, y[2], y[3]);
              if constexpr (L::CODED) {
                const float4 f = *reinterpret_cast<const float4*>(meta_s + kTok + e);
                const float w[4] = {f.x, f.y, f.z, f.w};
                // (a masked position's scale may be anything: its weight stays zero)
#pragma unroll
                for (int z = 0; z < 4; ++z) y[z] = !whole && y[z] == 0.f ? 0.f : y[z] * w[z];
              }
              p[(e - 32 * h) / 2] = pack<CT>(y[0], y[1]);
              p[(e - 32 * h) / 2 + 1] = pack<CT>(y[2], y[3]);
            }
            tmem_st16(s_at + 16 * h, p);
            if (h & 1) {                           // half of the products may begin
              tmem_wait_st();
              tmem_before();
              bar_arrive_warp(p_full + 2 * x + (h >> 1));
            }
          }
          l += halves_sum(l0, l1);
        }
        // the next unit's queries are on their way while the last products run, and its
        // first products run while this one's rows are written
        const uint32_t nn = nu + 1;
        const volatile Unit* wn = units + nn % kUnits;
        alive = alive && bar_wait(u_full + nn % kUnits, (nn / kUnits) & 1, dead);
        {
          const bool more = alive && wn->i >= 0 && wn->n_x[x] > 0;
          uint4 v[QS];
          if (more) q_load(wn, v);
          if (n_mine > 0) alive = alive && bar_wait(o_done + x, n_unit & 1, dead);
          if (more && alive) q_store(v);
        }
        n_tile += max(w->n_x[0], w->n_x[1]);
        n_own += n_mine;
        n_unit += n_mine > 0;
        tmem_after();

        // ---- a thread writes its row ------------------------------------------
        const int i = w->i, kvh = w->kvh, sp = w->sp, hi = w->hi, rows = w->rows;
        const int start = w->start, r = w->r0 + x * kRows + row;
        // (a row without weight gives zeros, whatever was multiplied for it)
        const bool mine = r < rows && alive;
        const int tok = a.by_group.div(min(r, rows - 1));
        const int h_q = kvh * a.group + (min(r, rows - 1) - tok * a.group);
        const int64_t t_row = (int64_t)(start + tok);
        const float by = saw_nothing(m, l) ? 0.f : a.parts > 1 ? 1.f : div_rn(1.f, l);
        const int64_t at = ((int64_t)sp * a.part_rows + t_row) * a.heads + h_q;
        uint64_t sum = 0;                        // (no number where some element is none)
#pragma unroll 1
        for (int h = 0; h < DIM / 32; ++h) {
          uint32_t o[32];
          if (n_mine > 0) {
            tmem_ld32(o_at + 32 * h, o);
            tmem_wait_ld(o);
          }
          float y[32];
#pragma unroll
          for (int e = 0; e < 32; ++e)
            y[e] = n_mine > 0 && by != 0.f ? __uint_as_float(o[e]) * by : 0.f;
          if constexpr (CODE != Code::kI8) {
#pragma unroll
            for (int e = 0; e < 32; e += 2) sum = sum2(sum, y[e], y[e + 1]);
          }
          if (mine) {
            if (a.parts > 1) {
              float4* q = reinterpret_cast<float4*>(a.part_o + at * DIM + 32 * h);
#pragma unroll
              for (int e = 0; e < 8; e += 2)     // 32 bytes at a time: whole sectors
                asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q + e),
                             "f"(y[4 * e]), "f"(y[4 * e + 1]), "f"(y[4 * e + 2]), "f"(y[4 * e + 3]),
                             "f"(y[4 * e + 4]), "f"(y[4 * e + 5]), "f"(y[4 * e + 6]), "f"(y[4 * e + 7])
                             : "memory");
            } else {
              uint4* q = reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + t_row * a.o_row +
                                                  (int64_t)h_q * a.o_head + 32 * h);
              if (a.wide) {
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                  const uint4 f = Vec<T>::put(y + 8 * e), g = Vec<T>::put(y + 8 * e + 8);
                  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q + e),
                               "r"(f.x), "r"(f.y), "r"(f.z), "r"(f.w), "r"(g.x), "r"(g.y), "r"(g.z),
                               "r"(g.w)
                               : "memory");
                }
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = Vec<T>::put(y + 8 * e);
              }
            }
          }
        }
        if (mine) row_state(a, sp, t_row, t_row, h_q, m, l);
        if constexpr (PASSES) {
          // (m is finite: the row saw a number)
          const float all = halves_sum(sum, 0);
          if (__any_sync(0xffffffffu, mine && all != all && m > -INFINITY) && lane == 0 &&
              !passes->careful && atomicExch(const_cast<int*>(&w->marked), 1) == 0)
            passes->unit[atomicAdd(const_cast<uint32_t*>(&passes->marked), 1u)] = w->u;
        }
        tmem_before();
        bar_arrive_warp(u_empty + nu % kUnits);
        ++nu;
      }
      if (alive) bar_arrive_warp(u_empty + nu % kUnits);
      if (!next_pass([] {})) break;
      ++nu;
    }
    return finish();
  }
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (warp < kMmaWarp) {
    // ---- copies --------------------------------------------------------------
    uint32_t n_tile = 0;
    bool alive = true;
    uint32_t u = blockIdx.x;
    uint32_t nu = 0;
    while (true) {
      const bool careful = PASSES && passes->careful;
      for (; alive; ++nu) {
        // units are found here, ahead of those who need them
        Unit w;
        Unit* shared = reinterpret_cast<Unit*>(sm + L::AT_UNIT + nu % kUnits * 64);
        if (warp == kCopyWarp) {
          w.u = u;
          bool full_list = false;
          if (careful) {
            const uint32_t k = passes->done;
            full_list = k == passes->marked;         // (all of it)
            if (!full_list) w.u = passes->unit[k];
            __syncwarp();
            if (lane == 0) passes->done = k + 1;
          } else if (PASSES) {
            // (those that are on their way may be marked yet)
            full_list = passes->marked + kUnits + 1 > kMarked;
          }
          if (full_list || !w.find(a, b, c, w.u)) w.i = -1;
          w.marked = 0;
          if (PASSES && w.i < 0 && !careful && lane == 0) passes->more = full_list;
          alive = bar_wait(u_empty + nu % kUnits, ((nu / kUnits) & 1) ^ 1, dead);
          if (!alive) break;
          if (lane == 0) *shared = w;
          bar_arrive_warp(u_full + nu % kUnits);
        } else {
          alive = bar_wait(u_full + nu % kUnits, (nu / kUnits) & 1, dead);
          if (!alive) break;
          w = *shared;
          bar_arrive_warp(u_empty + nu % kUnits);
        }
        if (w.i < 0) break;
        const int i = w.i, kvh = w.kvh, lo = w.lo, hi = w.hi, n = max(w.n_x[0], w.n_x[1]);
        const int cw = warp - kCopyWarp;
        // its queries into L2, before the row warps get there
        for (int r = w.r0 + cw * 32 + lane; r < min(w.r0 + 2 * kRows, w.rows); r += kCopyWarps * 32) {
          const int t = a.by_group.div(r);
          const T* p = reinterpret_cast<const T*>(a.q) + (int64_t)(w.start + t) * a.q_row +
                       (int64_t)(kvh * a.group + (r - t * a.group)) * a.q_head;
#pragma unroll
          for (int e = 0; e < DIM; e += 64)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p + e));
        }
        constexpr int CB = L::CODED ? 1 : 2, PPT = DIM * CB / 16;    // 16-byte pieces of a token
        constexpr int STEPS = kTok * PPT / 32, TPS = 32 / PPT;       // 32 pieces a step of a warp
        const int piece = lane % PPT, tok0 = lane / PPT;
        // A warp copies the tokens of steps cw, cw + 3, ..; its lanes find their places,
        // and those of the mask and scales: groups of 32 tokens, warp cw group cw and the
        // first warp group 3 too.
        // (What the tables say is looked at a tile later: nothing waits for it.)
        int64_t off[2] = {-1, -1};
        Ask list[2], group[2];
        auto look = [&](int k, bool pieces) {
          const int j0 = lo + k * kTok, end = k < n ? hi : 0;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (pieces) {
              const int q = g * 32 + lane, st = cw + kCopyWarps * (q / TPS);
              list[g].at(c, b, i, j0 + st * TPS + q % TPS, st < STEPS ? end : 0);
            }
            if (g == 0 || cw == 0) group[g].at(c, b, i, j0 + (g ? 96 : cw * 32) + lane, end);
          }
        };
        auto take = [&]() {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int pg = list[g].page(c);
            off[g] = pg < 0 ? -1
                            : (pg * c.s_page + list[g].slot * c.s_token + kvh * c.s_head) * CB;
          }
        };
        auto place = [&](int i_step) {           // of this lane's piece in the warp's step
          const int q = i_step * TPS + tok0;
          const int64_t x = __shfl_sync(0xffffffffu, off[0], q & 31);
          const int64_t y = __shfl_sync(0xffffffffu, off[1], q & 31);
          return q < 32 ? x : y;
        };
        float sc_k[2] = {0.f, 0.f}, sc_v[2] = {0.f, 0.f};
        bool sc_there[2] = {false, false};
        auto scales = [&]() {                    // (asked for when their page is known)
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (g == 1 && cw != 0) break;
            const int pg = group[g].page(c);
            sc_there[g] = pg >= 0;
            const int64_t o = pg * c.c_page + group[g].slot * c.c_token + kvh * c.c_head;
            sc_k[g] = pg >= 0 ? c.k_scale[o] : 0.f;
            sc_v[g] = pg >= 0 ? c.v_scale[o] : 0.f;
          }
        };
        auto note = [&](int k) {                 // mask bits and scales, for tile k
          const int ms = (n_tile + k) % L::META;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (g == 1 && cw != 0) break;
            const int t = (g ? 96 : cw * 32) + lane;
            const bool there = L::CODED ? sc_there[g] : group[g].page(c) >= 0;
            const unsigned held = __ballot_sync(0xffffffffu, there);
            if (lane == 0) mask_s[ms * 4 + (t >> 5)] = held;
            if constexpr (L::CODED) {
              const float ks = sc_k[g] * a.scale2, vs = sc_v[g];
              scale_s[ms * 3 * kTok + t] = ks;
              scale_s[ms * 3 * kTok + kTok + t] = vs;
              scale_s[ms * 3 * kTok + 2 * kTok + t] = weight_exponent(vs);
            }
            bar_arrive_warp(meta + ms);
          }
        };
        // Boxes of whole tiles, every third a warp, one a lane: its page (one that the cache
        // does not have where the table names none: its rows come as zeros).
        const int box = maps.box, boxes = box ? kTok / box : 0;
        const int my_box = cw + kCopyWarps * lane, my_boxes = (boxes + 2 - cw) / kCopyWarps;
        auto whole_box = [&](int k) { return box > 0 && lo + (k + 1) * kTok <= hi; };
        Ask boxed;
        auto ask_box = [&](int k) {
          if (my_box < boxes) boxed.at(c, b, i, lo + k * kTok + my_box * box, k < n ? hi : 0);
        };
        if constexpr (L::CODED) {
          // ---- codes: raw tiles come a tile ahead, and are widened from shared memory ----
          int box_page = 0, box_slot = 0;
          auto fetch = [&](int k, int kv) {
            {
              const uint32_t seq = 2 * (n_tile + k) + kv, buf = seq % L::RAWS;
              const uint8_t* src = (kv ? c.v : c.k) + piece * 16;
              const uint32_t to = smem_of(sm + L::AT_RAW + buf * L::RAW);
              alive = alive && bar_wait(raw_empty + buf, ((seq / L::RAWS) & 1) ^ 1, dead);
              if (!alive) return;
              if (whole_box(k)) {
                if (lane == 0) bar_expect(raw_full + buf, my_boxes * box * DIM);
                __syncwarp();
                if (my_box < boxes)
                  box_load(to + my_box * box * DIM, kv ? &maps.v : &maps.k, 0, box_slot, kvh, box_page,
                           raw_full + buf);
                __syncwarp();
              } else {
#pragma unroll 4
                for (int is = 0; is < (STEPS + 2) / kCopyWarps; ++is) {
                  const int64_t o = place(is);
                  const int st = cw + is * kCopyWarps;
                  if (st >= STEPS) break;
                  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                   to + (st * 32 + lane) * 16),
                               "l"(src + (o < 0 ? 0 : o)), "r"(o < 0 ? 0 : 16)
                               : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                bar_arrive_warp(raw_full + buf);
              }
            }
          };
          auto convert = [&](int k, int kv) {
            const uint32_t seq = 2 * (n_tile + k) + kv, raw = seq % L::RAWS, buf = seq % L::RING;
            alive = alive && bar_wait(raw_full + raw, (seq / L::RAWS) & 1, dead) &&
                    bar_wait(empty + buf, ((seq / L::RING) & 1) ^ 1, dead);
            if (!alive) return;
            // 16 codes are two 16-byte pieces of a row
            const uint4* from = reinterpret_cast<const uint4*>(sm + L::AT_RAW + raw * L::RAW) + lane;
            uint8_t* to = sm + L::AT_RING + buf * L::BUF + (piece >> 2) * (kTok * 128);
            const int pc = (piece & 3) * 2;
#pragma unroll 4
            for (int st = cw; st < STEPS; st += kCopyWarps) {
              const int tk = tok0 + st * TPS;
              uint4 w0, w1;
              widen<CODE>(from[st * 32], w0, w1);
              *reinterpret_cast<uint4*>(to + tk * 128 + ((pc ^ (tk & 7)) << 4)) = w0;
              *reinterpret_cast<uint4*>(to + tk * 128 + (((pc + 1) ^ (tk & 7)) << 4)) = w1;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive_warp(full + buf);
            bar_arrive_warp(raw_empty + raw);
          };
          auto resolve = [&](int k) {            // tile k's places and scales, k + 1 asked for
            box_page = boxed.page(c);
            box_slot = boxed.slot;
            if (box_page < 0) box_page = c.n_pages;
            if (!whole_box(k)) take();
            scales();
            look(k + 1, !whole_box(k + 1));
            ask_box(k + 1);
          };
          look(0, !whole_box(0));
          ask_box(0);
          resolve(0);
          if (n > 0) {
            fetch(0, 0);
            fetch(0, 1);
          }
#pragma unroll 1
          for (int k = 0; k < n && alive; ++k) {
            note(k);
            if (k + 1 < n) resolve(k + 1);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
              if (k + 1 < n) fetch(k + 1, kv);
              convert(k, kv);
            }
          }
        } else {
          look(0, !whole_box(0));
          ask_box(0);
          int pending = -1;                      // a tile copied by pieces, not yet announced
#pragma unroll 1
          for (int k = 0; k < n && alive; ++k) {
            const bool by_box = whole_box(k);
            note(k);
            if (!by_box) take();
            int box_page = boxed.page(c);
            const int box_slot = boxed.slot;
            if (box_page < 0) box_page = c.n_pages;
            look(k + 1, !whole_box(k + 1));
            ask_box(k + 1);
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
              const uint32_t seq = 2 * (n_tile + k) + kv, buf = seq % L::RING;
              const uint8_t* src = (kv ? c.v : c.k) + piece * 16;
              uint8_t* dst = sm + L::AT_RING + buf * L::BUF;
              alive = alive && bar_wait(empty + buf, ((seq / L::RING) & 1) ^ 1, dead);
              if (!alive) break;
              if (by_box) {
                if (lane == 0) bar_expect(full + buf, my_boxes * box * DIM * 2);
                __syncwarp();
                if (my_box < boxes) {
                  const uint32_t to = smem_of(dst) + my_box * box * 128;
#pragma unroll
                  for (int h = 0; h < DIM / 64; ++h)
                    box_load(to + h * (kTok * 128), kv ? &maps.v : &maps.k, h * 64, box_slot, kvh,
                             box_page, full + buf);
                }
                __syncwarp();
              } else {
                const uint32_t to = smem_of(dst) + (piece >> 3) * (kTok * 128);
#pragma unroll 4
                for (int is = 0; is < (STEPS + 2) / kCopyWarps; ++is) {
                  const int64_t o = place(is);
                  const int st = cw + is * kCopyWarps, tk = tok0 + st * TPS;
                  if (st >= STEPS) break;
                  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                   to + tk * 128 + (((piece & 7) ^ (tk & 7)) << 4)),
                               "l"(src + (o < 0 ? 0 : o)), "r"(o < 0 ? 0 : 16)
                               : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (pending >= 0) {
                  asm volatile("cp.async.wait_group 1;" ::: "memory");
                  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                  bar_arrive_warp(full + pending);
                }
                pending = buf;
              }
            }
          }
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          if (alive && pending >= 0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive_warp(full + pending);
          }
        }
        n_tile += n;
        if (careful) continue;
        u += gridDim.x;
        if (a.next && warp == kCopyWarp) {         // whoever is first takes the next unit
          if (lane == 0) u = gridDim.x + atomicAdd(a.next, 1u);
          u = __shfl_sync(0xffffffffu, u, 0);
        }
      }
      if (!next_pass([&] {
            for (uint32_t k = 0; k < passes->marked; ++k) {
              Unit w;
              if (w.find(a, b, c, passes->unit[k]))
                give_back<T, CODE, DIM>(a, b, c, w, w.r0 + warp - kCopyWarp, kCopyWarps);
            }
          }))
        break;
      ++nu;
      if (warp == kCopyWarp) {
        if (lane == 0) {
          passes->done = 0;
          if (!passes->careful) passes->marked = 0;
        }
        __syncwarp();
      }
    }
  } else {
    // ---- products --------------------------------------------------------------
    uint32_t n_tile = 0, n_own[2] = {0, 0}, n_unit[2] = {0, 0};
    bool alive = true;
    uint32_t nu = 0;
    // (a careful pass) values that are no finite numbers out of a tile of the unit's edges
    auto leave_out = [&](const volatile Unit* w, int k, uint8_t* values) {
      const int r0 = w->r0, base = w->base, j = w->lo + k * kTok;
      const Edges edge = edges_of<kTok>(a.window, base + a.by_group.div(r0),
                                        base + a.by_group.div(min(r0 + 2 * kRows, w->rows) - 1),
                                        w->lo, w->hi);
      if (j >= edge.behind && j < edge.ahead) return;
      uint4* v = reinterpret_cast<uint4*>(values);
#pragma unroll 4
      for (int e = lane; e < L::BUF / 16; e += 32) v[e] = finite<CT, Code::kHalf>(v[e]);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    };
    while (true) {
      const bool careful = PASSES && __shfl_sync(0xffffffffu, passes->careful, 0);
      for (; alive; ++nu) {
        alive = bar_wait(u_full + nu % kUnits, (nu / kUnits) & 1, dead);
        if (!alive) break;
        const volatile Unit* w = units + nu % kUnits;
        if (__shfl_sync(0xffffffffu, w->i, 0) < 0) {
          bar_arrive_warp(u_empty + nu % kUnits);
          break;
        }
        const int n_x[2] = {__shfl_sync(0xffffffffu, w->n_x[0], 0),
                            __shfl_sync(0xffffffffu, w->n_x[1], 0)};
        const int n = max(n_x[0], n_x[1]);
        bar_arrive_warp(u_empty + nu % kUnits);
        {
          constexpr uint32_t id_s = idesc_of<CT>(kTok, false), id_o = idesc_of<CT>(DIM, true);
          const uint32_t q_op = operand(smem_of(sm), 16);
          const uint32_t k_op = operand(smem_of(sm + L::AT_RING), 16);
          const uint32_t v_op = operand(smem_of(sm + L::AT_RING), kTok * 128);
          auto scores = [&](int x, int buf) {
            const uint32_t qa = q_op + x * (kRows * DIM * 2 >> 4), ka = k_op + buf * (L::BUF >> 4);
            const uint32_t d = tmem + x * kTok;
#pragma unroll
            for (int k = 0; k < DIM / 16; ++k) {
              const uint32_t step = ((k / 4) * (kTok * 128) + (k % 4) * 32) >> 4;
              mma_ss(d, qa + step, ka + step, id_s, k > 0);
            }
            commit(s_full + x);
          };
          if (n == 0) continue;
          const uint32_t at = 2 * n_tile;
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (n_x[x] > 0) alive = alive && bar_wait(q_full + x, n_unit[x] & 1, dead);
          alive = alive && bar_wait(full + at % L::RING, (at / L::RING) & 1, dead);
          if (alive) {
            tmem_after();
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (n_x[x] > 0 && one_lane()) scores(x, at % L::RING);
            if (one_lane()) commit(empty + at % L::RING);
          }
#pragma unroll 1
          for (int k = 0; k < n && alive; ++k) {
            const uint32_t vs = at + 2 * k + 1, vb = vs % L::RING, kb = (vs + 1) % L::RING;
            alive = bar_wait(full + vb, (vs / L::RING) & 1, dead);
            if (careful && alive) leave_out(w, k, sm + L::AT_RING + vb * L::BUF);
            bool have = false;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (k < n_x[x]) {
                const uint32_t va = v_op + vb * (L::BUF >> 4), d = tmem + 256 + x * 128;
                const uint32_t pa = tmem + x * kTok;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                  alive = alive && bar_wait(p_full + 2 * x + hf, (n_own[x] + k) & 1, dead);
                  tmem_after();
                  if (alive && one_lane()) {
#pragma unroll
                    for (int s = 4 * hf; s < 4 * hf + 4; ++s)
                      mma_ts(d, pa + s * 8, va + s * (2048 >> 4), id_o, k > 0 || s > 0);
                    if (hf && k == n_x[x] - 1) commit(o_done + x);
                  }
                }
              }
              if (k + 1 < n_x[x]) {
                if (!have) alive = alive && bar_wait(full + kb, ((vs + 1) / L::RING) & 1, dead);
                have = true;
                tmem_after();
                if (alive && one_lane()) scores(x, kb);
              }
            }
            if (alive && one_lane()) {
              commit(empty + vb);
              if (k + 1 < n) commit(empty + kb);
            }
          }
          n_tile += n;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            n_own[x] += n_x[x];
            n_unit[x] += n_x[x] > 0;
          }
          __syncwarp();
        }
      }
      // the arrivals that no copy waits for any more
      for (uint32_t s = 2 * n_tile; alive && s > 0 && s + 2 > 2 * n_tile;) {
        --s;
        alive = bar_wait(empty + s % L::RING, (s / L::RING) & 1, dead);
      }
      if (!next_pass([] {})) break;
      ++nu;
    }
  }
  finish();
}

// The driver's encoder of tensor maps, looked up once (it is not part of the runtime).
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                            const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
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

// Maps of a cache. Tiles start at multiples of 128, so a box of the greatest common
// divisor of 128 and the page lies in one page; below 8 slots (or where the encoder
// refuses the strides) tiles are copied by pieces. Elements of 16 bits come in columns of
// 64 with the products' order of pieces, codes in whole rows as they are.
void make_maps(Maps& m, const CacheArgs& c, CUtensorMapDataType type, int dim) {
  m.box = 0;
  const bool coded = type == CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const int box = std::gcd(c.page, kTok), el = coded ? 1 : 2;
  const Encode enc = box >= 8 && c.n_pages > 0 ? encoder() : nullptr;
  if (!enc) return;
  const int64_t st[3] = {c.s_token * el, c.s_head * el, c.s_page * el};
  cuuint64_t strides[3];
  for (int x = 0; x < 3; ++x) {
    if (st[x] <= 0 || st[x] >= (1ll << 40)) return;
    strides[x] = (cuuint64_t)st[x];
  }
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)c.page, (cuuint64_t)c.heads,
                              (cuuint64_t)c.n_pages};
  const cuuint32_t size[4] = {(cuuint32_t)(coded ? dim : 64), (cuuint32_t)box, 1, 1};
  const cuuint32_t one[4] = {1, 1, 1, 1};
  for (int x = 0; x < 2; ++x)
    if (enc(x ? &m.v : &m.k, type, 4, x ? c.v : c.k, dims, strides, size, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            coded ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return;
  m.box = box;
}

template <class T, Code CODE, int DIM>
cudaError_t launch_typed(const AttendArgs& a, const BatchArgs& b, const CacheArgs& c,
                         int64_t units, tre_diag* diag, cudaStream_t s) {
  using L = Tc<CODE, DIM>;
  const void* fn = (const void*)k_attend_tc<T, CODE, DIM>;
  cudaError_t e = func_smem_once(fn, L::SMEM, true);
  if (e) return e;
  if (units > 2000000000) return cudaErrorInvalidValue;
  const int64_t blocks = std::min<int64_t>(units, device_sm_count());
  Maps maps;
  memset(&maps, 0, sizeof(maps));
  make_maps(maps, c,
            CODE != Code::kHalf                       ? CU_TENSOR_MAP_DATA_TYPE_UINT8
            : std::is_same<T, __nv_bfloat16>::value   ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                      : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
            DIM);
  k_attend_tc<T, CODE, DIM><<<(unsigned)blocks, kThreads, L::SMEM, s>>>(a, b, c, maps, diag);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_code(int code, int dim, const AttendArgs& a, const BatchArgs& b,
                        const CacheArgs& c, int64_t units, tre_diag* diag,
                        cudaStream_t s) {
  if (code == TRE_E4M3)
    return dim == 64 ? launch_typed<T, Code::kE4m3, 64>(a, b, c, units, diag, s)
                     : launch_typed<T, Code::kE4m3, 128>(a, b, c, units, diag, s);
  if (code == TRE_I8)
    return dim == 64 ? launch_typed<T, Code::kI8, 64>(a, b, c, units, diag, s)
                     : launch_typed<T, Code::kI8, 128>(a, b, c, units, diag, s);
  return dim == 64 ? launch_typed<T, Code::kHalf, 64>(a, b, c, units, diag, s)
                   : launch_typed<T, Code::kHalf, 128>(a, b, c, units, diag, s);
}

}  // namespace

cudaError_t launch_attend_tc(int dtype, int code, int dim, const AttendArgs& a,
                             const BatchArgs& b, const CacheArgs& c, int64_t units,
                             tre_diag* diag, cudaStream_t s) {
  return dtype == TRE_BF16 ? launch_code<__nv_bfloat16>(code, dim, a, b, c, units, diag, s)
                           : launch_code<__half>(code, dim, a, b, c, units, diag, s);
}

}  // namespace tre
