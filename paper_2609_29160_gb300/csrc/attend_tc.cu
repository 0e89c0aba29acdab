// Attention of many new tokens (chunks of prompts) over a paged cache, on the
// tensor cores with their accumulators in tensor memory.
//
// The same sum as k_attend (attend.cu), for sequences with more rows (new tokens x
// query heads of a cache head) than its 16-row tiles serve well: these calls are
// bound by the products, 4 * dim operations a (row, position). One CTA takes two
// tiles of 128 rows against a part of the context, 128 positions at a time:
//
//   S = Q K^T       both operands in shared memory, S (128 x 128, float) in TMEM
//   P = exp2(S - m) a thread a row: S out of TMEM, P back over it in 16 bits
//   O += P V        P from TMEM, V from shared memory, O (128 x dim, float) in TMEM
//
// While one tile's warps take exponentials the tensor cores multiply for the other.
// O is only rescaled when a row's maximum has grown by more than 2^8 since the last
// time (weights then reach 256, far inside either 16-bit type's range; m and l are
// exact in any case), so the pass over O is rare.
//
// Warps 0-3, 4-7: a tile's rows. Warps 8-11: copies, through pages, of keys and
// values into a ring of 128-token tiles (codes are converted on the way: both kinds
// are exact in 16 bits; the scales go into the scores and weights instead). Warp 12
// issues the products. Registers go to the row warps.
#include <algorithm>

#include "attend.cuh"
#include "attend_tc.h"
#include "internal.h"

namespace tre {
namespace {

constexpr int kThreads = 512, kRows = 128, kTok = 128;
constexpr long long kWaitClocks = 4000000000ll;

__device__ __forceinline__ uint32_t smem_of(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(smem_of(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(smem_of(b)) : "memory");
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
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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
// D (TMEM) = or += A * B, both operands in shared memory / A in TMEM
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{ .reg .pred p; setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{ .reg .pred p; setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}

// Shared-memory operand in rows of 128 bytes, 16-byte pieces of row r at piece ^ (r & 7).
// lead: bytes to the next 64 elements along the dense axis (where that axis is not
// the one summed over), 1024 bytes to the next eight rows.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t lead) {
  return (uint64_t)((at >> 4) & 0x3fff) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         1ull << 46 | 2ull << 61;
}
template <class T> __host__ __device__ constexpr uint32_t idesc_of(int n, bool b_turned) {
  const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (b_turned ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 |
         (uint32_t)(kRows >> 4) << 24;
}

template <Code CODE, int DIM> struct Tc {
  static constexpr bool CODED = CODE != Code::kHalf;
  static constexpr int BUF = kTok * DIM * 2;            // a tile of keys or values
  static constexpr int RING = DIM == 128 ? (CODED ? 4 : 5) : (CODED ? 8 : 8);
  static constexpr int META = 8;                        // tiles whose scales and masks are kept
  static constexpr int Q = 2 * kRows * DIM * 2;
  static constexpr int AT_RING = Q;
  static constexpr int AT_OFF = AT_RING + RING * BUF;   // int64 [2][kTok]
  static constexpr int AT_MASK = AT_OFF + 2 * kTok * 8; // uint32 [META][4]
  static constexpr int AT_SCALE = AT_MASK + META * 16;  // float [META][3][kTok]
  static constexpr int AT_BAR = AT_SCALE + (CODED ? META * 3 * kTok * 4 : 0);
  static constexpr int BARS = 2 * RING + META + 7;
  static constexpr int SMEM = AT_BAR + BARS * 8 + 16;
};

// 16 bytes of codes as 16 elements of T
template <class T, Code CODE>
__device__ __forceinline__ void widen(const uint4& v, uint4& lo, uint4& hi) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t r[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[4];
    codes4(w[i], x, CODE == Code::kI8);
    r[2 * i] = pack<T>(x[0], x[1]);
    r[2 * i + 1] = pack<T>(x[2], x[3]);
  }
  lo = make_uint4(r[0], r[1], r[2], r[3]);
  hi = make_uint4(r[4], r[5], r[6], r[7]);
}

template <class T, Code CODE, int DIM>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(AttendArgs a, BatchArgs b, CacheArgs c, tre_diag* diag) {
  using L = Tc<CODE, DIM>;
  extern __shared__ __align__(1024) uint8_t sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kvh = blockIdx.x % c.heads;
  int rest = blockIdx.x / c.heads;
  const int sp = rest % a.parts;
  rest /= a.parts;
  const int i = rest % b.n_seq;
  const int rt0 = a.row_tiles - 1 - rest / b.n_seq;     // the longest ranges first
  const Seq sq = seq_of(b, i);
  const int rows = sq.n * a.group, base = sq.ctx - sq.n;
  if (rows <= a.few || rt0 * 2 * kRows >= rows) return;

  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + L::AT_BAR);
  uint64_t *full = bars, *empty = bars + L::RING, *meta = empty + L::RING, *s_full = meta + L::META,
           *p_full = s_full + 2, *o_done = p_full + 2, *q_full = o_done + 2;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(bars + L::BARS);
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_at + 1);
  int64_t* off_s = reinterpret_cast<int64_t*>(sm + L::AT_OFF);
  uint32_t* mask_s = reinterpret_cast<uint32_t*>(sm + L::AT_MASK);
  float* scale_s = reinterpret_cast<float*>(sm + L::AT_SCALE);

  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     smem_of(tmem_at))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) *dead = 0;

  // Rows r0.. of the block's turn: the two tiles' positions, and how many 128-token
  // tiles each sees. (One turn, unless a sequence has more rows than the host said.)
  int r0, lo, hi, n_x[2], n;
  uint32_t tmem;
  auto turn = [&](int rt) {
    r0 = rt * 2 * kRows;
    const int end = min(r0 + 2 * kRows, rows) - 1;
    range_of(sq, c, b, a.window, a.by_group.div(r0), a.by_group.div(end), lo, hi);
    part_of<kTok>(a, sp, lo, hi);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int f = r0 + x * kRows, l = min(f + kRows, rows) - 1;
      int l2 = 0, h2 = 0;
      if (f < rows) range_of(sq, c, b, a.window, a.by_group.div(f), a.by_group.div(l), l2, h2);
      h2 = min(h2, hi);
      n_x[x] = h2 > lo ? (h2 - lo + kTok - 1) / kTok : 0;
    }
    n = max(n_x[0], n_x[1]);
    __syncthreads();
    if (tid == 0) {
      // (every arrival of an earlier turn has been waited for)
      if (rt != rt0)
        for (int k = 0; k < L::BARS; ++k)
          asm volatile("mbarrier.inval.shared.b64 [%0];" ::"r"(smem_of(bars + k)) : "memory");
      for (int k = 0; k < L::RING; ++k) {
        bar_init(full + k, 128);
        bar_init(empty + k, 1);
      }
      for (int k = 0; k < L::META; ++k) bar_init(meta + k, 128);
      for (int x = 0; x < 2; ++x) {
        bar_init(s_full + x, 1);
        bar_init(p_full + x, 128);
        bar_init(o_done + x, 1);
      }
      bar_init(q_full, 256);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    tmem = *tmem_at;
  };

  // Registers move once: 184 for the row warps, 96 for the copies, 48 for the rest,
  // together the launch's 4 x 128 (in groups of four warps).
  if (warp < 8) {
    // ---- rows --------------------------------------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    for (int rt = rt0; rt * 2 * kRows < rows; rt += a.row_tiles) {
      turn(rt);
      const int x = warp >> 2, row = (warp & 3) * 32 + lane, r = r0 + x * kRows + row;
      const int n_mine = n_x[x];
      // queries: 16-byte pieces, neighbouring lanes along a row
      {
        constexpr int PPR = DIM / 8, RPW = 32 / PPR;
        uint8_t* q_s = sm + x * kRows * DIM * 2;
        const int piece = lane % PPR;
#pragma unroll 4
        for (int k = 0; k < 32 / RPW; ++k) {
          const int rr = (warp & 3) * 32 + k * RPW + lane / PPR, rg = r0 + x * kRows + rr;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (rg < rows) {
            const int t = a.by_group.div(rg);
            const T* p = reinterpret_cast<const T*>(a.q) + (int64_t)(sq.start + t) * a.q_row +
                         (int64_t)(kvh * a.group + (rg - t * a.group)) * a.q_head;
            v = reinterpret_cast<const uint4*>(p)[piece];
          }
          const int hf = piece >> 3, pc = piece & 7;
          *reinterpret_cast<uint4*>(q_s + hf * (kRows * 128) + rr * 128 + ((pc ^ (rr & 7)) << 4)) = v;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(q_full);
      }
      const int tok = a.by_group.div(min(r, rows - 1));
      const int pos = base + tok;
      const int first = base + a.by_group.div(r0 + x * kRows < rows ? r0 + x * kRows : 0);
      const int last = base + a.by_group.div(min(r0 + x * kRows + kRows, rows) - 1);
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t s_at = tmem + lanes + x * kTok, o_at = tmem + lanes + 256 + x * 128;
      float m = -INFINITY, l = 0.f;
      bool alive = true;
#pragma unroll 1
      for (int k = 0; k < n_mine; ++k) {
        const int ms = k % L::META;
        if (!bar_wait(meta + ms, (k / L::META) & 1, dead) || !bar_wait(s_full + x, k & 1, dead)) {
          alive = false;
          break;
        }
        tmem_after();
        uint32_t s[kTok];
#pragma unroll
        for (int h = 0; h < 4; ++h) tmem_ld32(s_at + 32 * h, s + 32 * h);
        tmem_wait_ld();
        const int j0 = lo + k * kTok;
        const uint4 held = *reinterpret_cast<const uint4*>(mask_s + ms * 4);
        const bool whole = (held.x & held.y & held.z & held.w) == 0xffffffffu &&
                           j0 + kTok - 1 <= first && (a.window == 0 || j0 > last - a.window);
        const float4* ks4 = reinterpret_cast<const float4*>(scale_s + ms * 3 * kTok);
        const float4* vs4 = ks4 + kTok / 4;
        const float4* lv4 = vs4 + kTok / 4;
        if constexpr (L::CODED) {
#pragma unroll
          for (int e = 0; e < kTok / 4; ++e) {
            const float4 f = ks4[e];
            s[4 * e] = __float_as_uint(__uint_as_float(s[4 * e]) * f.x);
            s[4 * e + 1] = __float_as_uint(__uint_as_float(s[4 * e + 1]) * f.y);
            s[4 * e + 2] = __float_as_uint(__uint_as_float(s[4 * e + 2]) * f.z);
            s[4 * e + 3] = __float_as_uint(__uint_as_float(s[4 * e + 3]) * f.w);
          }
        }
        if (!whole) {
          const uint32_t hw[4] = {held.x, held.y, held.z, held.w};
          const int top = pos - j0, bottom = a.window ? pos - a.window + 1 - j0 : 0;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int t = min(max(top - 32 * h + 1, 0), 32), u = min(max(bottom - 32 * h, 0), 32);
            const uint32_t below = t == 32 ? 0xffffffffu : (1u << t) - 1;
            const uint32_t above = u == 32 ? 0u : 0xffffffffu << u;
            const uint32_t see = hw[h] & below & above;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(see >> e & 1)) s[32 * h + e] = 0xff800000u;
          }
        }
        float t0 = -INFINITY, t1 = -INFINITY, t2 = -INFINITY, t3 = -INFINITY;
        if constexpr (L::CODED) {
          // a value's scale counts in its weight: the largest weight is below one
#pragma unroll
          for (int e = 0; e < kTok / 4; ++e) {
            const float4 f = lv4[e];
            t0 = fmaxf(t0, __uint_as_float(s[4 * e]) + f.x);
            t1 = fmaxf(t1, __uint_as_float(s[4 * e + 1]) + f.y);
            t2 = fmaxf(t2, __uint_as_float(s[4 * e + 2]) + f.z);
            t3 = fmaxf(t3, __uint_as_float(s[4 * e + 3]) + f.w);
          }
        } else {
#pragma unroll
          for (int e = 0; e < kTok; e += 4) {
            t0 = fmaxf(t0, __uint_as_float(s[e]));
            t1 = fmaxf(t1, __uint_as_float(s[e + 1]));
            t2 = fmaxf(t2, __uint_as_float(s[e + 2]));
            t3 = fmaxf(t3, __uint_as_float(s[e + 3]));
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
#pragma unroll
            for (int h = 0; h < DIM / 32; ++h) {
              uint32_t o[32];
              tmem_ld32(o_at + 32 * h, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st32(o_at + 32 * h, o);
            }
          }
        }
        const float use = m == -INFINITY ? 0.f : m;
        float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[32];
#pragma unroll
          for (int e = 0; e < 64; e += 4) {
            const int at = 64 * h + e;
            float y[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const float v = __uint_as_float(s[at + z]);
              y[z] = exp2_fast(L::CODED ? v - use : __fmaf_rn(v, a.scale2, -use));
            }
            l0 += y[0];
            l1 += y[1];
            l2 += y[2];
            l3 += y[3];
            if constexpr (L::CODED) {
              const float4 f = vs4[at / 4];
              const float w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
              for (int z = 0; z < 4; ++z)
                y[z] = !whole && s[at + z] == 0xff800000u ? 0.f : y[z] * w[z];
            }
            p[e / 2] = pack<T>(y[0], y[1]);
            p[e / 2 + 1] = pack<T>(y[2], y[3]);
          }
          tmem_st32(s_at + 32 * h, p);
        }
        l += (l0 + l1) + (l2 + l3);
        tmem_wait_st();
        tmem_before();
        bar_arrive(p_full + x);
      }
      if (alive && n_mine > 0 && !bar_wait(o_done + x, 0, dead)) alive = false;
      tmem_after();

      // ---- a thread writes its row ------------------------------------------
      // (a row without weight gives zeros, whatever was multiplied for it)
      const bool mine = r < rows && alive;
      const int h_q = kvh * a.group + (min(r, rows - 1) - tok * a.group);
      const int64_t t_row = (int64_t)(sq.start + tok);
      const float by = m == -INFINITY ? 0.f : a.parts > 1 ? 1.f : div_rn(1.f, l);
      const int64_t at = ((int64_t)sp * b.n_rows + t_row) * a.heads + h_q;
      bool odd = false;
#pragma unroll 1
      for (int h = 0; h < DIM / 32; ++h) {
        uint32_t o[32];
        if (n_mine > 0) {
          tmem_ld32(o_at + 32 * h, o);
          tmem_wait_ld();
        }
        float y[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          y[e] = n_mine > 0 && by != 0.f ? __uint_as_float(o[e]) * by : 0.f;
          odd |= !(fabsf(y[e]) < INFINITY);
        }
        if (mine) {
          if (a.parts > 1) {
            float4* p = reinterpret_cast<float4*>(a.part_o + at * DIM + 32 * h);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              p[e] = make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
          } else {
            uint4* p = reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + t_row * a.o_row +
                                                h_q * a.o_head + 32 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = Vec<T>::put(y + 8 * e);
          }
        }
      }
      if (mine) row_state(a, b, sp, t_row, h_q, m, l);
      // rows with values that are no number, one at a time by the whole warp
      unsigned redo = __ballot_sync(0xffffffffu, mine && odd && m > -INFINITY);
      while (redo) {
        const int who = __ffs(redo) - 1;
        redo &= redo - 1;
        const int64_t tr = __shfl_sync(0xffffffffu, t_row, who);
        const int hq = __shfl_sync(0xffffffffu, h_q, who), ps = __shfl_sync(0xffffffffu, pos, who);
        const float mm = __shfl_sync(0xffffffffu, m, who), bb = __shfl_sync(0xffffffffu, by, who);
        constexpr int EL = DIM / 32;
        float acc[EL];
        row_again<T, CODE, DIM>(a, b, c, i, kvh,
                                reinterpret_cast<const T*>(a.q) + tr * a.q_row + hq * a.q_head, ps,
                                lo, hi, mm, acc);
#pragma unroll
        for (int e = 0; e < EL; ++e) {
          if (a.parts > 1)
            a.part_o[(((int64_t)sp * b.n_rows + tr) * a.heads + hq) * DIM + lane * EL + e] = acc[e];
          else
            (reinterpret_cast<T*>(a.out) + tr * a.o_row + hq * a.o_head)[lane * EL + e] =
                T(acc[e] * bb);
        }
      }
      tmem_before();
    }
  } else if (warp < 12) {
    // ---- copies --------------------------------------------------------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    for (int rt = rt0; rt * 2 * kRows < rows; rt += a.row_tiles) {
      turn(rt);
      const int t = tid - 256;                 // the token whose place this thread finds
      constexpr int CB = L::CODED ? 1 : 2, PPT = DIM * CB / 16;    // 16-byte pieces of a token
      const int piece = t % PPT, tok0 = t / PPT;
      constexpr int TPI = 128 / PPT, ITS = kTok / TPI;
      int page = -1, slot = 0;
      auto look = [&](int k) {
        const int j = lo + k * kTok + t;
        page = k < n && j < hi ? page_of(c, b, i, j, slot) : -1;
      };
      auto note = [&](int k) {                 // its place, mask bit and scales, for tile k
        const bool there = page >= 0;
        off_s[(k & 1) * kTok + t] =
            there ? (page * c.s_page + slot * c.s_token + kvh * c.s_head) * CB : -1;
        const unsigned held = __ballot_sync(0xffffffffu, there);
        const int ms = k % L::META;
        if (lane == 0) mask_s[ms * 4 + (t >> 5)] = held;
        if constexpr (L::CODED) {
          float ks = 0.f, vs = 0.f;
          if (there) {
            const int64_t o = page * c.c_page + slot * c.c_token + kvh * c.c_head;
            ks = c.k_scale[o] * a.scale2;
            vs = c.v_scale[o];
          }
          scale_s[ms * 3 * kTok + t] = ks;
          scale_s[ms * 3 * kTok + kTok + t] = vs;
          scale_s[ms * 3 * kTok + 2 * kTok + t] = weight_exponent(vs);
        }
        bar_arrive(meta + ms);
      };
      look(0);
      bool alive = true;
#pragma unroll 1
      for (int k = 0; k < n; ++k) {
        note(k);
        asm volatile("bar.sync 1, 128;" ::: "memory");
        look(k + 1);
        const int64_t* off = off_s + (k & 1) * kTok;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int seq = 2 * k + kv, buf = seq % L::RING;
          const uint8_t* src = kv ? c.v : c.k;
          uint8_t* dst = sm + L::AT_RING + buf * L::BUF;
          if constexpr (!L::CODED) {
            alive = alive && bar_wait(empty + buf, ((seq / L::RING) & 1) ^ 1, dead);
            if (!alive) break;           // (not out of the loop over k: its barrier is shared)
            const uint32_t to = smem_of(dst) + (piece >> 3) * (kTok * 128);
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
              const int tk = tok0 + it * TPI;
              const int64_t o = off[tk];
              const uint8_t* p = src + (o < 0 ? 0 : o + piece * 16);
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                               to + tk * 128 + (((piece & 7) ^ (tk & 7)) << 4)),
                           "l"(p), "r"(o < 0 ? 0 : 16)
                           : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (seq > 0) {
              asm volatile("cp.async.wait_group 1;" ::: "memory");
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              bar_arrive(full + (seq - 1) % L::RING);
            }
          } else {
            uint4 v[ITS];
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
              const int64_t o = off[tok0 + it * TPI];
              v[it] = make_uint4(0, 0, 0, 0);
              if (o >= 0) v[it] = *reinterpret_cast<const uint4*>(src + o + piece * 16);
            }
            alive = alive && bar_wait(empty + buf, ((seq / L::RING) & 1) ^ 1, dead);
            if (!alive) break;
            // 16 codes are two 16-byte pieces of a row
            uint8_t* to = dst + (piece >> 2) * (kTok * 128);
            const int pc = (piece & 3) * 2;
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
              const int tk = tok0 + it * TPI;
              uint4 w0, w1;
              widen<T, CODE>(v[it], w0, w1);
              *reinterpret_cast<uint4*>(to + tk * 128 + ((pc ^ (tk & 7)) << 4)) = w0;
              *reinterpret_cast<uint4*>(to + tk * 128 + (((pc + 1) ^ (tk & 7)) << 4)) = w1;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive(full + buf);
          }
        }
      }
      if constexpr (!L::CODED) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (alive && n > 0) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          bar_arrive(full + (2 * n - 1) % L::RING);
        }
      }
    }
  } else {
    // ---- products --------------------------------------------------------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    for (int rt = rt0; rt * 2 * kRows < rows; rt += a.row_tiles) {
      turn(rt);
      if (warp == 12) {
        constexpr uint32_t id_s = idesc_of<T>(kTok, false), id_o = idesc_of<T>(DIM, true);
        const uint32_t q_at = smem_of(sm), ring_at = smem_of(sm + L::AT_RING);
        auto scores = [&](int x, int buf) {
          if (lane == 0) {
#pragma unroll
            for (int k = 0; k < DIM / 16; ++k) {
              const uint32_t step = (k / 4) * (kTok * 128) + (k % 4) * 32;
              mma_ss(tmem + x * kTok, operand(q_at + x * kRows * DIM * 2 + step, 16),
                     operand(ring_at + buf * L::BUF + step, 16), id_s, k > 0);
            }
            commit(s_full + x);
          }
        };
        bool alive = n > 0 && bar_wait(q_full, 0, dead) && bar_wait(full, 0, dead);
        if (alive) {
          tmem_after();
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (n_x[x] > 0) scores(x, 0);
          if (lane == 0 && L::RING < 2 * n) commit(empty);
        }
#pragma unroll 1
        for (int k = 0; k < n && alive; ++k) {
          const int vb = (2 * k + 1) % L::RING, kb = (2 * k + 2) % L::RING;
          if (!bar_wait(full + vb, ((2 * k + 1) / L::RING) & 1, dead)) break;
          bool have = false;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (k < n_x[x]) {
              if (!bar_wait(p_full + x, k & 1, dead)) {
                alive = false;
                break;
              }
              tmem_after();
              if (lane == 0) {
#pragma unroll
                for (int s = 0; s < kTok / 16; ++s)
                  mma_ts(tmem + 256 + x * 128, tmem + x * kTok + s * 8,
                         operand(ring_at + vb * L::BUF + s * 2048, kTok * 128), id_o,
                         k > 0 || s > 0);
                if (k == n_x[x] - 1) commit(o_done + x);
              }
            }
            if (k + 1 < n_x[x]) {
              if (!have && !bar_wait(full + kb, ((2 * k + 2) / L::RING) & 1, dead)) {
                alive = false;
                break;
              }
              have = true;
              tmem_after();
              scores(x, kb);
            }
          }
          if (alive && lane == 0) {
            // only where the copies go round once more, so that no arrival is left over
            if (2 * k + 1 + L::RING < 2 * n) commit(empty + vb);
            if (2 * k + 2 + L::RING < 2 * n) commit(empty + kb);
          }
        }
        __syncwarp();
      }
    }
  }
  __syncthreads();
  if (warp == 12) {
    tmem_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(*tmem_at));
  }
  if (tid == 0 && *dead && diag) diag->err = TRE_ETIMEOUT;
}

template <class T, Code CODE, int DIM>
cudaError_t launch_typed(const AttendArgs& a, const BatchArgs& b, const CacheArgs& c,
                         tre_diag* diag, cudaStream_t s) {
  using L = Tc<CODE, DIM>;
  const void* fn = (const void*)k_attend_tc<T, CODE, DIM>;
  cudaError_t e = func_smem_once(fn, L::SMEM, true);
  if (e) return e;
  const int64_t blocks = (int64_t)c.heads * a.parts * b.n_seq * a.row_tiles;
  if (blocks > 2147483647) return cudaErrorInvalidValue;
  k_attend_tc<T, CODE, DIM><<<(unsigned)blocks, kThreads, L::SMEM, s>>>(a, b, c, diag);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_code(int code, int dim, const AttendArgs& a, const BatchArgs& b,
                        const CacheArgs& c, tre_diag* diag, cudaStream_t s) {
  if (code == TRE_E4M3)
    return dim == 64 ? launch_typed<T, Code::kE4m3, 64>(a, b, c, diag, s)
                     : launch_typed<T, Code::kE4m3, 128>(a, b, c, diag, s);
  if (code == TRE_I8)
    return dim == 64 ? launch_typed<T, Code::kI8, 64>(a, b, c, diag, s)
                     : launch_typed<T, Code::kI8, 128>(a, b, c, diag, s);
  return dim == 64 ? launch_typed<T, Code::kHalf, 64>(a, b, c, diag, s)
                   : launch_typed<T, Code::kHalf, 128>(a, b, c, diag, s);
}

}  // namespace

cudaError_t launch_attend_tc(int dtype, int code, int dim, const AttendArgs& a,
                             const BatchArgs& b, const CacheArgs& c, tre_diag* diag,
                             cudaStream_t s) {
  return dtype == TRE_BF16 ? launch_code<__nv_bfloat16>(code, dim, a, b, c, diag, s)
                           : launch_code<__half>(code, dim, a, b, c, diag, s);
}

}  // namespace tre
