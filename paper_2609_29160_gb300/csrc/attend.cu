// Attention of new tokens over a paged cache.
//
//   out_r = sum_j softmax_j(scale * q_r . k_j) v_j  over the positions j <= pos(r)
//   (j > pos(r) - window with a window) whose page is mapped
//
// in one pass over the keys and values: a running maximum m, the sum l of
// exp2(s - m), and the weighted sum of values, all in 32 bits.
//
// k_attend takes 8 * NT rows at a time (tokens x query heads of one cache head: the
// heads that share a key read it once) against a part of the context. Its four
// warps each run their own stream of 16-token tiles through a ring of asynchronous
// 16-byte copies of their own, so no warp waits for another before the end, when
// their four (m, l, O) are joined. Products are m16n8k16 matrix instructions with
// positions (then elements) along m and rows along n, S^T = K Q^T and O^T = V^T P^T:
// eight rows, the query heads of one token, fill a tile that way, and a lane holds two
// rows' weights of two positions. Elements of a key and columns of values are taken in
// the order in which a lane's 16-byte reads deliver them, which a sum does not see.
//
// Bound by HBM on 16-bit caches: one token of 96 requests of up to 16,000, 32 query heads
// on 8 of 128, 303 us, 6.3 TB/s. On codes the widening takes half of the issue slots as
// well: 8 requests of up to 120,000, 64 heads on 8, e4m3, 202 us, 5.6 TB/s.
#include <algorithm>

#include "attend.cuh"
#include "attend_tc.h"
#include "internal.h"

namespace tre {
namespace {

constexpr int kWarps = 4, kTile = 16;

template <class T> struct Mma;
template <> struct Mma<__nv_bfloat16> {
  static __device__ __forceinline__ void run(float* d, const uint32_t* a, uint32_t b0,
                                             uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <> struct Mma<__half> {
  static __device__ __forceinline__ void run(float* d, const uint32_t* a, uint32_t b0,
                                             uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

template <int N> __device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <Code CODE, int DIM, int NT> struct Shape {
  static constexpr int CB = CODE == Code::kHalf ? 2 : 1;
  static constexpr int ROW = DIM * CB;                  // bytes of one key
  static constexpr int CPR = ROW / 16;                  // 16-byte pieces of one key
  static constexpr int SCALES = CODE == Code::kHalf ? 0 : 2 * kTile * 4;
  static constexpr int STAGE = 2 * kTile * ROW + SCALES + 128;
  static constexpr int ROWS = 8 * NT;
  // about 200 KB of copies in flight an SM, four blocks where registers allow
  static constexpr int BLOCKS_AN_SM = ROW == 256 ? 2 : NT == 1 ? 4 : 3;
  static constexpr int STAGES = ROW == 256 ? 3 : ROW == 128 ? (NT == 1 ? 3 : 4) : (NT == 1 ? 5 : 7);
  static constexpr int SMEM_RING = kWarps * STAGES * STAGE;
  static constexpr int SMEM_JOIN = kWarps * ROWS * (DIM + 4) * 4;
  static constexpr int SMEM = SMEM_RING > SMEM_JOIN ? SMEM_RING : SMEM_JOIN;
  // Place of 16-byte piece u = token * CPR + piece: eight neighbours of a read
  // (two tokens x four pieces of keys, four even or odd tokens x two pieces of
  // values) fall on different banks.
  static __device__ __forceinline__ int place(int tok, int piece) {
    const int u = tok * CPR + piece;
    if constexpr (CPR == 4) return u ^ (((tok >> 1) & 3) << 1);
    return u ^ ((((tok >> 1) & 3) << 1) ^ ((tok & 1) << 2));
  }
};

// An 8 x 8 tile of 16-bit elements turned within the warp.
__device__ __forceinline__ uint32_t turned(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <class T, Code CODE, int DIM, int NT>
__device__ __forceinline__ void attend_block(const AttendArgs& a, const BatchArgs& b,
                                             const CacheArgs& c) {
  using S = Shape<CODE, DIM, NT>;
  using CT = typename std::conditional<CODE == Code::kHalf, T, __half>::type;
  constexpr int EPT = 16 / S::CB, SPB = EPT / 4, BLOCKS = DIM / (4 * EPT);
  // Weights are rounded to 16 bits for their product with values, over codes and float16 to
  // halves of 11 significant bits. In bfloat16 that is 8, as coarse as the output's own
  // rounding (2.5e-3 off for 2 requests of up to 700, 1.7e-3 rounded once): what it leaves
  // over is multiplied as well. That took 1% on long contexts, 5 to 17% where sequences
  // have 16 to 64 rows.
  constexpr bool SPLIT = CODE == Code::kHalf && std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ float w_m[kWarps][S::ROWS], w_l[kWarps][S::ROWS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, cc = lane & 3;
  const int kvh = blockIdx.x % c.heads;
  int rest = blockIdx.x / c.heads;
  const int sp = rest % a.parts;
  rest /= a.parts;
  const int rt0 = rest % a.row_tiles, i = rest / a.row_tiles;
  if (blockIdx.x == 0) loose_rows<T, DIM>(a, b);
  const Seq sq = seq_of(b, i);
  const int rows = sq.n * a.group, base = sq.ctx - sq.n;
  if (rows > a.few) return;
  for (int rt = rt0; rt * S::ROWS < rows; rt += a.row_tiles) {
    const int r_first = rt * S::ROWS, r_last = min(r_first + S::ROWS, rows) - 1;
    const int t_first = a.by_group.div(r_first), t_last = a.by_group.div(r_last);
    int lo, hi;
    range_of<kTile>(sq, c, b, a.window, t_first, t_last, lo, hi);
    part_of<kTile * kWarps>(a, sp, lo, hi);
    const int n_tiles = hi > lo ? (hi - lo + kTile - 1) / kTile : 0;
    const int mine = n_tiles > warp ? (n_tiles - warp + kWarps - 1) / kWarps : 0;

    const Edges edge = edges_of<kTile>(a.window, base + t_first, base + t_last, lo, hi);
    bool left_out = false;           // values of theirs (see finite)
    uint8_t* ring = sm + warp * (S::STAGES * S::STAGE);
    const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
    // the page of token (lane & 15) of the next tile to copy
    int next_tile = 0, page = -1, slot = 0;
    auto look = [&]() {
      const int j = lo + (warp + next_tile * kWarps) * kTile + (lane & 15);
      page = next_tile < mine && j < hi ? page_of(c, b, i, j, slot) : -1;
    };
    auto issue = [&]() {
      if (next_tile < mine) {
        const int st = next_tile % S::STAGES;
        const uint32_t dst = ring_s + st * S::STAGE;
        const bool there = page >= 0;
        const int64_t off =
            there ? (page * c.s_page + slot * c.s_token + kvh * c.s_head) * S::CB : 0;
        const unsigned held = __ballot_sync(0xffffffffu, there);
#pragma unroll
        for (int it = 0; it < S::CPR / 2; ++it) {
          const int u = it * 32 + lane, tok = u / S::CPR, piece = u % S::CPR;
          const int64_t o = __shfl_sync(0xffffffffu, off, tok) + piece * 16;
          const int n = held >> tok & 1 ? 16 : 0;
          const uint32_t at = dst + S::place(tok, piece) * 16;
          const uint8_t *pk = n ? c.k + o : c.k, *pv = n ? c.v + o : c.v;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(pk), "r"(n)
                       : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + kTile * S::ROW),
                       "l"(pv), "r"(n)
                       : "memory");
        }
        if (S::SCALES) {
          const float* sc = lane < 16 ? c.k_scale : c.v_scale;
          const float* p = there ? sc + page * c.c_page + slot * c.c_token + kvh * c.c_head : sc;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 2 * kTile * S::ROW +
                                                                            lane * 4),
                       "l"(p), "r"(there ? 4 : 0)
                       : "memory");
        }
        if (lane == 0)
          *reinterpret_cast<uint32_t*>(ring + st * S::STAGE + 2 * kTile * S::ROW + S::SCALES) = held;
        ++next_tile;
        look();
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };

    look();
#pragma unroll 1
    for (int k = 0; k < S::STAGES - 1; ++k) issue();

    // queries: row g of each eight, in the order of a key's reads
    uint32_t qf[NT][DIM / 16][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = r_first + 8 * nt + g, t = a.by_group.div(r);
      const T* qp = reinterpret_cast<const T*>(a.q) + (int64_t)(sq.start + t) * a.q_row +
                    (int64_t)(kvh * a.group + (r - t * a.group)) * a.q_head;
#pragma unroll
      for (int s = 0; s < DIM / 16; ++s) {
        uint2 v = make_uint2(0, 0);
        if (r < rows) v = *reinterpret_cast<const uint2*>(qp + (s / SPB * 4 + cc) * EPT + (s % SPB) * 4);
        qf[nt][s][0] = v.x;
        qf[nt][s][1] = v.y;
      }
    }
    // The rows whose weights this lane holds: 2 cc and 2 cc + 1 of each eight.
    // Codes are multiplied as halves, which both kinds turn into in a step or two;
    // bfloat16 queries then go as halves too, each row divided by a power of two
    // (its largest element's) that its scores get back: what is below 2^-24 of that is
    // cut.
    int pos[NT][2];
    float back[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        pos[nt][x] = base + a.by_group.div(min(r_first + 8 * nt + 2 * cc + x, rows - 1));
        back[nt][x] = a.scale2;
      }
      if constexpr (!std::is_same<T, CT>::value) {
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float u, v;
            unpack(qf[nt][s][y], u, v, T());
            top = fmaxf(top, fmaxf(fabsf(u), fabsf(v)));
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ex = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
        const float f = __uint_as_float((uint32_t)ex << 23) * a.scale2;
        const float by = __uint_as_float((uint32_t)(254 - ex) << 23);
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float u, v;
            unpack(qf[nt][s][y], u, v, T());
            qf[nt][s][y] = pack<CT>(u * by, v * by);
          }
#pragma unroll
        for (int x = 0; x < 2; ++x)          // (row r's factor is in lanes 4 r ..)
          back[nt][x] = __shfl_sync(0xffffffffu, f, 4 * (2 * cc + x));
      }
    }

    float o[NT][DIM / 16][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int n = 0; n < DIM / 16; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][n][e] = 0.f;
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        m[nt][x] = -INFINITY;
        l[nt][x] = 0.f;
      }

#pragma unroll 1
    for (int k = 0; k < mine; ++k) {
      wait_copies<S::STAGES - 2>();
      __syncwarp();
      uint8_t* st = ring + (k % S::STAGES) * S::STAGE;
      const uint4* kt = reinterpret_cast<const uint4*>(st);
      uint4* vt = reinterpret_cast<uint4*>(st + kTile * S::ROW);
      const int j0 = lo + (warp + k * kWarps) * kTile;
      if (CODE != Code::kI8 && (j0 < edge.behind || j0 >= edge.ahead)) {
        for (int u = lane; u < kTile * S::CPR; u += 32) {
          const uint4 x = vt[u], y = finite<T, CODE>(x);
          if (differ(x, y)) {
            vt[u] = y;
            left_out = true;
          }
        }
        __syncwarp();
      }
      const float* sc = reinterpret_cast<const float*>(st + 2 * kTile * S::ROW);
      const uint32_t held =
          *reinterpret_cast<const uint32_t*>(st + 2 * kTile * S::ROW + S::SCALES) & 0xffffu;
      float s[NT][4];                // positions g, g + 8 by rows 2 cc, 2 cc + 1
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
      for (int bl = 0; bl < BLOCKS; ++bl) {
        const uint4 u = kt[S::place(g, 4 * bl + cc)], v = kt[S::place(g + 8, 4 * bl + cc)];
        if constexpr (CODE == Code::kHalf) {
          const uint32_t f0[4] = {u.x, v.x, u.y, v.y}, f1[4] = {u.z, v.z, u.w, v.w};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            Mma<CT>::run(s[nt], f0, qf[nt][2 * bl][0], qf[nt][2 * bl][1]);
            Mma<CT>::run(s[nt], f1, qf[nt][2 * bl + 1][0], qf[nt][2 * bl + 1][1]);
          }
        } else {
          const uint32_t wu[4] = {u.x, u.y, u.z, u.w}, wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t f[4] = {halves<CODE>(wu[x]), halves<CODE>(wv[x]),
                                   halves<CODE>(wu[x] >> 16), halves<CODE>(wv[x] >> 16)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              Mma<CT>::run(s[nt], f, qf[nt][4 * bl + x][0], qf[nt][4 * bl + x][1]);
          }
        }
      }

      float vs[2] = {1.f, 1.f}, ex[2] = {0.f, 0.f}, ks[2] = {1.f, 1.f};
      if constexpr (S::SCALES > 0) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          ks[y] = sc[g + 8 * y];
          vs[y] = sc[kTile + g + 8 * y];
          ex[y] = weight_exponent(vs[y]);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[nt][e] *= back[nt][e & 1];
          if (S::SCALES) s[nt][e] *= ks[e >> 1];
        }
      const bool whole = held == 0xffffu && j0 + kTile - 1 <= base + t_first &&
                         (a.window == 0 || j0 > base + t_last - a.window);
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = g + 8 * (e >> 1), j = j0 + tok;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int p = pos[nt][e & 1];
            const bool vis = (held >> tok & 1) && j <= p && (a.window == 0 || j > p - a.window);
            if (!vis) s[nt][e] = -INFINITY;
          }
        }
      }
      // The maximum moves when some weight would pass 2^8 (first of all from nothing);
      // until then no lane needs another's scores.
      bool past = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = s[nt][e] + ex[e >> 1];
          past |= t > m[nt][e & 1] + 8.f;
        }
      if (__any_sync(0xffffffffu, past)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float t = fmaxf(s[nt][x] + ex[0], s[nt][x + 2] + ex[1]);
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
            const float mn = fmaxf(m[nt][x], t);
            const float f = m[nt][x] == -INFINITY ? 0.f : exp2_fast(m[nt][x] - mn);
            m[nt][x] = mn;
            l[nt][x] *= f;
#pragma unroll
            for (int n = 0; n < DIM / 16; ++n) {
              o[nt][n][x] *= f;
              o[nt][n][x + 2] *= f;
            }
          }
      }
      // rows g by positions 2 cc, 2 cc + 1 (+ 8); with SPLIT also what a weight's rounding
      // left over
      uint32_t pf[NT][2], rest[SPLIT ? NT : 1][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float use = m[nt][e & 1] == -INFINITY ? 0.f : m[nt][e & 1];
          p[e] = exp2_fast(s[nt][e] - use);
          l[nt][e & 1] += p[e];
          // (a masked position's scale may be anything: its weight stays zero)
          if (S::SCALES) p[e] = p[e] == 0.f ? 0.f : p[e] * vs[e >> 1];
        }
        if constexpr (SPLIT) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            // the largest bfloat16 below a weight, so that what is left over is above zero
            // and a value that is infinite stays so in both products
            uint32_t b0 = __float_as_uint(p[2 * y]), b1 = __float_as_uint(p[2 * y + 1]);
            b0 -= min(b0, 1u);
            b1 -= min(b1, 1u);
            pf[nt][y] = turned(__byte_perm(b0, b1, 0x7632));
            rest[nt][y] = turned(pack<CT>(p[2 * y] - __uint_as_float(b0 & 0xffff0000u),
                                          p[2 * y + 1] - __uint_as_float(b1 & 0xffff0000u)));
          }
        } else {
          pf[nt][0] = turned(pack<CT>(p[0], p[1]));
          pf[nt][1] = turned(pack<CT>(p[2], p[3]));
        }
      }
      // values: an m-tile's rows g and g + 8 are neighbouring elements, as a lane's
      // read delivers them
      if constexpr (CODE == Code::kHalf) {
#pragma unroll
        for (int set = 0; set < DIM / 64; ++set) {
          uint4 v[4];
#pragma unroll
          for (int x = 0; x < 4; ++x)
            v[x] = vt[S::place(2 * cc + (x & 1) + (x >> 1) * 8, 8 * set + g)];
          const uint32_t w[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w},
                                    {v[1].x, v[1].y, v[1].z, v[1].w},
                                    {v[2].x, v[2].y, v[2].z, v[2].w},
                                    {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const uint32_t f[4] = {__byte_perm(w[0][y], w[1][y], 0x5410),
                                   __byte_perm(w[0][y], w[1][y], 0x7632),
                                   __byte_perm(w[2][y], w[3][y], 0x5410),
                                   __byte_perm(w[2][y], w[3][y], 0x7632)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              Mma<CT>::run(o[nt][set * 4 + y], f, pf[nt][0], pf[nt][1]);
              if constexpr (SPLIT) Mma<CT>::run(o[nt][set * 4 + y], f, rest[nt][0], rest[nt][1]);
            }
          }
        }
      } else {
        constexpr int W = DIM / 32;       // words of codes a lane reads of a token
        uint32_t w[4][W];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int tok = 2 * cc + (x & 1) + (x >> 1) * 8;
          if constexpr (W == 4) {
            const uint4 v = vt[S::place(tok, g)];
            w[x][0] = v.x;
            w[x][1] = v.y;
            w[x][2] = v.z;
            w[x][3] = v.w;
          } else {
            const uint2 v = reinterpret_cast<const uint2*>(vt + S::place(tok, g >> 1))[g & 1];
            w[x][0] = v.x;
            w[x][1] = v.y;
          }
        }
#pragma unroll
        for (int y = 0; y < W; ++y)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const uint32_t sel = hf ? 0x7362 : 0x5140;
            const uint32_t u = __byte_perm(w[0][y], w[1][y], sel);
            const uint32_t z = __byte_perm(w[2][y], w[3][y], sel);
            const uint32_t f[4] = {halves<CODE>(u), halves<CODE>(u >> 16),
                                   halves<CODE>(z), halves<CODE>(z >> 16)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) Mma<CT>::run(o[nt][2 * y + hf], f, pf[nt][0], pf[nt][1]);
          }
      }
      __syncwarp();
      issue();
    }
    wait_copies<0>();

    // join the four warps
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float sum = l[nt][x];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (g == 0) {
          w_m[warp][8 * nt + 2 * cc + x] = m[nt][x];
          w_l[warp][8 * nt + 2 * cc + x] = sum;
        }
      }
    left_out = __syncthreads_or(left_out);
    constexpr int PITCH = DIM + 4;
    float* os = reinterpret_cast<float*>(sm);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = 8 * nt + 2 * cc + x;
        float top = w_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, w_m[w][r]);
        const float f = m[nt][x] == -INFINITY ? 0.f : exp2_fast(m[nt][x] - top);
        float* dst = os + (warp * S::ROWS + r) * PITCH;
#pragma unroll
        for (int n = 0; n < DIM / 16; ++n) {
          // elements of m-tile n that this lane holds: see the reads above
          int d;
          if constexpr (CODE == Code::kHalf) d = (n / 4) * 64 + 8 * g + 2 * (n % 4);
          else d = (DIM / 8) * g + 2 * n;
          // a warp that saw nothing has nothing to add, whatever it multiplied
          *reinterpret_cast<float2*>(dst + d) =
              f == 0.f ? make_float2(0.f, 0.f)
                       : make_float2(o[nt][n][x] * f, o[nt][n][x + 2] * f);
        }
      }
    __syncthreads();
    constexpr int LPR = 32, EL = DIM / LPR;
    for (int r = warp; r < S::ROWS; r += kWarps) {
      const int rr = r_first + r;
      if (rr >= rows) break;
      float top = w_m[0][r];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, w_m[w][r]);
      float sum = 0.f, x[EL];
#pragma unroll
      for (int e = 0; e < EL; ++e) x[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = w_m[w][r] == -INFINITY ? 0.f : exp2_fast(w_m[w][r] - top);
        sum = __fmaf_rn(w_l[w][r], f, sum);
#pragma unroll
        for (int e = 0; e < EL; ++e) x[e] += os[(w * S::ROWS + r) * PITCH + lane * EL + e];
      }
      const int t = a.by_group.div(rr), h = kvh * a.group + (rr - t * a.group);
      const int64_t row = (int64_t)(sq.start + t);
      if (CODE != Code::kI8 && left_out && top > -INFINITY)
        add_seen<T, CODE, DIM>(b, c, a.window, i, kvh, base + t, lo, edge, hi, x);
      const int64_t part_row = a.tokens > 0 ? (int64_t)i * a.tokens + t : row;
      if (lane == 0) row_state(a, sp, row, part_row, h, top, sum);
      if (a.parts > 1) {
        const int64_t at = (sp * a.part_rows + part_row) * a.heads + h;
        float* p = a.part_o + at * DIM + lane * EL;
        if (sum > 0.f || sum != sum) {
          if constexpr (EL == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
          else *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
        }
      } else {
        const float by = saw_nothing(top, sum) ? 0.f : div_rn(1.f, sum);
        T* p = reinterpret_cast<T*>(a.out) + row * a.o_row + (int64_t)h * a.o_head + lane * EL;
#pragma unroll
        for (int e = 0; e < EL; e += 2)
          *reinterpret_cast<uint32_t*>(p + e) = pack<T>(x[e] * by, x[e + 1] * by);
      }
    }
    __syncthreads();
  }
}

// Beside k_attend_tc: this launch does not wait for that one, so that its blocks run on
// SMs that are left over. Neither reads what the other writes (rows of different
// sequences, and the marks of those in the other's part_ml); the last block stays until
// the other launch is done, so that what comes next in the stream waits for both.
template <class T, Code CODE, int DIM, int NT>
__global__ void __launch_bounds__(kWarps * 32, Shape<CODE, DIM, NT>::BLOCKS_AN_SM)
k_attend(AttendArgs a, BatchArgs b, CacheArgs c) {
  attend_block<T, CODE, DIM, NT>(a, b, c);
  if (a.beside && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Joins the parts of each row, W warps a (row, head), the parts dealt out among them: all
// eight warps from 16 parts on (few rows then), one below (many). Parts are taken in their
// order. A few us: latency, and the partial sums come from L2.
constexpr int kJoinWarps = 8;
struct JoinSets {
  AttendArgs of[2];
};
template <class T, int DIM, int W>
__device__ __forceinline__ void join_rows(const AttendArgs& a, const BatchArgs& b, int parts) {
  constexpr int EL = DIM / 32, HEADS = kJoinWarps / W;       // heads of a block's turn
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp % W;
  {
    const int per_row = (a.heads + HEADS - 1) / HEADS;
    for (int64_t turn = blockIdx.x; turn < a.part_rows * per_row; turn += gridDim.x) {
      const int64_t row = turn / per_row;
      const int h = (int)(turn - row * per_row) * HEADS + warp / W;
      int64_t t = row;
      if (a.tokens > 0) {
        const int i = (int)(row / a.tokens), r = (int)(row - (int64_t)i * a.tokens);
        const Seq s = seq_of(b, i);
        if (r >= s.n || s.n * a.group > a.few) continue;
        t = s.start + r;
      }
      const int64_t w = row * a.heads + h, all = a.part_rows * a.heads;
      const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
      float top = -INFINITY, first = 0.f;
      bool go = h < a.heads;
      if (go) {
        for (int sp = lane; sp < parts; sp += 32) {
          const float2 v = ml[sp * all + w];
          if (sp == 0) first = v.y;
          top = fmaxf(top, v.x);
        }
      }
      go = go && !(__shfl_sync(0xffffffffu, first, 0) < 0.f);         // not this join's
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float sum = 0.f, x[EL];
#pragma unroll
      for (int e = 0; e < EL; ++e) x[e] = 0.f;
      if (go) {
#pragma unroll 4
        for (int sp = mine; sp < parts; sp += W) {
          const int64_t at = sp * all + w;
          const float2 v = ml[at];
          const float f = v.x == -INFINITY ? 0.f : exp2_fast(v.x - top);
          sum = __fmaf_rn(v.y, f, sum);
          if (f == 0.f) continue;            // (nothing was left there)
          const float* p = a.part_o + at * DIM + lane * EL;
          float y[EL];
          if constexpr (EL == 4) {
            const float4 u = *reinterpret_cast<const float4*>(p);
            y[0] = u.x; y[1] = u.y; y[2] = u.z; y[3] = u.w;
          } else {
            const float2 u = *reinterpret_cast<const float2*>(p);
            y[0] = u.x; y[1] = u.y;
          }
#pragma unroll
          for (int e = 0; e < EL; ++e) x[e] = __fmaf_rn(y[e], f, x[e]);
        }
      }
      if constexpr (W > 1) {
        __shared__ float part[kJoinWarps][DIM + 1];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < EL; ++e) part[warp][lane * EL + e] = x[e];
        if (lane == 0) part[warp][DIM] = sum;
        __syncthreads();
        go = go && mine == 0;
        if (go) {
#pragma unroll
          for (int y = 1; y < W; ++y) {
            sum += part[warp + y][DIM];
#pragma unroll
            for (int e = 0; e < EL; ++e) x[e] += part[warp + y][lane * EL + e];
          }
        }
      }
      if (!go) continue;
      const float by = saw_nothing(top, sum) ? 0.f : div_rn(1.f, sum);
      T* p = reinterpret_cast<T*>(a.out) + t * a.o_row + (int64_t)h * a.o_head + lane * EL;
#pragma unroll
      for (int e = 0; e < EL; e += 2)
        *reinterpret_cast<uint32_t*>(p + e) = pack<T>(x[e] * by, x[e + 1] * by);
      if (a.lse && lane == 0)
        a.lse[t * a.heads + h] = saw_nothing(top, sum) ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
  }
}

// Both kernels' parts in one launch. From 16 parts on a block's eight warps share a row:
// a warp alone reads them one after another.
template <class T, int DIM>
__global__ void __launch_bounds__(kJoinWarps * 32, 4)
k_join(const __grid_constant__ JoinSets sets, BatchArgs b) {
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const AttendArgs& a = sets.of[k];
    const int parts = a.parts_taken ? *a.parts_taken : a.parts;
    if (parts >= 16) join_rows<T, DIM, kJoinWarps>(a, b, parts);
    else if (parts > 1) join_rows<T, DIM, 1>(a, b, parts);   // (else rows are written already)
  }
}

template <class T, Code CODE, int DIM, int NT>
cudaError_t launch_typed(const AttendArgs& a, const BatchArgs& b, const CacheArgs& c,
                         cudaStream_t s) {
  using S = Shape<CODE, DIM, NT>;
  const void* fn = (const void*)k_attend<T, CODE, DIM, NT>;
  cudaError_t e = func_smem_once(fn, S::SMEM, true);
  if (e) return e;
  const int64_t blocks = (int64_t)c.heads * a.parts * a.row_tiles * b.n_seq;
  if (blocks > 2147483647) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = a.beside ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_attend<T, CODE, DIM, NT>, a, b, c);
}

template <class T, Code CODE, int DIM>
cudaError_t launch_rows(int nt, const AttendArgs& a, const BatchArgs& b, const CacheArgs& c,
                        cudaStream_t s) {
  return nt == 1 ? launch_typed<T, CODE, DIM, 1>(a, b, c, s) : launch_typed<T, CODE, DIM, 2>(a, b, c, s);
}

template <class T>
cudaError_t launch_code(int code, int dim, int nt, const AttendArgs& a, const BatchArgs& b,
                        const CacheArgs& c, cudaStream_t s) {
  if (code == TRE_E4M3)
    return dim == 64 ? launch_rows<T, Code::kE4m3, 64>(nt, a, b, c, s)
                     : launch_rows<T, Code::kE4m3, 128>(nt, a, b, c, s);
  if (code == TRE_I8)
    return dim == 64 ? launch_rows<T, Code::kI8, 64>(nt, a, b, c, s)
                     : launch_rows<T, Code::kI8, 128>(nt, a, b, c, s);
  return dim == 64 ? launch_rows<T, Code::kHalf, 64>(nt, a, b, c, s)
                   : launch_rows<T, Code::kHalf, 128>(nt, a, b, c, s);
}

template <class T, int DIM>
cudaError_t launch_join(const JoinSets& sets, const BatchArgs& b, cudaStream_t s) {
  int64_t turns = 0;
  for (const AttendArgs& a : sets.of) {
    const int64_t heads = a.parts >= 16 ? 1 : kJoinWarps;
    if (a.parts > 1) turns = std::max(turns, a.part_rows * ((a.heads + heads - 1) / heads));
  }
  const unsigned blocks = (unsigned)std::min<int64_t>(turns, (int64_t)device_sm_count() * 64);
  k_join<T, DIM><<<blocks, kJoinWarps * 32, 0, s>>>(sets, b);
  return cudaGetLastError();
}

cudaError_t join(int dtype, int dim, const JoinSets& sets, const BatchArgs& b, cudaStream_t s) {
  if (sets.of[0].parts < 2 && sets.of[1].parts < 2) return cudaSuccess;
  if (dtype == TRE_BF16)
    return dim == 64 ? launch_join<__nv_bfloat16, 64>(sets, b, s)
                     : launch_join<__nv_bfloat16, 128>(sets, b, s);
  return dim == 64 ? launch_join<__half, 64>(sets, b, s) : launch_join<__half, 128>(sets, b, s);
}

// How a call is split, from what the host knows of it.
struct Plan {
  bool tc;                        // some sequence may have more than `few` rows
  int32_t few, tokens;            // (see AttendArgs)
  int32_t parts[2], split[2];     // k_attend, k_attend_tc
  int64_t part_rows[2];
  int32_t row_tiles, nt;          // of k_attend: tiles of 8 * nt rows
  int64_t units;                  // of k_attend_tc, at most
  bool shared;                    // its blocks take units as they get to them
};

// Which kernel takes a sequence, by its rows. k_attend reads keys and values once for 8 or
// 16 rows (again from L2 for the next), k_attend_tc takes 128 rows in the time of one:
// Batches of up to 64 rows a sequence are k_attend's alone: with 32, 48 and 64 rows each
// (bf16, k_attend against k_attend_tc) 4 sequences of 6,000 to 12,000 tokens, dim 128, took 38,
// 58 and 60 us against 70 to 74; 64 of 500 to 2,000, dim 64, 50, 60 and 72 against 81 to 99; 100
// of up to 1,000, dim 128, 42, 47 and 52 against 54 to 58; 4 of 25,000 over e4m3 72, - and 112
// against 175. Only 32 of 1,500 to 4,000, dim 128, were the other way from 48 rows on (90, 115
// and 139 against 112 to 100). Where k_attend_tc runs in any case, sequences of more than 16
// rows are its (at up to 64 in k_attend chunks of up to 128 rows took 250 us, all of them in
// k_attend_tc 107), except one new token's heads.
constexpr int kFew = 64, kFewBeside = 16;

Plan plan_of(const tre_kv_batch* b, const AttendArgs& a, int heads, int page, int dim, bool coded) {
  Plan p{};
  const int64_t max_new = std::max(1, b->max_new > 0 ? b->max_new : b->n_rows);
  const int64_t rows = max_new * a.group;
  int64_t len = b->max_ctx > 0 ? b->max_ctx : (int64_t)b->max_pages * page;
  if (a.window > 0) len = std::min<int64_t>(len, (int64_t)a.window + max_new + 15);
  len = std::max<int64_t>(len, 1);
  const int64_t sms = device_sm_count();
  p.tc = rows > kFew;
  p.few = !p.tc ? 2147483647 : a.group <= kFew ? std::max(kFewBeside, a.group) : kFewBeside;
  {
    // Parts of a context: about 16 blocks an SM, so that sequences of unequal length
    // even out (8 blocks an SM took 3 to 14% longer on ragged batches, 48 up to 9%), of
    // 1,024 tokens at least (parts of 256 cost 10% on short contexts) unless there are
    // then fewer than two blocks an SM, where parts go down to 256.
    // Tiles of 8 rows where one new token's heads (or all rows there are) fit in one (16
    // took 235 for 205 us over e4m3, 8 requests of up to 120,000, and 308 for 300 over
    // bf16), else of 16, which read keys and values once for twice the rows (82 us with
    // 8, 72 with 16 for 16 rows of 32 sequences of 1,500 to 4,000, 167 and 124 for 64 rows;
    // both before bfloat16 weights were multiplied in two halves, now 75 and 139).
    p.nt = (p.tc ? a.group : rows) <= 8 ? 1 : 2;
    p.row_tiles = p.tc ? 1 : (int)std::min<int64_t>((rows + 8 * p.nt - 1) / (8 * p.nt), 1 << 20);
    const int64_t units = std::max<int64_t>(1, (int64_t)b->n_seq * heads * p.row_tiles);
    const int64_t want = (sms * 16 + units - 1) / units, few = (sms * 2 + units - 1) / units;
    const int64_t most = std::max(len / 1024, std::min(few, len / 256));
    p.parts[0] = (int)std::max<int64_t>(1, std::min<int64_t>({want, most, 256}));
    p.split[0] = (int)std::max<int64_t>(kTile * kWarps, (len + p.parts[0] - 1) / p.parts[0]);
  }
  p.tokens = p.tc ? std::max(1, p.few / a.group) : 0;
  p.part_rows[0] = p.tc ? (int64_t)b->n_seq * p.tokens : b->n_rows;
  p.part_rows[1] = b->n_rows;
  p.parts[1] = 1;
  if (p.tc) {
    // Parts are worth their join where there are fewer units than half the SMs (64, 256 and
    // 512 new tokens after 32,000, 32 heads on 8 of 128: 80, 135 and 209 us, whole contexts
    // 342 to 350), two to six rounds of long ones (a part then evens out the last round), or
    // by the lengths known here a tenth less time
    // (1,280 and 1,536 tokens: 521 and 548 us, 666 and 675 whole; where it is less than
    // that, the join's launch took 3 to 7% more). Long: 2,500 to 7,200 tokens after 32,000 in
    // bf16 took 9% less to 2% more in parts (4,096: 1,422 us, 1,458 whole), after 24,000 6% less
    // to 4% more, after 16,000 1% less to 5% more, after 8,000 1 to 14% more; over codes, whose
    // tiles take longer, 3,000 and 5,000 after 16,000 2 to 8% less, after 8,000 1% less to 2%
    // more, after 4,000 1 to 4% more. As many as 256 MB of partial sums allow,
    // none shorter than 512 tokens; how many are taken is seen on the device, where all
    // lengths are known.
    const int64_t all = (int64_t)b->n_rows * a.group;
    const int64_t tiles = std::min<int64_t>(
        (int64_t)b->n_seq * ((rows + kTcRows - 1) / kTcRows), all / kTcRows + b->n_seq);
    const int64_t row = ((int64_t)dim * 4 + 8) * a.heads * std::max(b->n_rows, 1);
    const int64_t least = std::max<int64_t>(all - (int64_t)b->n_seq * p.few, 1) / kTcRows * heads;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>({64, len / 512, (256ll << 20) / row}));
    bool worth = 2 * least <= sms || (least >= 2 * sms && least <= 6 * sms && len >= (coded ? 12288 : 30000));
    if (!worth && least < 2 * sms)
      for (int64_t n = 2; n <= most; ++n)
        worth |= parts_time(n, tiles * heads, len, sms) <
                 0.9f * parts_time(1, tiles * heads, len, sms);
    if (worth) p.parts[1] = (int)most;
    p.split[1] = (int)std::max<int64_t>(kTcTokens, (len + p.parts[1] - 1) / p.parts[1]);
    p.units = std::max<int64_t>(1, tiles * heads) * p.parts[1];
    // Ragged sequences: units in turn leave some blocks a fifth more than the mean; a count
    // that blocks take from evens that out for a 4-byte clear before the launch. 24 prompts of
    // up to 2,000, 16 heads of 64, 131 -> 125 us; 24 chunks of up to 2,000 after up to 3,000,
    // 8 heads, 178 -> 149; 32 of up to 1,000, 32 on 8 heads of 128, 397 -> 371; eight of up to
    // 4,000 between 2% more and 12% less. One sequence's units are even in turn (1,392 us,
    // 1,402 so), and with fewer units than SMs there is nothing to take.
    p.shared = b->n_seq > 1 && least > sms;
  }
  return p;
}

cudaError_t launch_all(int dtype, int code, int dim, AttendArgs a, const Plan& p,
                       float* const* part_o, float* const* part_ml, int32_t* parts_taken, uint32_t* next,
                       const BatchArgs& b, const CacheArgs& c, tre_diag* diag, cudaStream_t s) {
  const bool bf = dtype == TRE_BF16;
  a.few = p.few;
  auto of = [&](int k) {
    AttendArgs x = a;
    x.parts = p.parts[k];
    x.split = p.split[k];
    x.part_o = part_o[k];
    x.part_ml = part_ml[k];
    x.part_rows = p.part_rows[k];
    return x;
  };
  cudaError_t e = cudaSuccess;
  AttendArgs y = of(1);
  y.parts_taken = parts_taken;
  y.sms = device_sm_count();
  y.next = next;
  if (p.tc) {
    if (next) e = cudaMemsetAsync(next, 0, sizeof(*next), s);
    if (e) return e;
    e = launch_attend_tc(dtype, code, dim, y, b, c, p.units, diag, s);
    if (e) return e;
  }
  AttendArgs x = of(0);
  x.row_tiles = p.row_tiles;
  x.tokens = p.tokens;
  x.beside = p.tc;
  if (p.parts[1] > 1) x.done = reinterpret_cast<float2*>(part_ml[1]);
  e = bf ? launch_code<__nv_bfloat16>(code, dim, p.nt, x, b, c, s)
         : launch_code<__half>(code, dim, p.nt, x, b, c, s);
  if (!e) e = join(dtype, dim, JoinSets{{x, y}}, b, s);
  return e;
}

}  // namespace
}  // namespace tre

using namespace tre;

extern "C" tre_status tre_chunk_attention(const tre_kv_cache* cache, const tre_kv_batch* batch,
                                          const tre_attend* at, void* ws, size_t* ws_bytes,
                                          tre_diag* diag, tre_stream stream) {
  AttendArgs a{};
  BatchArgs b;
  CacheArgs c;
  if (!at || !ws_bytes || !batch_args(batch, b) || !cache_args(cache, c)) return TRE_EINVAL;
  if (at->dtype != TRE_BF16 && at->dtype != TRE_F16) return TRE_EINVAL;
  if (cache->dtype != at->dtype && cache->dtype != TRE_E4M3 && cache->dtype != TRE_I8)
    return TRE_EINVAL;
  if (at->heads < 1 || at->heads % cache->heads || at->heads > 65536 || at->window < 0)
    return TRE_EINVAL;
  if (!(at->scale > 0.f) || !(at->scale < 3e38f)) return TRE_EINVAL;
  const int64_t strides[4] = {at->q_row, at->q_head, at->out_row, at->out_head};
  for (int64_t x : strides)
    if (x % 8 || x < 0 || x > 2147483647) return TRE_EINVAL;
  if (((uintptr_t)at->q & 15) || ((uintptr_t)at->out & 15)) return TRE_EINVAL;
  a.heads = at->heads;
  a.group = at->heads / cache->heads;
  if (b.n_rows > 0 && (int64_t)b.n_rows * a.group > 2147483647ll / 2) return TRE_EINVAL;
  a.by_group = FastDiv31((uint32_t)a.group);
  a.window = at->window;
  Plan plan{};
  if (b.n_seq > 0) plan = plan_of(batch, a, c.heads, c.page, cache->dim, cache->dtype != at->dtype);
  Arena arena(ws);
  float *part_o[2] = {}, *part_ml[2] = {};
  int32_t* parts_taken = plan.parts[1] > 1 ? arena.take<int32_t>(1) : nullptr;
  uint32_t* next = plan.shared ? arena.take<uint32_t>(1) : nullptr;
  for (int k = 0; k < 2; ++k) {
    if (plan.parts[k] < 2) continue;
    const size_t rh = (size_t)plan.part_rows[k] * a.heads * plan.parts[k];
    part_ml[k] = arena.take<float>(2 * rh);
    part_o[k] = arena.take<float>(rh * cache->dim);
  }
  if (!ws) {
    *ws_bytes = arena.off;
    return TRE_OK;
  }
  if (*ws_bytes < arena.off) return TRE_ENOMEM;
  if (b.n_rows == 0) return TRE_OK;
  if (b.n_seq == 0 || !at->q || !at->out) return TRE_EINVAL;
  a.q = static_cast<const uint8_t*>(at->q);
  if (c.n_pages == 0) {                  // nothing will be read, but copies name an address
    c.k = c.v = const_cast<uint8_t*>(a.q);
    c.k_scale = c.v_scale = reinterpret_cast<float*>(c.k);
  }
  a.out = static_cast<uint8_t*>(at->out);
  a.lse = at->lse;
  a.q_row = (int32_t)at->q_row;
  a.q_head = (int32_t)at->q_head;
  a.o_row = (int32_t)at->out_row;
  a.o_head = (int32_t)at->out_head;
  a.wide = ((uintptr_t)at->out & 31) == 0 && at->out_row % 16 == 0 && at->out_head % 16 == 0;
  a.scale2 = (float)((double)at->scale * 1.4426950408889634);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      launch_all(at->dtype, cache->dtype, cache->dim, a, plan, part_o, part_ml, parts_taken, next,
                 b, c,
                 diag, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}
