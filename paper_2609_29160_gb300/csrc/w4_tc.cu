// Products with matrices in 4 bits of many rows, on the tensor cores with their
// accumulators in tensor memory.
//
//   y[t][n] = sum over groups q of scale[n][q] * sum over k in q of (code[n][k] - zero[n][q]) x[t][k]
//
// The matrix is the product's A operand: a unit is 256 rows of it against up to 256 rows of
// x, for two blocks on neighbouring SMs (cta_group::2), each of which holds 128 rows of the
// matrix and half of the rows of x in shared memory, and in tensor memory its 128 rows of
// the sums. Codes less their zeros are whole numbers that 16 bits hold, so the products
// inside a group are exact and its sum is one accumulator in tensor memory; the scale comes
// when that accumulator is added, in 32 bits, to the sums that the scaling warps keep in
// registers. (Scaling the codes instead would round every element of the matrix to 16 bits.)
//
// A block's warps: 0-7 add groups (a thread a row of the matrix and half of the columns) and
// write rows of y; 8-12 turn codes into the operand, a stage of 128 x 64 elements a warp; 13
// copies rows of x, 14 codes; 15 of the pair's first block issues the products. Of a gated matrix a
// warp of the first eight holds 16 rows of the gate and the 16 that they multiply.
//
// 4,096 x 4,096 x 8,192, bf16, groups of 128: 165 us, 1.66 PFLOP/s; the tensor pipe is busy three
// quarters of the time. A stage takes its products' time with 256 rows of x and groups of 128 (0.36
// us), with fewer rows no less than 0.28 us (0.38 with groups of 64, 0.75 with 32: the round of
// products, adding and products again over two to four accumulators then binds).
#include <algorithm>
#include <cstring>

#include "internal.h"
#include "tensor.cuh"
#include "w4.cuh"

namespace tre {
namespace {

constexpr int kScaleWarps = 8, kCodeWarp = 8, kCodeWarps = 5, kRowWarp = 13, kRawWarp = 14, kMmaWarp = 15;
constexpr int kThreads = 512;
constexpr int kAsk = 12;               // stages of codes that are asked for ahead

// Shared memory of a block for units of up to WIDTH rows of x. A place of the operand is taken
// from the products that free it, through the turning of codes and an arrival at the other
// block, to its next products: some 1.5 us.
template <int WIDTH> struct Ring {
  static constexpr int A = WIDTH == 256 ? 6 : 7, B = WIDTH == 256 ? 6 : 8, RAW = WIDTH == 256 ? 6 : 8;
  static constexpr int BYTES_A = 128 * 128, BYTES_B = WIDTH / 2 * 128, BYTES_RAW = 4096;
  static constexpr int SUMS = 512 / WIDTH;             // accumulators
  static constexpr int AT_B = A * BYTES_A, AT_RAW = AT_B + B * BYTES_B;
  static constexpr int AT_OUT = AT_RAW + RAW * BYTES_RAW, AT_BAR = AT_OUT + kScaleWarps * 1024;
  static constexpr int BARS = 2 * (RAW + B + SUMS);
  static constexpr int SMEM = AT_BAR + BARS * 8 + 16;
  static_assert(SMEM <= 227 * 1024, "shared memory of a block");
};

// A tile of rows of x, the same for both blocks of a pair.
struct Unit {
  int expert, block;                   // block: of 256 rows of the matrix
  int start, count, columns;           // rows of x; to whole 32
};

struct TcArgs {
  ProductArgs p;
  int32_t row_blocks, tile;            // tile: most rows of x of a unit
  int32_t box;                         // rows of x of one copy
};

__device__ __forceinline__ bool unit_at(const TcArgs& a, int u, Unit& w) {
  const int t = u / a.row_blocks;
  w.block = u - t * a.row_blocks;
  if (a.p.plan.order) {
    if (t >= a.p.plan.n[0]) return false;
    const Slot s = a.p.plan.tiles[t];
    w.expert = s.expert;
    w.start = s.start;
    w.count = s.count;
  } else {
    w.expert = 0;
    w.start = t * a.tile;
    w.count = min(a.tile, a.p.n_rows - w.start);
    if (w.count <= 0) return false;
    w.columns = a.tile;                // (whole copies; rows past the last come as zeros)
    return true;
  }
  w.columns = (w.count + 31) & ~31;
  return true;
}

// The same barrier of the pair's first block
__device__ __forceinline__ uint32_t first_of(uint64_t* b) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_of(b)));
  return r;
}
// A warp's arrival at a barrier of the pair's first block. What it announces has been ordered
// already, for the unit that will read it: rows written to shared memory by a proxy fence,
// tensor memory read by a wait. (A release for the cluster takes a microsecond here, which a
// warp would spend at every stage.)
__device__ __forceinline__ void arrive_first(uint64_t* b) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0)
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(first_of(b)) : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* b) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
      "[%0], %1;" ::"r"(smem_of(b)),
      "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 x, y; setp.ne.b32 p, %4, 0; mov.b64 x, {%1, %5}; "
      "mov.b64 y, {%2, %5};\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], x, y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "n"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Four matrices of eight rows of 16 bytes (lane l names row l % 8 of the (l / 8)th), turned: a
// lane gets column l / 4, elements 2 (l % 4) and the next, of each.
__device__ __forceinline__ void turned(uint32_t at, uint32_t* v) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(at)
               : "memory");
}
// acc += s * v, two at a time
__device__ __forceinline__ void add_scaled(float* acc, const uint32_t* v, float s) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(two(v)), "l"(two(s, s)), "l"(two(acc[0], acc[1])));
  uint32_t x[2];
  split(r, x);
  acc[0] = __uint_as_float(x[0]);
  acc[1] = __uint_as_float(x[1]);
}

// A warp's sums into rows of y: lane l holds row l of its two tiles of the matrix, acc[c] the
// column first + c of the unit's, `columns` of them. Elements of 16 bits are turned through
// shared memory, sixteen columns at a time (a row of the matrix, its columns along it, and
// back by ldmatrix, which turns), so that a lane has eight neighbours of a row of y: written
// as they lie, 64 bytes a store, they took 6.5 us a unit of 256 columns, a fifth of its time.
template <class T>
__device__ __forceinline__ void write_rows(const ProductArgs& p, const Unit& u, int tile, int first,
                                           int columns, const float* acc, uint8_t* room) {
  const W4Args& w = p.w;
  const int lane = threadIdx.x & 31;
  const int there = min(u.count - first, columns);      // columns that are rows of y
  const int64_t row0 = (int64_t)u.start + first;
  const int halves = w.n / 2;
  if (p.y_f32) {
    const int r = lane & 15;
    int feature = tile * 16 + r, end = w.n;
    if (w.gated) {                                       // (the two halves as they are)
      feature = (tile >> 1) * 16 + r;
      end = feature < halves ? w.n : 0;
      if (lane >= 16) feature += halves;
    }
    float* y = reinterpret_cast<float*>(p.y) + row0 * p.y_row + feature;
    const int mine = feature < end ? there : 0;
#pragma unroll
    for (int c = 0; c < 128; ++c) {
      if (c < mine) *y = acc[c];
      y += p.y_row;
    }
    return;
  }
  const bool joined = w.gated;
  // where this lane's row stands in the turned tile, so that a matrix of eight by eight has the
  // rows that give a lane neighbours: all 32, or of a gated matrix 16
  const int f = joined ? lane & 15 : lane;
  const int i = joined ? f >> 1 & 1 : f >> 1 & 3, at = 8 * i + 2 * (joined ? f >> 2 : f >> 3) + (f & 1);
  auto place = [&](int row, int piece) { return room + row * 32 + ((piece ^ ((row >> 2 ^ row >> 3) & 1)) << 4); };
  const int per = joined ? 4 : 8;                        // neighbours of a lane
  const int feature = (joined ? (tile >> 1) * 16 : (tile & ~1) * 16) + (lane & 3) * per;
  const int end = joined ? halves : w.n;
  const bool wide = p.y_wide && feature + per <= end;
  T* y = reinterpret_cast<T*>(p.y) + (row0 + (lane >> 2)) * p.y_row + feature;
  auto store = [&](int col, const uint32_t* v) {         // of column col + lane / 4
    if (col + (lane >> 2) >= there) return;
    T* to = y + (int64_t)col * p.y_row;
    if (wide) {
      if (joined) *reinterpret_cast<uint2*>(to) = make_uint2(v[0], v[1]);
      else *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < per && feature + e < end)
          to[e] = reinterpret_cast<const T*>(v)[e];
    }
  };
#pragma unroll
  for (int c = 0; c < 128; c += 16) {
    if (c >= columns) break;
    __syncwarp();
    if (joined) {
      // lanes of gates take the first eight columns, the others the next
      const bool gate = lane < 16;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float other = __shfl_xor_sync(0xffffffffu, gate ? acc[c + 8 + e] : acc[c + e], 16);
        v[e] = gated<true>(gate ? acc[c + e] : other, gate ? other : acc[c + 8 + e]);
      }
      *reinterpret_cast<uint4*>(place(at, gate ? 0 : 1)) = Vec<T>::put(v);
    } else {
      *reinterpret_cast<uint4*>(place(at, 0)) = Vec<T>::put(acc + c);
      *reinterpret_cast<uint4*>(place(at, 1)) = Vec<T>::put(acc + c + 8);
    }
    __syncwarp();
    if (joined) {
      // matrices: rows 0-7 and 8-15 of the first eight columns, then of the next
      uint32_t v[4];
      turned(smem_of(place((lane >> 3 & 1) * 8 + (lane & 7), lane >> 4)), v);
      store(c, v);
      store(c + 8, v + 2);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t v[4];
        turned(smem_of(place(lane, h)), v);
        store(c + 8 * h, v);
      }
    }
  }
}

template <class T, class S, int GROUP, int WIDTH>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_w4_tc(const __grid_constant__ TcArgs a, const __grid_constant__ CUtensorMap rows, tre_diag* diag) {
  extern __shared__ __align__(1024) uint8_t sm[];
  constexpr int PER = GROUP >= 64 ? 1 : 2;             // groups of a stage
  constexpr int STAGES_OF = GROUP == 128 ? 2 : 1;      // stages of a group
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int side = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const W4Args& w = a.p.w;

  using R = Ring<WIDTH>;
  // What products need (full) and free accumulators (sum_empty) are barriers of the pair's
  // first block, the others each block's own. `done` says that a stage's products are over: its
  // rows' place is free for the stage R::B later, its operand's for the one R::A later.
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + R::AT_BAR);
  uint64_t *raw_full = bars, *raw_empty = raw_full + R::RAW, *full = raw_empty + R::RAW,
           *done = full + R::B, *sum_full = done + R::B, *sum_empty = sum_full + R::SUMS;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(bars + R::BARS);
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_at + 1);
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     smem_of(tmem_at))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  if (tid == 0) {
    *dead = 0;
    for (int k = 0; k < R::RAW; ++k) {
      bar_init(raw_full + k, 1);
      bar_init(raw_empty + k, 1);
    }
    for (int k = 0; k < R::B; ++k) {
      bar_init(full + k, 3);             // both blocks' operands, and the rows
      bar_init(done + k, 1);
    }
    for (int k = 0; k < R::SUMS; ++k) {
      bar_init(sum_full + k, 1);
      bar_init(sum_empty + k, 2 * kScaleWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tmem_before();
  __syncthreads();
  pair_sync();
  tmem_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_at, 0);
  Unit u;

  // Registers move once, from the launch's 4 x 128 (in groups of four warps).
  if (warp < kScaleWarps) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  if (warp < kScaleWarps) {
    // ---- sums of groups ----------------------------------------------------------
    const int quarter = warp & 3, half = warp >> 2, r16 = lane & 15;
    const int g = (r16 & 3) << 1 | (r16 >> 2 & 1);       // turn(g) == r16 & 7
    uint32_t n = 0;                                      // groups so far
    bool alive = true;
    for (int i = pair; alive && unit_at(a, i, u); i += pairs) {
      const int mine = u.columns / 2;                    // columns of this warp, from half * mine on
      const int tile = (2 * u.block + side) * 8 + 2 * quarter + (lane >> 4);
      const uint16_t* scale =
          reinterpret_cast<const uint16_t*>(
              w.scales + (((int64_t)u.expert * w.tiles + min(tile, w.tiles - 1)) * w.groups) * 8 + g) +
          (r16 >> 3);
      float acc[128];
#pragma unroll
      for (int c = 0; c < 128; ++c) acc[c] = 0.f;
      uint16_t ahead = scale[0];
#pragma unroll 1
      for (int q = 0; q < w.groups; ++q, ++n) {
        const uint16_t bits = ahead;
        if (q + 1 < w.groups) ahead = scale[(q + 1) * 16];
        const uint32_t buf = n % R::SUMS;
        if (!(alive = bar_wait(sum_full + buf, (n / R::SUMS) & 1, dead))) break;
        tmem_after();
        float s, unused;
        unpack((uint32_t)bits, s, unused, S());
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + buf * WIDTH + half * mine;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (b * 32 >= mine) break;
          uint32_t v[32];
          tmem_ld32(at + b * 32, v);
          tmem_wait_ld(v);
          if ((b + 1) * 32 >= mine) {                    // all read
            tmem_before();
            arrive_first(sum_empty + buf);
          }
#pragma unroll
          for (int c = 0; c < 32; c += 2) add_scaled(acc + b * 32 + c, v + c, s);
        }
      }
      if (!alive) break;
      write_rows<T>(a.p, u, tile, half * mine, mine, acc, sm + R::AT_OUT + warp * 1024);
    }
  } else if (warp < kCodeWarp + kCodeWarps) {
    // ---- codes to an operand -------------------------------------------------------
    // A warp takes every fifth stage: what happens to one, step after step, takes three times
    // as long as its products.
    const int cw = warp - kCodeWarp, g = lane >> 2, t = lane & 3;
    const uint32_t bits = hidden(Whole<T>::bits);
    uint32_t n = 0, own = cw;                            // stages so far, and this warp's next
    bool alive = true;
    for (int i = pair; alive && unit_at(a, i, u); i += pairs) {
      const int tile0 = (2 * u.block + side) * 8;
      const uint32_t* zeros = w.zeros + ((int64_t)u.expert * w.tiles * w.groups) * 8 + g;
#pragma unroll 1
      for (; own < n + w.chunks; own += kCodeWarps) {
        const uint32_t k = own, s = k % R::A, r = k % R::RAW;
        const int c = (int)(k - n);
        uint32_t z[8][PER];
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int y = 0; y < PER; ++y)
            z[x][y] = zero_as<T, S>(
                w.zeros ? zeros[((int64_t)min(tile0 + x, w.tiles - 1) * w.groups + (c * 64 / GROUP + y)) * 8]
                        : Whole<S>::bits + 0x00080008u);
        // A wait for a parity also passes a phase early, and this warp does not see all phases.
        // With the products of stage k - A over those before it are: the code copied to this
        // stage's place before has been used, and `done` itself has come so far.
        static_assert(R::A <= R::RAW && R::B >= kCodeWarps && R::A <= R::B, "phases that are known to be over");
        const uint32_t last = k - R::A;
        if (k >= R::A && !(alive = bar_wait(done + last % R::B, (last / R::B) & 1, dead))) break;
        if (!(alive = bar_wait(raw_full + r, (k / R::RAW) & 1, dead))) break;
        const uint4* codes = reinterpret_cast<const uint4*>(sm + R::AT_RAW + r * R::BYTES_RAW) + lane;
        uint8_t* to = sm + s * R::BYTES_A;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const uint4 code = codes[x * 32];
          const int row = x * 16 + turn(g);
#pragma unroll
          for (int h = 0; h < 2; ++h) {                  // 32 elements each
            const uint32_t zz = z[x][h * (PER - 1)];
            uint32_t p[4], q[4];
            whole<T>(h ? code.z : code.x, both_lo(zz), both_hi(zz), bits, p);
            whole<T>(h ? code.w : code.y, both_lo(zz), both_hi(zz), bits, q);
            const int at = ((4 * h + t) ^ (row & 7)) << 4;
            *reinterpret_cast<uint4*>(to + row * 128 + at) = make_uint4(p[0], p[2], q[0], q[2]);
            *reinterpret_cast<uint4*>(to + (row + 8) * 128 + at) = make_uint4(p[1], p[3], q[1], q[3]);
          }
        }
        bar_arrive_warp(raw_empty + r);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        arrive_first(full + k % R::B);
      }
      n += w.chunks;
    }
  } else {
    if (warp == kRowWarp) {
      // ---- rows of x ---------------------------------------------------------------
      uint32_t n = 0;
      bool alive = true;
      for (int i = pair; alive && unit_at(a, i, u); i += pairs) {
        const int mine = u.columns / 2, first = u.start + side * mine;
        const uint32_t bytes = (mine + a.box - 1) / a.box * a.box * 128;
#pragma unroll 1
        for (int c = 0; c < w.chunks; ++c, ++n) {
          const uint32_t s = n % R::B;
          if (!(alive = bar_wait(done + s, ((n / R::B) & 1) ^ 1, dead))) break;
          if (side == 0 && lane == 0) bar_expect(full + s, 2 * bytes);
          __syncwarp();
          if (lane * a.box < mine)
            asm volatile(
                "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                "[%0], [%1, {%2, %3}], [%4];" ::"r"(smem_of(sm + R::AT_B + s * R::BYTES_B) + lane * a.box * 128),
                "l"(&rows), "r"(c * 64), "r"(first + lane * a.box), "r"(first_of(full + s))
                : "memory");
          __syncwarp();
        }
      }
      // the products' arrivals that nothing waits for any more
      for (uint32_t k = n > R::B ? n - R::B : 0; alive && k < n; ++k)
        alive = bar_wait(done + k % R::B, (k / R::B) & 1, dead);
    } else if (warp == kRawWarp) {
      // ---- codes -------------------------------------------------------------------
      uint32_t n = 0;
      bool alive = true;
      for (int i = pair; alive && unit_at(a, i, u); i += pairs) {
        // (past the last block of 128 rows: the last again, whose sums are not written)
        // Copies ask for codes some way ahead of the ring, whose places are taken while codes are
        // turned: memory's latency then stays out of that round.
        const uint4* from = w.codes_of(u.expert, min(2 * u.block + side, w.blocks - 1) * 8);
        auto ask = [&](int c) {
          if (c < w.chunks && lane == 0)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from + (int64_t)c * kNextChunk),
                         "n"(R::BYTES_RAW)
                         : "memory");
        };
#pragma unroll 1
        for (int c = 0; c < kAsk; ++c) ask(c);
#pragma unroll 1
        for (int c = 0; c < w.chunks; ++c, ++n) {
          const uint32_t r = n % R::RAW;
          ask(c + kAsk);
          if (!(alive = bar_wait(raw_empty + r, ((n / R::RAW) & 1) ^ 1, dead))) break;
          if (one_lane()) {
            bar_expect(raw_full + r, R::BYTES_RAW);
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                    smem_of(sm + R::AT_RAW + r * R::BYTES_RAW)),
                "l"(from + (int64_t)c * kNextChunk), "n"(R::BYTES_RAW), "r"(smem_of(raw_full + r))
                : "memory");
          }
          __syncwarp();
        }
      }
    } else if (warp == kMmaWarp && side == 0 && one_lane()) {
      // ---- products ------------------------------------------------------------------
      // One thread, which does as little as it can: with waits of a whole warp and an arrival
      // for each ring a stage took it 700 cycles, more than the stage's products.
      const uint32_t x0 = operand(smem_of(sm), 16), y0 = operand(smem_of(sm + R::AT_B), 16);
      uint32_t sa = 0, sb = 0, full_phase = 0, buf = 0, sum_phase = 1;
      bool alive = true, fresh = true;                   // fresh: a group begins
      for (int i = pair; alive && unit_at(a, i, u); i += pairs) {
        // 256 rows of the matrix over the two blocks
        const uint32_t id = (idesc_of<T>(u.columns, false) & 0x00ffffffu) | (256u >> 4) << 24;
#pragma unroll 1
        for (int c = 0; c < w.chunks; ++c) {
          if (!(alive = bar_wait_one(full + sb, full_phase, dead))) break;
          const uint32_t x = x0 + sa * (R::BYTES_A >> 4), y = y0 + sb * (R::BYTES_B >> 4);
#pragma unroll
          for (int h = 0; h < PER; ++h) {
            if (fresh && !(alive = bar_wait_one(sum_empty + buf, sum_phase, dead))) break;
            tmem_after();
#pragma unroll
            for (int k = h * 4 / PER; k < (h + 1) * 4 / PER; ++k)
              mma_pair(tmem + buf * WIDTH, x + k * 2, y + k * 2, id, !(fresh && k == h * 4 / PER));
            if (STAGES_OF == 1 || !fresh) {              // the group is whole
              commit_pair(sum_full + buf);
              fresh = true;
              if (++buf == R::SUMS) {
                buf = 0;
                sum_phase ^= 1;
              }
            } else {
              fresh = false;
            }
          }
          if (!alive) break;
          commit_pair(done + sb);
          if (++sa == R::A) sa = 0;
          if (++sb == R::B) {
            sb = 0;
            full_phase ^= 1;
          }
        }
      }
    }
    __syncwarp();
  }
  // A block that has given up does not know which of its copies and products are still on
  // their way: it stays some 20 ms, far longer than any takes.
  __syncthreads();
  if (*dead) {
    const long long from = clock64();
    while (clock64() - from < kDrainClocks) {
    }
  }
  tmem_before();
  pair_sync();
  tmem_after();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  if (tid == 0 && *dead && diag) diag->err = TRE_ETIMEOUT;
}

// Rows of x in boxes of `box` rows and 64 elements.
bool make_map(CUtensorMap& m, bool bf16, const ProductArgs& p, int64_t rows, int box) {
  const Encode enc = encoder();
  const int64_t stride = p.x_row * 2;
  if (!enc || stride <= 0 || stride >= (1ll << 40)) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)p.w.k, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride};
  const cuuint32_t size[2] = {64, (cuuint32_t)box}, one[2] = {1, 1};
  return enc(&m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
             const_cast<uint8_t*>(p.x), dims, strides, size, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, class S, int GROUP, int WIDTH>
cudaError_t launch_wide(const TcArgs& a, const CUtensorMap& rows, int64_t units, tre_diag* diag,
                        cudaStream_t s) {
  const void* fn = (const void*)k_w4_tc<T, S, GROUP, WIDTH>;
  cudaError_t e = func_smem_once(fn, Ring<WIDTH>::SMEM, true);
  if (e) return e;
  const int64_t pairs = std::min<int64_t>(units, std::max(1, device_sm_count() / 2));
  k_w4_tc<T, S, GROUP, WIDTH><<<(unsigned)(2 * pairs), kThreads, Ring<WIDTH>::SMEM, s>>>(a, rows, diag);
  return cudaGetLastError();
}
template <class T, class S, int GROUP>
cudaError_t launch_typed(const TcArgs& a, const CUtensorMap& rows, int64_t units, tre_diag* diag,
                         cudaStream_t s) {
  return a.tile <= 128 ? launch_wide<T, S, GROUP, 128>(a, rows, units, diag, s)
                       : launch_wide<T, S, GROUP, 256>(a, rows, units, diag, s);
}
template <class T, class S>
cudaError_t launch_group(int group, const TcArgs& a, const CUtensorMap& rows, int64_t units, tre_diag* diag,
                         cudaStream_t s) {
  if (group == 32) return launch_typed<T, S, 32>(a, rows, units, diag, s);
  if (group == 64) return launch_typed<T, S, 64>(a, rows, units, diag, s);
  return launch_typed<T, S, 128>(a, rows, units, diag, s);
}

}  // namespace

cudaError_t launch_w4_tc(int dtype, int scale_dtype, int group, const ProductArgs& p, int64_t rows,
                         int64_t tiles, tre_diag* diag, cudaStream_t s) {
  TcArgs a;
  a.p = p;
  a.p.y_wide = p.y_row % 8 == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
  a.row_blocks = (p.w.tiles + 15) / 16;
  a.tile = p.plan.piece;
  if (!p.plan.order) {
    // Rows of a unit: those with which the rounds of units take least. A round of 64 stages took
    // 17, 20 and 23 us with 128, 192 and 256 rows (30,000 rows of 4,096, groups of 128).
    const int64_t pairs = std::max(1, device_sm_count() / 2);
    int64_t least = -1;
    for (int n = 32; n <= kTileTokens; n += 32) {
      const int64_t units = (rows + n - 1) / n * a.row_blocks;
      const int64_t cost = (units + pairs - 1) / pairs * (n + 280);
      if (least < 0 || cost < least) {
        least = cost;
        a.tile = n;
      }
    }
    tiles = (rows + a.tile - 1) / a.tile;
  }
  // (a copy is issued in some hundred cycles, whatever its size: few of them, of a power of
  // two so that they fit)
  a.box = a.tile / 2;
  if (p.plan.order) {
    a.box = 16;
    while (a.box < a.tile / 2 && a.box * 2 * tiles < rows) a.box *= 2;
  }
  if (tiles * a.row_blocks > 2000000000) return cudaErrorNotSupported;
  CUtensorMap map;
  memset(&map, 0, sizeof(map));
  if (!make_map(map, dtype == TRE_BF16, p, rows, a.box)) return cudaErrorNotSupported;
  const int64_t units = tiles * a.row_blocks;
  if (dtype == TRE_BF16) return launch_group<__nv_bfloat16, __nv_bfloat16>(group, a, map, units, diag, s);
  return scale_dtype == TRE_BF16 ? launch_group<__half, __nv_bfloat16>(group, a, map, units, diag, s)
                                 : launch_group<__half, __half>(group, a, map, units, diag, s);
}

}  // namespace tre
