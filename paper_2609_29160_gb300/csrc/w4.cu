// Products with matrices in 4 bits: their layout, the products of few rows, and the plan of
// experts' tokens. Many rows are w4_tc.cu's.
#include <algorithm>

#include "internal.h"
#include "w4.cuh"
#include "w4_rule.h"

namespace tre {
namespace {

// ---------------------------------------------------------------------------
// Layout
// ---------------------------------------------------------------------------
struct Layout {
  int64_t tiles, blocks, chunks, groups;
  size_t codes, scales, zeros, bytes;      // where each begins, and the whole
};
Layout layout_of(int experts, int n, int k, int group, bool gated, bool zeros) {
  Layout l;
  l.tiles = gated ? (n / 2 + 15) / 16 * 2 : ((int64_t)n + 31) / 32 * 2;
  l.blocks = (l.tiles + 7) / 8;
  l.chunks = ((int64_t)k + 63) / 64;
  l.groups = l.chunks * 64 / group > 0 ? l.chunks * 64 / group : 1;
  Arena a(nullptr);
  a.take<uint4>((size_t)experts * l.blocks * l.chunks * 256);
  l.codes = 0;
  l.scales = (a.off + 255) & ~size_t(255);
  a.take<uint32_t>((size_t)experts * l.tiles * l.groups * 8);
  l.zeros = (a.off + 255) & ~size_t(255);
  if (zeros) a.take<uint32_t>((size_t)experts * l.tiles * l.groups * 8);
  l.bytes = a.off;
  return l;
}

struct PackArgs {
  const uint8_t *codes, *zeros;
  const uint16_t* scales;
  uint32_t *to_codes, *to_scales, *to_zeros;
  int64_t tiles, blocks, chunks, groups;
  int32_t n, k, group;
  bool gated, bf16;
};
// Row r of tile `tile`, -1: none.
__device__ __forceinline__ int row_of(const PackArgs& a, int64_t tile, int r) {
  if (a.gated) {
    const int64_t i = (tile >> 1) * 16 + r;
    return i < a.n / 2 ? (int)((tile & 1) * (a.n / 2) + i) : -1;
  }
  const int64_t i = tile * 16 + r;
  return i < a.n ? (int)i : -1;
}
// A thread a word of codes (once in a program's life).
__global__ void k_w4_codes(PackArgs a, int64_t words) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= words) return;
  const int s = at & 3, lane = (at >> 2) & 31, g = lane >> 2, t = lane & 3;
  const int64_t block = (at >> 10) / a.chunks, chunk = (at >> 10) - block * a.chunks;
  const int64_t e = block / a.blocks, tile = block % a.blocks * 8 + (at >> 7 & 7);
  uint32_t w = 0;
  for (int i = 0; i < 4; ++i) {
    const int row = row_of(a, tile, turn(g) + 8 * (i & 1));
    const int64_t k = chunk * 64 + 32 * (s >> 1) + 8 * t + 4 * (s & 1) + 2 * (i >> 1);
    if (row < 0 || k >= a.k) continue;
    const uint32_t b = a.codes[((e * a.n + row) * a.k + k) / 2];
    w |= (b & 15) << (4 * i) | (b >> 4) << (4 * i + 16);
  }
  a.to_codes[at] = w;
}
// A thread a pair of scales and zeros. Those of no row or no element are 0, which takes what
// the codes there give out of the sums.
__global__ void k_w4_scales(PackArgs a, int64_t words) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= words) return;
  const int g = at & 7;
  const int64_t group = (at >> 3) % a.groups, tile = (at >> 3) / a.groups, e = tile / a.tiles;
  uint32_t sc = 0, ze = 0;
  for (int h = 0; h < 2; ++h) {
    const int row = row_of(a, tile % a.tiles, turn(g) + 8 * h);
    uint32_t s = 0, z = 8;
    if (row >= 0 && group * a.group < a.k) {
      const int64_t from = (e * a.n + row) * (a.k / a.group) + group;
      s = a.scales[from];
      if (a.zeros) z = a.zeros[from] & 15;
    }
    sc |= s << (16 * h);
    ze |= (z | (a.bf16 ? 0x4300u : 0x6400u)) << (16 * h);
  }
  a.to_scales[at] = sc;
  if (a.to_zeros) a.to_zeros[at] = ze;
}

// ---------------------------------------------------------------------------
// Launches that may begin while the one before still runs (programmatic serialisation): what
// it has written is read after after_launch alone, which every block comes to. Only launches that
// are followed by one of these let it begin: what a caller launches next is ordered as ever.
__device__ __forceinline__ void after_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <class... A, class... B>
cudaError_t launch_behind(void (*kernel)(A...), dim3 grid, int threads, int room, cudaStream_t s, B... args) {
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = grid;
  c.blockDim = dim3((unsigned)threads);
  c.dynamicSmemBytes = (size_t)room;
  c.stream = s;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, A(args)...);
}

// ---------------------------------------------------------------------------
// Products of few rows.
//
// Bound by reading the codes, and as much by the instructions that turn them: some 350 for the
// 2 KB that a step of a warp takes, of which 110 are shifts and masks and 64 subtractions. A warp
// takes two tiles of 16 rows, 128 elements of k at a time, out of a ring of its own that
// asynchronous copies fill two steps ahead with codes and with x, and multiplies them by up to
// 8 NB rows of x with warp products whose accumulators are a group's sums (codes less zeros are
// whole numbers, exact in 16 bits; the scale is applied once a group, in 32 bits). Where there
// are few tiles `split` warps share one and go through k in turn; their sums are joined in order
// through shared memory.
// 8 rows x 4,096 x 65,536, bf16, groups of 128: 36 us for 139 MB (3.9 TB/s), issue slots 60%
// taken; 61 tokens over 128 experts (2,048 x 768 x 3, f16, groups of 64 with zeros): 45 us a
// product on average, 68 with one load of x a step ahead and passes of eight rows.
// ---------------------------------------------------------------------------
constexpr int kFewWarps = 8;

// d = a b, or d += a b
template <class T, bool FRESH>
__device__ __forceinline__ void mma_few(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
#define TRE_MMA(type)                                                                              \
  if constexpr (FRESH)                                                                             \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." type "." type                                     \
                 ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"                  \
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])                                  \
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));        \
  else                                                                                             \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." type "." type                                     \
                 ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"                      \
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])                                  \
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1))
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    TRE_MMA("bf16");
  } else {
    TRE_MMA("f16");
  }
#undef TRE_MMA
}

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

__device__ __forceinline__ void zero16(uint32_t to) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
}

// A step's place in a warp's ring: codes [tile][chunk][lane], scales and zeros
// [tile][group][g], x [32 elements][8 rows][lane]; and how many there are. Two blocks an SM
// with up to 16 rows, one with more.
template <int NB, int GROUP> struct FewRoom {
  static constexpr int PER = 128 / GROUP, SCALES = 2 * PER * 32;
  static constexpr int AT_SCALE = 2048, AT_ZERO = AT_SCALE + SCALES, AT_X = AT_ZERO + SCALES;
  static constexpr int STEP = AT_X + 4 * NB * 512, STEPS = NB % 2 ? 3 : 2;
  static constexpr int RING = STEPS * STEP, SUMS = 8 * NB * 33 * 4;
  static constexpr int WARP = RING > SUMS ? RING : (SUMS + 15) / 16 * 16;
  static constexpr int BLOCKS = NB <= 2 ? 2 : 1;
  static_assert(kFewWarps * WARP * BLOCKS <= 227 * 1024, "shared memory of an SM");
};

// A warp's part of the product of its tiles with the rows of a slot. WARP: bytes of a warp's
// room.
template <class T, class S, int NB, int GROUP, int WARP>
__device__ __forceinline__ void few_rows(const ProductArgs& p, const Slot& slot, int split, uint8_t* room) {
  using St = FewRoom<NB, GROUP>;
  constexpr int PER = St::PER;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const W4Args& w = p.w;
  const int pair = blockIdx.x * (kFewWarps / split) + warp / split, part = warp % split;
  const uint32_t bits = hidden(Whole<T>::bits);
  uint8_t* ring = room + warp * WARP;
  const bool works = 2 * pair < w.tiles;
  const int pr = works ? pair : 0;
  const int64_t tile = (int64_t)slot.expert * w.tiles + 2 * pr;
  const uint4* codes = w.codes_of(slot.expert, 2 * pr) + lane;   // the other tile lies behind it
  const int steps = works ? (w.chunks + 1) / 2 : 0;
  // Each lane's copies of a step: 16 bytes of both chunks of both tiles, and of the scales and
  // zeros of one (tile, group); all go on by `split` steps.
  const bool scale_lane = lane < 4 * PER;
  const int sr = lane / (2 * PER), sq = lane / 2 % PER;
  const int64_t scale0 = ((tile + sr) * w.groups + sq) * 8 + (lane & 1) * 4;
  const uint32_t to_scale = St::AT_SCALE + ((sr * PER + sq) * 2 + (lane & 1)) * 16;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  for (int from = 0; from < slot.count; from += 8 * NB) {
    // What is fetched next: step `next`, its codes, scales and x, into the ring at `put`
    const uint4* next_codes = codes + (int64_t)part * 2 * kNextChunk;
    const uint32_t* next_scale = w.scales + scale0 + part * PER * 8;
    const uint32_t* next_zero = w.zeros + scale0 + part * PER * 8;
    const T* x[NB];
    uint32_t get = 0, put = ring_at;                     // places in the ring
    auto fetch_codes = [&](int step) {
      const uint32_t to = put + lane * 16;
      if ((step + 1) * 128 <= w.k) {                     // (nearly always: no more to ask)
        copy16(to, next_codes);
        copy16(to + 1024, next_codes + 32);
        copy16(to + 512, next_codes + kNextChunk);
        copy16(to + 1536, next_codes + kNextChunk + 32);
        if (scale_lane) {
          copy16(put + to_scale, next_scale);
          if (w.zeros) copy16(put + to_scale + St::SCALES, next_zero);
        }
      } else if (step < steps) {
        copy16(to, next_codes);
        copy16(to + 1024, next_codes + 32);
        if (2 * step + 1 < w.chunks) {
          copy16(to + 512, next_codes + kNextChunk);
          copy16(to + 1536, next_codes + kNextChunk + 32);
        }
        if (scale_lane && step * PER + sq < w.groups) {
          copy16(put + to_scale, next_scale);
          if (w.zeros) copy16(put + to_scale + St::SCALES, next_zero);
        }
      }
      next_codes += split * 2 * kNextChunk;
      next_scale += split * PER * 8;
      next_zero += split * PER * 8;
    };
    auto fetch_x = [&](int step) {
      const uint32_t to = put + St::AT_X + lane * 16;
      const int left = w.k - step * 128;                 // elements from this step on
      if (left >= 128) {
#pragma unroll
        for (int half = 0; half < 4; ++half)
#pragma unroll
          for (int b = 0; b < NB; ++b) copy16(to + (half * NB + b) * 512, x[b] + half * 32);
      } else if (step < steps) {
#pragma unroll
        for (int half = 0; half < 4; ++half)
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if (half * 32 < left) copy16(to + (half * NB + b) * 512, x[b] + half * 32);
            else zero16(to + (half * NB + b) * 512);     // past k
          }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
      for (int b = 0; b < NB; ++b) x[b] += split * 128;
    };
    auto go_on = [&]() { put = put + St::STEP == ring_at + St::RING ? ring_at : put + St::STEP; };
    // (codes do not depend on the launch before, x may)
#pragma unroll
    for (int k = 0; k < St::STEPS - 1; ++k) {
      fetch_codes(part + k * split);
      go_on();
    }
    if (from == 0) after_launch();
    // rows of x of this lane's columns (of columns that are not there, the last one's: what
    // comes of them is not written)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int place = slot.start + min(from + b * 8 + g, slot.count - 1);
      const int64_t row = !p.gather ? place : (p.plan.order ? p.plan.order[place] : place) / p.top;
      x[b] = reinterpret_cast<const T*>(p.x) + row * p.x_row + 8 * t + part * 128;
    }
    put = ring_at;
#pragma unroll
    for (int k = 0; k < St::STEPS - 1; ++k) {
      fetch_x(part + k * split);
      go_on();
    }
    float acc[2][NB][4];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][b][e] = 0.f;
    for (int kb = part; kb < steps; kb += split) {
      const int next = kb + (St::STEPS - 1) * split;
      fetch_codes(next);
      fetch_x(next);
      go_on();
      asm volatile("cp.async.wait_group %0;" ::"n"(St::STEPS - 1) : "memory");
      __syncwarp();
      const uint8_t* now = ring + get;
      get = get + St::STEP == St::RING ? 0 : get + St::STEP;
      const int left = w.k - kb * 128;
      uint4 words[2];                                    // of a chunk, of both tiles
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        // (past the last group: whatever codes by elements of x that are zeros)
        const bool there = PER == 1 || q * GROUP < left;
        uint32_t sc[2], z0[2], z8[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          sc[r] = there ? reinterpret_cast<const uint32_t*>(now + St::AT_SCALE)[(r * PER + q) * 8 + g] : 0u;
          uint32_t z = Whole<S>::bits + 0x00080008u;
          if (w.zeros && there) z = reinterpret_cast<const uint32_t*>(now + St::AT_ZERO)[(r * PER + q) * 8 + g];
          z = zero_as<T, S>(z);
          z0[r] = both_lo(z);
          z8[r] = both_hi(z);
        }
        float sum[2][NB][4];
#pragma unroll
        for (int h = 0; h < GROUP / 32; ++h) {           // 32 elements at a time
          const int half = q * GROUP / 32 + h;
          uint4 v[NB];
#pragma unroll
          for (int b = 0; b < NB; ++b)
            v[b] = *reinterpret_cast<const uint4*>(now + St::AT_X + (half * NB + b) * 512 + lane * 16);
          // (past the last chunk: old codes, by elements of x that are zeros)
          if ((half & 1) == 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
              words[r] = *reinterpret_cast<const uint4*>(now + ((r * 2 + (half >> 1)) * 32 + lane) * 16);
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint2 word = half & 1 ? make_uint2(words[r].z, words[r].w) : make_uint2(words[r].x, words[r].y);
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
              uint32_t a[4];
              whole<T>(sub ? word.y : word.x, z0[r], z8[r], bits, a);
#pragma unroll
              for (int b = 0; b < NB; ++b) {
                const uint32_t b0 = sub ? v[b].z : v[b].x, b1 = sub ? v[b].w : v[b].y;
                if (h == 0 && sub == 0) mma_few<T, true>(sum[r][b], a, b0, b1);
                else mma_few<T, false>(sum[r][b], a, b0, b1);
              }
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float s0, s8;
          unpack(sc[r], s0, s8, S());
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            acc[r][b][0] = fmaf(s0, sum[r][b][0], acc[r][b][0]);
            acc[r][b][1] = fmaf(s0, sum[r][b][1], acc[r][b][1]);
            acc[r][b][2] = fmaf(s8, sum[r][b][2], acc[r][b][2]);
            acc[r][b][3] = fmaf(s8, sum[r][b][3], acc[r][b][3]);
          }
        }
      }
      __syncwarp();
    }
    // The sums take the ring's place: [column][row]
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    auto sums = [&](int of) {
      return reinterpret_cast<float(*)[33]>(room + of * WARP);
    };
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sums(warp)[b * 8 + 2 * t + (e & 1)][r * 16 + turn(g) + 8 * (e >> 1)] = acc[r][b][e];
    if (split > 1) __syncthreads();
    else __syncwarp();
    const int columns = works ? min(8 * NB, slot.count - from) : 0;
    const bool joined = w.gated && !p.apart;
    const int wide = joined ? 16 : 32, first = warp - part;
    for (int i = part * 32 + lane; i < columns * wide; i += split * 32) {
      const int col = i / wide, r = i % wide;
      int64_t n = (int64_t)pair * (w.gated ? 16 : 32) + (w.gated ? r & 15 : r);
      if (n >= (w.gated ? w.n / 2 : w.n)) continue;
      if (w.gated) n += (r >> 4) * (w.n / 2);
      float a = 0.f, u = 0.f;
      for (int k = 0; k < split; ++k) {
        a += sums(first + k)[col][r];
        if (joined) u += sums(first + k)[col][16 + r];
      }
      if (joined) a = gated<true>(a, u);
      const int64_t row = slot.start + from + col;
      if (p.y_f32) reinterpret_cast<float*>(p.y)[row * p.y_row + n] = a;
      else reinterpret_cast<T*>(p.y)[row * p.y_row + n] = T(a);
    }
    if (split > 1) __syncthreads();
    else __syncwarp();
  }
}

// NB: rows of x in eights; 0: one or two, as a slot has them (experts).
template <int NB, int GROUP> struct FewKernel {
  using One = FewRoom<NB ? NB : 1, GROUP>;
  using Two = FewRoom<NB ? NB : 2, GROUP>;
  static constexpr int WARP = One::WARP > Two::WARP ? One::WARP : Two::WARP, BLOCKS = Two::BLOCKS;
};
template <class T, class S, int NB, int GROUP>
__global__ void __launch_bounds__(kFewWarps * 32, FewKernel<NB, GROUP>::BLOCKS)
k_w4_few(const __grid_constant__ ProductArgs p, int split) {
  extern __shared__ __align__(16) uint8_t room[];
  constexpr int WARP = FewKernel<NB, GROUP>::WARP;
  if (p.leads) let_next();
  Slot slot{0, 0, p.n_rows, 0};
  const int piece = p.first_slot + (int)blockIdx.y;
  if (p.ids) {                                         // a pair of a token and its expert each
    const int e = p.ids[piece];
    slot = Slot{e, piece, e >= 0 && e < p.w.experts ? 1 : 0, 0};
  } else if (p.plan.order) {
    after_launch();
    if (piece < p.plan.n[0]) slot = p.plan.tiles[piece];
    else slot.count = 0;
  }
  if (slot.count == 0) {
    after_launch();
    return;
  }
  if constexpr (NB > 0) {
    few_rows<T, S, NB, GROUP, WARP>(p, slot, split, room);
  } else {
    if (slot.count <= 8) few_rows<T, S, 1, GROUP, WARP>(p, slot, split, room);
    else few_rows<T, S, 2, GROUP, WARP>(p, slot, split, room);
  }
}

template <class T, class S, int NB, int GROUP>
cudaError_t few_typed(const ProductArgs& p, int64_t slots, cudaStream_t s) {
  using K = FewKernel<NB, GROUP>;
  constexpr int room = kFewWarps * K::WARP;
  const void* fn = (const void*)k_w4_few<T, S, NB, GROUP>;
  cudaError_t e = func_smem_once(fn, room, true);
  if (e) return e;
  // Warps a tile of 32 rows: the fewest that give each SM twice what it takes at once (8 rows x 4,096
  // x 65,536: 39 us with once as many, 36 with twice, 38 with four times; 1 x 4,096 x 28,672
  // gated 29, 22 and 22).
  const int64_t pairs = p.w.tiles / 2, warps = (int64_t)K::BLOCKS * kFewWarps * device_sm_count();
  const int64_t steps = (p.w.chunks + 1) / 2;
  int split = 1;
  while (split < kFewWarps && pairs * slots * split < 2 * warps && split < steps) split *= 2;
  const int per = kFewWarps / split;
  for (int64_t from = 0; from < slots; from += 65535) {          // (a grid has no more rows)
    ProductArgs q = p;
    q.first_slot = (int32_t)from;
    const dim3 grid((unsigned)((pairs + per - 1) / per), (unsigned)std::min<int64_t>(slots - from, 65535));
    // (behind the plan, or behind the first product)
    if (p.behind && from == 0) e = launch_behind(k_w4_few<T, S, NB, GROUP>, grid, kFewWarps * 32, room, s, q, split);
    else k_w4_few<T, S, NB, GROUP><<<grid, kFewWarps * 32, room, s>>>(q, split);
    if (!e) e = cudaGetLastError();
    if (e) return e;
  }
  return cudaSuccess;
}
template <class T, class S, int NB>
cudaError_t few_by_group(int group, const ProductArgs& p, int64_t slots, cudaStream_t s) {
  if (group == 32) return few_typed<T, S, NB, 32>(p, slots, s);
  if (group == 64) return few_typed<T, S, NB, 64>(p, slots, s);
  return few_typed<T, S, NB, 128>(p, slots, s);
}
template <class T, class S>
cudaError_t few_by_columns(int group, const ProductArgs& p, cudaStream_t s) {
  if (p.n_rows <= 8) return few_by_group<T, S, 1>(group, p, 1, s);
  if (p.n_rows <= 16) return few_by_group<T, S, 2>(group, p, 1, s);
  if (p.n_rows <= 24) return few_by_group<T, S, 3>(group, p, 1, s);
  return few_by_group<T, S, 4>(group, p, 1, s);
}
// tiles: pairs, or pieces that a plan has at most.
cudaError_t launch_few(int dtype, int scale_dtype, int group, const ProductArgs& p, int64_t tiles,
                       cudaStream_t s) {
  if (p.ids)
    return dtype == TRE_BF16 ? few_by_group<__nv_bfloat16, __nv_bfloat16, 1>(group, p, tiles, s)
                             : few_by_group<__half, __half, 1>(group, p, tiles, s);
  if (p.plan.order)
    return dtype == TRE_BF16 ? few_by_group<__nv_bfloat16, __nv_bfloat16, 0>(group, p, tiles, s)
                             : few_by_group<__half, __half, 0>(group, p, tiles, s);
  if (dtype == TRE_BF16) return few_by_columns<__nv_bfloat16, __nv_bfloat16>(group, p, s);
  return scale_dtype == TRE_BF16 ? few_by_columns<__half, __nv_bfloat16>(group, p, s)
                                 : few_by_columns<__half, __half>(group, p, s);
}

cudaError_t launch_rows(int dtype, int scale_dtype, int group, const ProductArgs& p, tre_diag* diag,
                        cudaStream_t s) {
  if (!few_is_quicker(p.n_rows, p.w.tiles, p.w.chunks, group, device_sm_count())) {
    const cudaError_t e = launch_w4_tc(dtype, scale_dtype, group, p, p.n_rows, 0, diag, s);
    if (e != cudaErrorNotSupported) return e;
  }
  return launch_few(dtype, scale_dtype, group, p, 0, s);
}

// ---------------------------------------------------------------------------
// Rows in 32 bits: each is two rows of halves, which times codes (whole numbers, exact as
// halves too) give exact products. The first half has the row's elements over a power of two
// that puts the largest at 2^14 to 2^15, the second what that leaves of them, 2^kSecond times
// (at most 2^3 in the first's steps, so it has room for 2^11 of them): 22 bits together of elements down
// to 2^-28 of the largest, as the second's least step is then 2^-35. With both at one power it
// was 2^-24, and bits went from 2^-17 of the largest on.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;
constexpr int kSecond = 11;

__global__ void __launch_bounds__(kRowThreads) k_split(const float* x, int64_t x_row, int k, int n_rows,
                                                       __half* to, float* back) {
  __shared__ float part[kRowThreads / 32];
  const int64_t t = blockIdx.x;
  const float* from = x + t * x_row;
  float top = 0.f;
  for (int i = threadIdx.x; i < k; i += kRowThreads) {
    const float v = fabsf(from[i]);
    if (v < INFINITY) top = fmaxf(top, v);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRowThreads / 32; ++i) top = fmaxf(top, part[i]);
  // (from the least with which both powers are normal numbers: smaller rows end lower, with a step
  // that is below the smallest float; the largest float's needs no bound)
  const int ex = max((int)(__float_as_uint(top) >> 23), 15);                 // 127 + exponent
  const float by = __uint_as_float((uint32_t)(254 + 14 - ex) << 23);
  if (threadIdx.x == 0) back[t] = __uint_as_float((uint32_t)(ex - 14) << 23);
  for (int i = threadIdx.x; i < k; i += kRowThreads) {
    const float v = from[i] * by;
    const __half hi = __float2half_rn(v);
    to[t * k + i] = hi;
    to[(n_rows + t) * k + i] =
        __float2half_rn(fabsf(v) < INFINITY ? (v - __half2float(hi)) * (float)(1 << kSecond) : 0.f);
  }
}
// both [2 n_rows][n] to y [n_rows][n], or [n_rows][n / 2] of a gated matrix
__global__ void __launch_bounds__(kRowThreads) k_whole_rows(const float* both, const float* back, int n,
                                                            int n_rows, bool join, float* y, int64_t y_row) {
  const int64_t t = blockIdx.x;
  const int wide = join ? n / 2 : n, i = blockIdx.y * kRowThreads + threadIdx.x;
  if (i >= wide) return;
  const float *hi = both + t * n, *lo = both + (n_rows + t) * n;
  const float f = back[t];
  constexpr float second = 1.f / (1 << kSecond);
  float a = fmaf(lo[i], second, hi[i]) * f;
  if (join) a = gated<false>(a, fmaf(lo[wide + i], second, hi[wide + i]) * f);
  y[t * y_row + i] = a;
}

// ---------------------------------------------------------------------------
// Experts: the plan of their tokens, and the sum of a token's experts.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kMaxExperts = 1024;
// Tokens an expert up to which k_w4_few is taken. 64 experts of 2,048 x 1,024 x 3, groups of 128,
// 12 tokens each: 98 us by it, 121 by the tensor cores' kernel, 16 each 124 and 124, 32 each 184 and
// 126; groups of 64, 24 each: 170 and 176; groups of 32, 32 each: 208 and 290, 48 each 286 and 292.
// It is the mean that counts: an expert that gets most of them is done in pieces of 16 that read its codes
// again, out of L2, and others' are not read at all. 900 tokens to 64 such experts take 99 us evenly
// spread and 74 all to one, 15,000 to 1,024 of 512 x 256 x 3 187 and 160, 56 with two of 8 of
// 4,096 x 14,336 x 3 each 278, and 324 with one for all of them.
constexpr int few_tokens(int group) { return group == 32 ? 48 : group == 64 ? 24 : 15; }

// Pairs (token, j) counted and sorted by expert, by one block or a cluster of eight that have a
// part of the pairs each and read one another's counts (24,576 pairs: 18 us by one, 7.6 by eight).
// Which place of its expert a pair gets depends on the order of atomics; the products do not
// depend on places.
constexpr int kPlanBlocks = 8;

__device__ __forceinline__ int count_of(const int32_t* count, int block, int e) {
  uint32_t at;
  int r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(count + e)), "r"(block));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ void all_blocks() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(kPlanThreads) k_plan(const int32_t* ids, int64_t pairs, int experts,
                                                       PlanArgs plan, tre_diag* diag) {
  __shared__ int32_t count[kMaxExperts], next[kMaxExperts];
  __shared__ int32_t warp_sums[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int block = blockIdx.x, blocks = gridDim.x;    // (one cluster)
  const int64_t part = (pairs + blocks - 1) / blocks, first = block * part, end = min64(pairs, first + part);
  let_next();
  count[tid] = 0;
  __syncthreads();
  unsigned long long past = 0;
  // (eight ids on their way at a time: one after the other the loads' latency is all there is)
  constexpr int kIds = 8;
  for (int64_t i = first + tid; i < end; i += kIds * kPlanThreads) {
    int e[kIds];
#pragma unroll
    for (int k = 0; k < kIds; ++k) e[k] = i + k * kPlanThreads < end ? ids[i + k * kPlanThreads] : -1;
#pragma unroll
    for (int k = 0; k < kIds; ++k) {
      if (e[k] >= experts) ++past;
      else if (e[k] >= 0) atomicAdd(&count[e[k]], 1);
    }
  }
  if (diag) warp_add_counter(reinterpret_cast<unsigned long long*>(&diag->dropped_range), past);
  __syncthreads();
  if (blocks > 1) all_blocks();
  int mine = count[tid], before = 0;                   // of this expert: all pairs, those of blocks before
  if (blocks > 1) {
    mine = 0;
    for (int k = 0; k < blocks; ++k) {
      const int c = count_of(count, k, tid);
      mine += c;
      if (k < block) before += c;
    }
  }
  const int tiles = (mine + plan.piece - 1) / plan.piece;
  int v[2] = {mine, tiles};                            // places and tiles up to this expert
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, v[x], o);
      if (lane >= o) v[x] += y;
    }
    if (lane == 31) warp_sums[x][warp] = v[x];
  }
  __syncthreads();
  if (warp < 2) {
    int y = warp_sums[warp][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) y += z;
    }
    warp_sums[warp][lane] = y;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 2; ++x) v[x] += warp > 0 ? warp_sums[x][warp - 1] : 0;
  const int start = v[0] - mine;
  next[tid] = start + before;
  if (block == 0) {
    if (mine > 0) {
      // pieces of one size, whole sixteens
      const int size = ((mine + tiles - 1) / tiles + 15) / 16 * 16;
      for (int k = 0; k < tiles; ++k)
        plan.tiles[v[1] - tiles + k] = Slot{tid, start + k * size, max(0, min(size, mine - k * size)), 0};
    }
    if (tid == kPlanThreads - 1) {
      plan.n[0] = v[1];
      plan.n[1] = v[0];
    }
  }
  __syncthreads();
  for (int64_t i = first + tid; i < end; i += kIds * kPlanThreads) {
    int e[kIds];
#pragma unroll
    for (int k = 0; k < kIds; ++k) e[k] = i + k * kPlanThreads < end ? ids[i + k * kPlanThreads] : -1;
#pragma unroll
    for (int k = 0; k < kIds; ++k)
      if (e[k] >= 0 && e[k] < experts) e[k] = atomicAdd(&next[e[k]], 1);
      else e[k] = -1;
#pragma unroll
    for (int k = 0; k < kIds; ++k)
      if (e[k] >= 0) {
        plan.order[e[k]] = (int)(i + k * kPlanThreads);
        plan.where[i + k * kPlanThreads] = e[k];
      }
  }
  if (blocks > 1) all_blocks();                        // (counts are read until here)
}

cudaError_t launch_plan(const int32_t* ids, int64_t pairs, int experts, const PlanArgs& plan, tre_diag* diag,
                        cudaStream_t s) {
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = pairs > 2 * kPlanThreads ? kPlanBlocks : 1;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(at.val.clusterDim.x);
  c.blockDim = dim3(kPlanThreads);
  c.stream = s;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, k_plan, ids, pairs, experts, plan, diag);
}

// Rows of tokens in the order of their places, for the tensor cores' kernel: copies that gather
// rows there took 1,350 cycles a stage of 256 rows (by tensor copies of four rows or by pieces
// of 16 bytes), 2.5 times its products; this pass 20 us for 24,576 rows of 2,048.
// A warp a row, four pieces a lane on their way.
__global__ void __launch_bounds__(kRowThreads) k_gather(const uint4* x, int64_t x_row, int pieces, int top,
                                                        PlanArgs plan, uint4* to) {
  const int64_t place = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (place >= plan.n[1]) return;                      // (pairs of no expert have no place)
  const uint4* from = x + (int64_t)(plan.order[place] / top) * x_row;
  to += place * pieces;
  for (int i = threadIdx.x & 31; i < pieces; i += 128) {
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + 32 * k < pieces) v[k] = from[i + 32 * k];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + 32 * k < pieces) to[i + 32 * k] = v[k];
  }
}

// y[t] = sum over j, in order, of weights[t][j] * each[where[t * top + j]] (where null: the pair's
// own number); a row of `each` has whole fours (row elements). Four elements a thread.
template <class T>
__global__ void __launch_bounds__(kRowThreads) k_combine(const float* each, const int32_t* where,
                                                         const int32_t* ids, const float* weights,
                                                         int experts, int top, int dim, int row, T* y,
                                                         int64_t y_row, tre_diag* diag) {
  __shared__ int32_t place[32];
  __shared__ float weight[32];
  const int64_t t = blockIdx.x;
  after_launch();
  const int i = (blockIdx.y * kRowThreads + threadIdx.x) * 4;
  if (threadIdx.x < top) {
    const int e = ids[t * top + threadIdx.x];
    const bool there = e >= 0 && e < experts;
    const int64_t pair = t * top + threadIdx.x;
    place[threadIdx.x] = !there ? -1 : where ? where[pair] : (int)pair;
    // (without a plan nobody has counted those yet)
    if (!where && diag && e >= experts && blockIdx.y == 0)
      atomicAdd(reinterpret_cast<unsigned long long*>(&diag->dropped_range), 1ull);
    weight[threadIdx.x] = weights[t * top + threadIdx.x];
  }
  __syncthreads();
  if (i >= dim) return;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j0 = 0; j0 < top; j0 += 8) {                // eight on their way
    float4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j0 + j < top && place[j0 + j] >= 0)
        v[j] = *reinterpret_cast<const float4*>(each + (int64_t)place[j0 + j] * row + i);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j0 + j < top && place[j0 + j] >= 0) {
        const float f = weight[j0 + j];
        sum = make_float4(fmaf(f, v[j].x, sum.x), fmaf(f, v[j].y, sum.y), fmaf(f, v[j].z, sum.z),
                          fmaf(f, v[j].w, sum.w));
      }
  }
  T* to = y + t * y_row + i;
  const float out[4] = {sum.x, sum.y, sum.z, sum.w};
  if (i + 4 <= dim && (reinterpret_cast<uintptr_t>(to) & 7) == 0) {
    *reinterpret_cast<uint2*>(to) = make_uint2(pack<T>(out[0], out[1]), pack<T>(out[2], out[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < dim) to[e] = T(out[e]);
  }
}

template <class T>
cudaError_t launch_combine(const float* each, int row, const int32_t* where, const tre_tokens* t, int experts,
                           int dim, tre_diag* diag, cudaStream_t s) {
  const dim3 grid((unsigned)t->n_rows, (unsigned)((dim + 4 * kRowThreads - 1) / (4 * kRowThreads)));
  return launch_behind(k_combine<T>, grid, kRowThreads, 0, s, each, where, t->ids, t->weights, experts, t->top,
                       dim, row, static_cast<T*>(t->y), t->y_row, diag);
}

bool half_type(int d) { return d == TRE_BF16 || d == TRE_F16; }
bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool shape_ok(int experts, int n, int k, int group, int gated) {
  return experts >= 1 && experts <= kMaxExperts && n >= 1 && n <= (1 << 20) && k >= 1 &&
         k <= (1 << 20) && (group == 32 || group == 64 || group == 128) && k % group == 0 &&
         (!gated || n % 2 == 0);
}

}  // namespace

bool w4_args(const tre_w4* w, W4Args& a) {
  if (!w || !half_type(w->dtype) || !shape_ok(w->experts, w->n, w->k, w->group, w->gated)) return false;
  if (!w->packed || (reinterpret_cast<uintptr_t>(w->packed) & 255)) return false;
  const Layout l = layout_of(w->experts, w->n, w->k, w->group, w->gated != 0, w->zeros != 0);
  const uint8_t* p = static_cast<const uint8_t*>(w->packed);
  a.codes = reinterpret_cast<const uint4*>(p + l.codes);
  a.scales = reinterpret_cast<const uint32_t*>(p + l.scales);
  a.zeros = w->zeros ? reinterpret_cast<const uint32_t*>(p + l.zeros) : nullptr;
  a.experts = w->experts;
  a.n = w->n;
  a.k = w->k;
  a.tiles = (int32_t)l.tiles;
  a.blocks = (int32_t)l.blocks;
  a.chunks = (int32_t)l.chunks;
  a.groups = (int32_t)l.groups;
  a.gated = w->gated != 0;
  return true;
}

}  // namespace tre

using namespace tre;

extern "C" {

tre_status tre_w4_pack(const tre_w4_source* f, void* packed, size_t* bytes, tre_stream stream) {
  if (!f || !bytes || !half_type(f->dtype) || !shape_ok(f->experts, f->n, f->k, f->group, f->gated))
    return TRE_EINVAL;
  const Layout l = layout_of(f->experts, f->n, f->k, f->group, f->gated != 0, f->zeros != nullptr);
  if (!packed) {
    *bytes = l.bytes;
    return TRE_OK;
  }
  if (*bytes < l.bytes) return TRE_ENOMEM;
  if (!f->codes || !f->scales || (reinterpret_cast<uintptr_t>(f->scales) & 1) ||
      (reinterpret_cast<uintptr_t>(packed) & 255))
    return TRE_EINVAL;
  uint8_t* p = static_cast<uint8_t*>(packed);
  PackArgs a;
  a.codes = f->codes;
  a.zeros = f->zeros;
  a.scales = static_cast<const uint16_t*>(f->scales);
  a.to_codes = reinterpret_cast<uint32_t*>(p + l.codes);
  a.to_scales = reinterpret_cast<uint32_t*>(p + l.scales);
  a.to_zeros = f->zeros ? reinterpret_cast<uint32_t*>(p + l.zeros) : nullptr;
  a.tiles = l.tiles;
  a.blocks = l.blocks;
  a.chunks = l.chunks;
  a.groups = l.groups;
  a.n = f->n;
  a.k = f->k;
  a.group = f->group;
  a.gated = f->gated != 0;
  a.bf16 = f->dtype == TRE_BF16;
  const int64_t words = f->experts * l.blocks * l.chunks * 1024, pairs = f->experts * l.tiles * l.groups * 8;
  if ((words + 255) / 256 > 2147483647) return TRE_EINVAL;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  k_w4_codes<<<(unsigned)((words + 255) / 256), 256, 0, s>>>(a, words);
  k_w4_scales<<<(unsigned)((pairs + 255) / 256), 256, 0, s>>>(a, pairs);
  return cudaGetLastError() == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

tre_status tre_linear4(const tre_w4* w, const tre_linear* l, void* ws, size_t* ws_bytes, tre_diag* diag,
                       tre_stream stream) {
  ProductArgs p{};
  if (!l || !ws_bytes || !w4_args(w, p.w) || w->experts != 1 || l->n_rows < 0) return TRE_EINVAL;
  const bool f32 = l->dtype == TRE_F32;
  const bool y_f32 = l->y_dtype == TRE_F32;
  if (!f32 && l->dtype != w->dtype) return TRE_EINVAL;
  if (l->y_dtype != l->dtype && (!y_f32 || p.w.gated)) return TRE_EINVAL;
  if (l->x_row < 0 || l->y_row < 0 || reinterpret_cast<uintptr_t>(l->y) % (y_f32 ? 4 : 2) ||
      reinterpret_cast<uintptr_t>(l->x) % (f32 ? 4 : 16) || (!f32 && l->x_row % 8))
    return TRE_EINVAL;
  if (l->n_rows > (f32 ? 1 << 29 : 1 << 30)) return TRE_EINVAL;
  Arena arena(ws);
  const size_t twice = f32 ? 2 * (size_t)l->n_rows : 0;
  __half* halves = arena.take<__half>(twice * w->k);
  float* both = arena.take<float>(twice * w->n);
  float* back = arena.take<float>(twice / 2);
  if (!ws) {
    *ws_bytes = f32 ? arena.off : 0;
    return TRE_OK;
  }
  if (f32 && *ws_bytes < arena.off) return TRE_ENOMEM;
  if (l->n_rows == 0) return TRE_OK;
  if (!l->x || !l->y) return TRE_EINVAL;
  p.x = static_cast<const uint8_t*>(l->x);
  p.x_row = l->x_row;
  p.y = static_cast<uint8_t*>(l->y);
  p.y_row = l->y_row;
  p.n_rows = l->n_rows;
  p.top = 1;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (!f32) {
    p.y_f32 = y_f32;
    e = launch_rows(w->dtype, w->dtype, w->group, p, diag, s);
  } else {
    k_split<<<l->n_rows, kRowThreads, 0, s>>>(static_cast<const float*>(l->x), l->x_row, w->k, l->n_rows,
                                              halves, back);
    e = cudaGetLastError();
    p.x = reinterpret_cast<const uint8_t*>(halves);
    p.x_row = w->k;
    p.y = reinterpret_cast<uint8_t*>(both);
    p.y_row = w->n;
    p.n_rows = 2 * l->n_rows;
    p.y_f32 = p.apart = true;
    if (!e) e = launch_rows(TRE_F16, w->dtype, w->group, p, diag, s);
    if (!e) {
      const int wide = p.w.gated ? w->n / 2 : w->n;
      k_whole_rows<<<dim3((unsigned)l->n_rows, (unsigned)((wide + kRowThreads - 1) / kRowThreads)),
                     kRowThreads, 0, s>>>(both, back, w->n, l->n_rows, p.w.gated,
                                          static_cast<float*>(l->y), l->y_row);
      e = cudaGetLastError();
    }
  }
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

tre_status tre_experts(const tre_w4* w1, const tre_w4* w2, const tre_tokens* t, void* ws,
                       size_t* ws_bytes, tre_diag* diag, tre_stream stream) {
  ProductArgs a{}, b{};
  if (!t || !ws_bytes || !w4_args(w1, a.w) || !w4_args(w2, b.w)) return TRE_EINVAL;
  if (w1->dtype != t->dtype || w2->dtype != t->dtype || !a.w.gated || b.w.gated ||
      w1->experts != w2->experts || w2->k != w1->n / 2)
    return TRE_EINVAL;
  if (t->n_rows < 0 || t->top < 1 || t->top > 32 || (int64_t)t->n_rows * t->top > 2147483647 / 2)
    return TRE_EINVAL;
  if (t->x_row % 8 || t->x_row < 0 || t->y_row < 0 || !at16(t->x) ||
      (reinterpret_cast<uintptr_t>(t->y) & 1) || (reinterpret_cast<uintptr_t>(t->ids) & 3) ||
      (reinterpret_cast<uintptr_t>(t->weights) & 3))
    return TRE_EINVAL;
  const int64_t pairs = (int64_t)t->n_rows * t->top;
  const int inner = w2->k, inner_row = (inner + 7) / 8 * 8, dim = w2->n;
  const int64_t slots = std::min<int64_t>(w1->experts, pairs);
  const bool few = pairs <= few_tokens(std::max(w1->group, w2->group)) * slots;
  // Hardly any expert twice: a pair is a piece of its own, without a plan.
  const bool direct = few && (t->n_rows == 1 || pairs * 4 <= w1->experts);
  Arena arena(ws);
  PlanArgs plan;
  plan.order = arena.take<int32_t>(pairs);
  plan.where = arena.take<int32_t>(pairs);
  // (pieces of up to 128 rows have twice the accumulators: 100 tokens each took 154 against 162 us;
  // but more than 128 are two pieces: 128 tokens each 210 against 177)
  plan.piece = few ? 16 : pairs <= 96 * slots ? 128 : kTileTokens;
  plan.tiles = arena.take<Slot>(slots + pairs / plan.piece);
  plan.n = arena.take<int32_t>(2);
  // act's output in 16 bits: the second product's operand has no more. Beside the output's own rounding
  // it takes the error against 64 bits from 1.7e-3 to 2.4e-3 in bfloat16, 2.1e-4 to 3.0e-4 in half, where past
  // 65,504 it is an infinity. As two rows, like rows in 32 bits, the second product would be done twice.
  uint8_t* h = arena.take<uint8_t>((size_t)pairs * inner_row * 2);
  const int row = (dim + 3) / 4 * 4;                  // of `each`
  float* each = arena.take<float>((size_t)pairs * row);
  uint4* gathered = arena.take<uint4>(few ? 0 : (size_t)pairs * (w1->k / 8));
  if (!ws) {
    *ws_bytes = arena.off;
    return TRE_OK;
  }
  if (*ws_bytes < arena.off) return TRE_ENOMEM;
  if (t->n_rows == 0) return TRE_OK;
  if (!t->x || !t->y || !t->ids || !t->weights) return TRE_EINVAL;
  a.x = static_cast<const uint8_t*>(t->x);
  a.x_row = t->x_row;
  a.y = h;
  a.y_row = inner_row;
  a.gather = true;
  b.x = h;
  b.x_row = inner_row;
  b.y = reinterpret_cast<uint8_t*>(each);
  b.y_row = row;
  b.y_f32 = true;
  a.plan = b.plan = plan;
  a.n_rows = b.n_rows = t->n_rows;
  a.top = b.top = t->top;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  const int32_t* where = plan.where;
  if (direct) {
    a.plan.order = b.plan.order = nullptr;
    a.ids = b.ids = t->ids;
    where = nullptr;
    b.behind = true;
  } else {
    e = launch_plan(t->ids, pairs, w1->experts, plan, diag, s);
    a.behind = b.behind = few;
  }
  a.leads = b.leads = few;
  const int64_t tiles = direct ? pairs : slots + pairs / plan.piece;
  if (!few && !e) {
    constexpr int rows = kRowThreads / 32;
    k_gather<<<(unsigned)((pairs + rows - 1) / rows), kRowThreads, 0, s>>>(
        static_cast<const uint4*>(t->x), t->x_row / 8, w1->k / 8, t->top, plan, gathered);
    e = cudaGetLastError();
    a.x = reinterpret_cast<const uint8_t*>(gathered);
    a.x_row = w1->k;
    a.gather = false;
  }
  auto product = [&](const ProductArgs& p, const tre_w4* w) {
    if (!few) {
      const cudaError_t x = launch_w4_tc(t->dtype, t->dtype, w->group, p, pairs, tiles, diag, s);
      if (x != cudaErrorNotSupported) return x;
    }
    return launch_few(t->dtype, t->dtype, w->group, p, tiles, s);
  };
  if (!e) e = product(a, w1);
  if (!e) e = product(b, w2);
  if (!e)
    e = t->dtype == TRE_BF16 ? launch_combine<__nv_bfloat16>(each, row, where, t, w1->experts, dim, diag, s)
                             : launch_combine<__half>(each, row, where, t, w1->experts, dim, diag, s);
  return e == cudaSuccess ? TRE_OK : TRE_ECUDA;
}

}  // extern "C"
