// Matrices in 4 bits as the products read them, and what both kernels of the products
// share.
//
// A tile is 16 rows by 64 elements of k, 512 bytes; eight tiles of 128 rows lie together (one
// copy), those blocks one after the other along k. Lane (g, t) = (lane / 4, lane % 4) of a warp has 16 bytes of it: word s holds, of
// rows r = turn(g) and r + 8, the elements k = 32 (s / 2) + 8 t + 4 (s % 2) + 0..3, as
//   half-byte i      : row r + 8 (i % 2), element 2 (i / 2)
//   half-byte i + 4  : the same row, the element after it        (i = 0..3)
// so that one mask gives two neighbours of a row as the two halves of a register. Four
// registers are a warp product's A operand (with the matching order of k in B: any order
// will do for a sum over k), and two words of a row are 16 bytes of a tile in shared memory
// as tcgen05 reads it. turn() puts rows r and r + 4 on neighbouring lanes, whose 16-byte
// pieces then lie in different banks.
// Scales [tile of 16 rows][group][g] are pairs (rows r, r + 8), 4 bytes; zeros the same, as
// the number that is taken from a code that has been read as the last bits of kWhole.
//
// Of a gated matrix every even tile holds 16 rows of the gate and the next tile those that
// they multiply.
#pragma once

#include <type_traits>

#include "kvcache.cuh"

namespace tre {

struct W4Args {
  const uint4* codes;
  const uint32_t *scales, *zeros;      // zeros may be null: 8
  int32_t experts, n, k, tiles, blocks, chunks, groups;   // blocks of eight tiles, of an expert;
  bool gated;                                              // groups of a row, to whole chunks
  // tile `tile` of expert e along k: from here on, kNextChunk further for the next 64 elements
  __device__ __forceinline__ const uint4* codes_of(int e, int tile) const {
    return codes + (((int64_t)e * blocks + (tile >> 3)) * chunks * 8 + (tile & 7)) * 32;
  }
};
constexpr int kNextChunk = 8 * 32;     // in pieces of 16 bytes

__host__ __device__ constexpr int turn(int g) { return g >> 1 | (g & 1) << 2; }

// A whole number below 16 in the last bits of this one is itself plus `kWhole`.
template <class T> struct Whole;
template <> struct Whole<__nv_bfloat16> {
  static constexpr uint32_t bits = 0x43004300u;      // 128
};
template <> struct Whole<__half> {
  static constexpr uint32_t bits = 0x64006400u;      // 1024
};
template <class T> __device__ __forceinline__ uint32_t minus2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t minus2<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a),
                                   *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t minus2<__half>(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
// A pair of zeros, kept for scales of type S, for rows of type T.
template <class T, class S> __device__ __forceinline__ uint32_t zero_as(uint32_t z) {
  return std::is_same<T, S>::value ? z : (z & 0x000f000fu) | Whole<T>::bits;
}
// Both halves the lower / upper half of x
__device__ __forceinline__ uint32_t both_lo(uint32_t x) { return __byte_perm(x, 0, 0x1010); }
__device__ __forceinline__ uint32_t both_hi(uint32_t x) { return __byte_perm(x, 0, 0x3232); }

// A word of codes as whole numbers: a[i] = (half-byte i, half-byte i + 4) less the zero of
// its row (z0: of row r, z8: of row r + 8, with kWhole, in both halves). Halves have room for
// a half-byte four bits up, which is sixteen times itself there: two of three shifts become
// part of the subtraction.
// (w & mask) | bits in one operation, which has room for one constant: `bits` is kept from the
// compiler's sight in a register (with both constants in sight it made two of it).
__device__ __forceinline__ uint32_t hidden(uint32_t bits) {
  uint32_t r;
  asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(bits));
  return r;
}
template <uint32_t MASK> __device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "n"(MASK), "r"(bits));
  return r;
}
// bits: hidden(Whole<T>::bits)
template <class T>
__device__ __forceinline__ void whole(uint32_t w, uint32_t z0, uint32_t z8, uint32_t bits, uint32_t* a) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 part = __float2half2_rn(0.0625f);
    // (1024 + 16 c) / 16 - (64 + z), of row r + 8; z8 has 1024 + z
    const __half2 z = __hsub2(__float2half2_rn(960.f), *reinterpret_cast<const __half2*>(&z8));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t v = w >> (8 * i);
      a[2 * i] = minus2<T>(masked<0x000f000fu>(v, bits), z0);
      const uint32_t up = masked<0x00f000f0u>(v, bits);
      const __half2 x = __hfma2(*reinterpret_cast<const __half2*>(&up), part, z);
      a[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = minus2<T>(masked<0x000f000fu>(w >> (4 * i), bits), i & 1 ? z8 : z0);
  }
}

// What a gate does: g / (1 + exp(-g)) * u, of a negative g as g e / (1 + e) * u with e = exp(-|g|), so
// that the denominator stays between 1 and 2, and e as the square of exp(-|g| / 2), which has an
// exponent left down to g = -206 and goes to g and u once each. QUICK, for outputs of 16 bits: the
// quick exponential is off by 2 + 1.2 |x| units of 2^-23 of itself, so e by 4 + 1.2 |g|, 2^-16 at
// g = -100. Else, for outputs of 32, all is within 18 units of 2^-24. 4,096 rows of 4,096 by
// 8,192 in 32 bits: 437 us with the quick form, 464 so.
template <bool QUICK> __device__ __forceinline__ float gated(float g, float u) {
  const float x = -0.5f * fabsf(g), half = QUICK ? __expf(x) : expf(x);
  const float below = fmaf(half, half, 1.f), by = g < 0.f ? half : 1.f;
  g *= by;
  if constexpr (QUICK) {
    float over;                                        // (off by a unit of 2^-23)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(over) : "f"(below));
    g *= over;
  } else {
    g /= below;
  }
  return g * (u * by);
}

// Tokens of experts, sorted by expert (k_plan): places of one expert lie together; place p is
// pair order[p] = token * top + j.
struct Slot {
  int32_t expert, start, count, pad;
};
struct PlanArgs {
  int32_t* order;                      // [pairs]
  int32_t* where;                      // [pairs]: the place of a pair
  Slot* tiles;                         // their places in pieces of up to `piece`
  int32_t* n;                          // [2]: how many tiles, places
  int32_t piece;
};
constexpr int kTileTokens = 256;       // columns of a product on the tensor cores

// One product of a call.
struct ProductArgs {
  W4Args w;
  const uint8_t* x;
  int64_t x_row;                       // elements
  uint8_t* y;
  int64_t y_row;
  PlanArgs plan;                       // order null: rows as they are, one matrix, or
  const int32_t* ids;                  // a pair each with an expert of these
  bool behind, leads;                  // launched behind what it reads; the next launch is behind it
  int32_t n_rows, top;
  int32_t first_slot;                  // of the plan's pieces that a launch of k_w4_few takes
  bool gather;                         // x's rows are tokens', by place
  bool y_f32;                          // and with it
  bool apart;                          // a gated matrix's two halves as they are
  bool y_wide;                         // eight neighbours of a row of y can be written at once
};

bool w4_args(const tre_w4* w, W4Args& a);
// w4_tc.cu. dtype: of the rows (TRE_BF16 only over scales of that type); rows: how many x has;
// tiles: most that a plan has. cudaErrorNotSupported (nothing was launched): no tensor copy
// takes these rows.
cudaError_t launch_w4_tc(int dtype, int scale_dtype, int group, const ProductArgs& p, int64_t rows,
                         int64_t tiles, tre_diag* diag, cudaStream_t s);

}  // namespace tre
