// A (block, KV head) tile of a KV pool held in 4 or 8 bits: its layout, and the conversions
// between its codes and bf16.
//
// 32 neighbouring features of a row share a scale 2^e, and each is an E2M1 (4 bits) or E4M3
// (8 bits) number times that.  All such numbers are bf16 numbers, so reading is exact, and
// gfx950 converts both ways with the scale in the instruction (v_cvt_scalef32_pk_*).
//
// The layout is the one that the matrix instructions' lanes want (16 keys x 16 rows tiles; lane
// l is row or key l & 15, and quarter l >> 4 of the contracted index):
//   K codes  [16 keys][D]: a lane's 32 features of a key (D = 128) are one scale group, 16
//            bytes at 4 bits, and 64 lanes read the tile's 1024 bytes in one instruction;
//   V codes  [16 groups][16 keys][D / 16 features]: with V^T as the A operand a lane supplies
//            D / 16 features (one to each of as many products) of four keys, again 16 bytes in a
//            row at 4 bits and D = 128.  In [key][D] order it would need a transpose in LDS;
//   scales   of K [16 keys][D / 32], of V [D / 32][16 keys], one byte e + 127 each, 255 = NaN.
// At D = 128 a tile is 2176 or 4224 bytes: whole 128-byte lines, K and V in one stretch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cs {
namespace {

constexpr int kScaleGroup = 32;      // features that share a scale

template <int D, int kBits>
struct QuantTile {
  static constexpr int kRowBytes = D * kBits / 8;          // codes of a row
  static constexpr int kGroups = D / kScaleGroup;          // scales of a row
  static constexpr int kPart = D / 16;                     // features of a V group
  static constexpr int kPartBytes = kPart * kBits / 8;
  static constexpr int kV = 16 * kRowBytes;                // offsets of V's codes and the scales
  static constexpr int kKScales = 2 * kV;
  static constexpr int kVScales = kKScales + 16 * kGroups;
  static constexpr int kBytes = kVScales + 16 * kGroups;
  // The smallest and largest scale bytes that are written.  With the smallest every nonzero
  // number is a normal bf16 number (half of 2^-125; 2^-9 of 2^-117), with the largest all are
  // finite (6 * 2^125; 448 * 2^119).
  static constexpr int kMinScale = kBits == 4 ? 2 : 10;
  static constexpr int kMaxScale = kBits == 4 ? 252 : 246;
};
constexpr int kNanScale = 255;

typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef short i16_pair __attribute__((ext_vector_type(2)));

// (A bit cast of a vector's element, with ROCm 7.2, casts element 0: this takes a copy.)
__device__ __forceinline__ bf16_pair as_pair(uint32_t x) { return __builtin_bit_cast(bf16_pair, x); }

__device__ __forceinline__ float scale_of(int byte) { return __builtin_bit_cast(float, byte << 23); }

// Scale byte of a group whose largest magnitude has the bf16 bits `top`: the smallest exponent
// for which it does not round past the format's largest number (6 or 448).  That is its own
// exponent less the largest number's (2 or 8), or one more from 1.75 (a tie, and 6 has an odd
// code) or above 1.8125 (at the tie 448 has the even one) times its power of two.
template <int D, int kBits>
__device__ __forceinline__ int scale_byte(unsigned top) {
  using T = QuantTile<D, kBits>;
  if (top >= 0x7f80u) return kNanScale;
  const int e = kBits == 4 ? (int)((top + 0x20u) >> 7) - 2 : (int)((top + 0x17u) >> 7) - 8;
  return min(max(e, T::kMinScale), T::kMaxScale);
}

// Two numbers of `code` as a pair of bf16: byte `sel` of it at 4 bits, its 16-bit half `sel` at 8.
template <int kBits>
__device__ __forceinline__ uint32_t read_pair(uint32_t code, float scale, int sel) {
  if constexpr (kBits == 4) {
    switch (sel) {
      case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
      case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
      case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
      default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    }
  } else {
    return sel ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, false));
  }
}

}  // namespace
}  // namespace cs
