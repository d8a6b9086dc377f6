// Tiles that go from HBM straight into LDS: the layout of the prefill kernels
// (prefill_paged_attn.hip) and of the key scores' (key_scores.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cs {
namespace {

// Direct-to-LDS staging.  buffer_load_dwordx4 with the
// LDS flag writes lane i's 16 bytes at the instruction's LDS address + 16 i,
// so one load moves 1 KB of a (block, head) tile: four 256-byte rows at
// D = 128, eight 128-byte rows at D = 64 (a "group").  Which 16-byte chunk
// each lane fetches is free, so the layout inside a group is any
// permutation of its chunks.  A buffer holds one 64-key step as 16 (D = 128)
// or 8 (D = 64) groups.
//   D = 128: groups 4 D + 8 elements apart (16 bytes of padding); chunk s of
//            row d holds the row's chunk s ^ 4d.
//   D = 64:  groups 8 D + 16 elements apart (32 bytes); chunk s of row d
//            holds the row's chunk s ^ y(d), y(d) = 4 ((d / 2) % 2) + d / 4.
// The K operand reads (ds_read_b128: 16 lanes, one chunk of 16 rows, per
// pass) and the transposing V reads (32 lanes, 64 bytes of 4 rows, per pass)
// are then free of bank conflicts at 64 banks (checked element by element,
// with the bank of every access, in the host layout test), and every
// per-lane address is one register plus a constant.  Buffer loads rather
// than global_load_lds: the compiler's wait insertion counts a global load
// into LDS as a flat access and then makes every LDS read wait for all loads
// in flight; with buffer loads it keeps exact counts.
template <int D>
struct DirectLayout;
template <>
struct DirectLayout<128> {
  static constexpr int kRows = 4;                 // rows per 1 KB group
  static constexpr int kGrp = 4 * 128 + 8;        // elements from group to group
  static __device__ __forceinline__ int swz(int d) { return 4 * d; }
};
template <>
struct DirectLayout<64> {
  static constexpr int kRows = 8;
  static constexpr int kGrp = 8 * 64 + 16;
  static __device__ __forceinline__ int swz(int d) { return 4 * ((d >> 1) & 1) + (d >> 2); }
};
//
// Word 3 of a raw buffer descriptor on gfx9-family parts: 32-bit data format
// (DATA_FORMAT = 4), no swizzle, no index stride.
constexpr int kRawBufferWord3 = 0x00020000;
// s_waitcnt immediates (gfx9 layout: vmcnt[3:0], expcnt[6:4], lgkmcnt[11:8],
// vmcnt[5:4] at [15:14]; a field at its maximum does not wait)
constexpr int kWaitVmcnt0 = 0x0F70;
constexpr int kWaitVmcnt2 = 0x0F72;
constexpr int kWaitVmcnt4 = 0x0F74;
constexpr int kWaitLgkmcnt0 = 0xC07F;

}  // namespace
}  // namespace cs
