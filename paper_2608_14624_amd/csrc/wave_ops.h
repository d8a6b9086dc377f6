// Wave-wide helpers of the kernels that plan their own work.
#pragma once

#include <hip/hip_runtime.h>

#include <math.h>

namespace cs {
namespace {

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// inclusive prefix sum over the 64 lanes (DPP: shifts within rows of 16, then
// row 15 and row 31 broadcasts; lanes without a source add 0)
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return x;
}

// largest of the 64 lanes' values, none of them negative
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

// A reference for the logits of a row that has seen no key, in softmaxes of exp2(c (s - m)) with
// c > 0: about the lowest m for which m and m c are finite, so that masked logits (-inf) weigh 0
// and not NaN.  -FLT_MAX / c itself will not do: it is rounded, and times c it is infinite for one
// c in seven above 1.  Both roundings are off by at most 2^-24 of the value, and the number here is
// about 2^-21 (eight times that) below FLT_MAX.
__host__ __device__ inline float lowest_reference(float c) { return -0x1.fffffp127f / fmaxf(c, 1.f); }

}  // namespace
}  // namespace cs
