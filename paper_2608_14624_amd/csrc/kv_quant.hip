// Quantising a KV cache and reading it back, for gfx950: the write-back of new tokens into a pool
// of 4- or 8-bit tiles (quant_tile.h), and whole blocks from a bf16 pool to such a pool and back.
//
//   e    = smallest exponent for which max |x_i| / 2^e over a group of 32 features does not
//          round past the format's largest number
//   code = x_i / 2^e to the nearest number, ties to even; value = number * 2^e
//
// Every byte is read and written once: HBM bound.  A lane holds 8 features of a row, so four
// neighbouring lanes hold a group and find its largest magnitude with two DPP moves.  A wave
// takes the 16 rows of one (block, KV head, K or V): lane l's rows are those of V's layout,
// consecutive keys, whose codes are then one run of bytes.
//
// The bf16 side, four or two times the bytes of the other, goes past the caches: non-temporal
// loads of what is quantised and stores of what is read back.  us of a call of each, there and
// back, with ordinary accesses and so: 16 prompts of 129-2047 tokens, 8 heads of 128, 8 bits, 60 and 51 (264 MB,
// 5.1 TB/s); 3001 blocks of 8 heads of 64, 8 bits, 65 and 53 (5.6 TB/s); 4096 blocks of 8 heads of 128
// read back from 4 bits 75 and 52 (6.5 TB/s).
#include "internal.h"
#include "quant_tile.h"

namespace cs {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// How a wave's lanes share the 16 rows of a tile: kRowLanes lanes to a row, kRows rows to a lane,
// consecutive ones.
template <int D>
struct Rows {
  static constexpr int kRowLanes = D / 8;
  static constexpr int kRows = 16 * kRowLanes / 64;
  __device__ static __forceinline__ int first(int lane) { return lane / kRowLanes * kRows; }
  __device__ static __forceinline__ int part(int lane) { return lane % kRowLanes; }      // features 8 part ..
};

// largest of the four lanes of a group
__device__ __forceinline__ unsigned group_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));      // quad_perm 1 0 3 2
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));      // quad_perm 2 3 0 1
  return x;
}

// A lane's 8 features as codes (8 or 4 bytes) and its group's scale byte.
template <int D, int kBits>
__device__ __forceinline__ u32x2 quantise(u32x4 x, int& byte) {
  u16x2 m = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
  const unsigned top = group_max(max((unsigned)m[0], (unsigned)m[1]));
  byte = scale_byte<D, kBits>(top);
  if (byte == kNanScale) return u32x2{0, 0};
  const float scale = scale_of(byte);
  if constexpr (kBits == 4) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[3]), scale, 3);
    return u32x2{c, 0};
  } else {
    // (this conversion makes NaN of what is past 448, where the 4-bit one saturates: only bf16's
    // topmost numbers are, at the largest scale)
    if (top > 0x7f68u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u16x2 a = __builtin_elementwise_min(__builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu), u16x2{0x7f60, 0x7f60});
        x[i] = (x[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, a);
      }
    }
    i16_pair lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, as_pair(x[0]), scale, false);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, as_pair(x[1]), scale, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, as_pair(x[2]), scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, as_pair(x[3]), scale, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

// One row's 8 features of lane part `part` into row `key` of a tile.
template <int D, int kBits>
__device__ __forceinline__ void store_row(uint8_t* tile, bool is_v, int key, int part, u32x2 c, int byte) {
  using T = QuantTile<D, kBits>;
  if (!is_v) {
    uint8_t* at = tile + key * T::kRowBytes + part * kBits;
    if constexpr (kBits == 4) *reinterpret_cast<uint32_t*>(at) = c[0];
    else *reinterpret_cast<u32x2*>(at) = c;
    if (part % 4 == 0) tile[T::kKScales + key * T::kGroups + part / 4] = (uint8_t)byte;
    return;
  }
  if constexpr (D == 128) {
    uint8_t* at = tile + T::kV + (part * 16 + key) * T::kPartBytes;
    if constexpr (kBits == 4) *reinterpret_cast<uint32_t*>(at) = c[0];
    else *reinterpret_cast<u32x2*>(at) = c;
  } else {
    // the 8 features are two groups of V's layout
    uint8_t* at = tile + T::kV + (2 * part * 16 + key) * T::kPartBytes;
    if constexpr (kBits == 4) {
      *reinterpret_cast<uint16_t*>(at) = (uint16_t)c[0];
      *reinterpret_cast<uint16_t*>(at + 16 * T::kPartBytes) = (uint16_t)(c[0] >> 16);
    } else {
      *reinterpret_cast<uint32_t*>(at) = c[0];
      *reinterpret_cast<uint32_t*>(at + 16 * T::kPartBytes) = c[1];
    }
  }
  if (part % 4 == 0) tile[T::kVScales + part / 4 * 16 + key] = (uint8_t)byte;
}

// New tokens: a wave takes 16 tokens of one KV head, K or V.
template <int D, int kBits>
__global__ __launch_bounds__(kThreads) void kv_write_quant_kernel(QuantCopyLaunch a) {
  using R = Rows<D>;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int h = (int)(unit / 2 % a.num_kv_heads);
  const long long tile = unit / 2 / a.num_kv_heads;
  const bool is_v = unit & 1;
  const uint16_t* src = is_v ? a.v : a.k;
  const int part = R::part(lane);
  u32x4 x[R::kRows];
  int slot[R::kRows];
#pragma unroll
  for (int i = 0; i < R::kRows; ++i) {
    const long long t = tile * 16 + R::first(lane) + i;
    slot[i] = -1;
    x[i] = u32x4{};
    if (t >= a.n) continue;
    slot[i] = a.ids[t];
    const uint16_t* row = src + ((size_t)t * a.num_kv_heads + h) * D;
    x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + 8 * part));
  }
#pragma unroll
  for (int i = 0; i < R::kRows; ++i) {
    int byte;
    const u32x2 c = quantise<D, kBits>(x[i], byte);
    if (slot[i] < 0) continue;
    uint8_t* to = a.pool + ((size_t)(slot[i] >> 4) * a.num_kv_heads + h) * QuantTile<D, kBits>::kBytes;
    store_row<D, kBits>(to, is_v, slot[i] & 15, part, c, byte);
  }
}

// Whole blocks of a bf16 pool: a wave takes one (block, KV head), K or V.
template <int D, int kBits>
__global__ __launch_bounds__(kThreads) void kv_quantize_kernel(QuantCopyLaunch a) {
  using R = Rows<D>;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int h = (int)(unit / 2 % a.num_kv_heads);
  const long long i = unit / 2 / a.num_kv_heads;
  if (i >= a.n) return;
  const bool is_v = unit & 1;
  const uint16_t* src = (is_v ? a.v : a.k) + ((size_t)a.ids[i] * a.num_kv_heads + h) * 16 * D;
  uint8_t* to = a.pool + ((size_t)a.pool_ids[i] * a.num_kv_heads + h) * QuantTile<D, kBits>::kBytes;
  const int part = R::part(lane);
  u32x4 x[R::kRows];
#pragma unroll
  for (int k = 0; k < R::kRows; ++k)
    x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (R::first(lane) + k) * D + 8 * part));
#pragma unroll
  for (int k = 0; k < R::kRows; ++k) {
    int byte;
    const u32x2 c = quantise<D, kBits>(x[k], byte);
    store_row<D, kBits>(to, is_v, R::first(lane) + k, part, c, byte);
  }
}

// Whole blocks back: as above, the other way.
template <int D, int kBits>
__global__ __launch_bounds__(kThreads) void kv_dequantize_kernel(QuantCopyLaunch a) {
  using R = Rows<D>;
  using T = QuantTile<D, kBits>;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int h = (int)(unit / 2 % a.num_kv_heads);
  const long long i = unit / 2 / a.num_kv_heads;
  if (i >= a.n) return;
  const bool is_v = unit & 1;
  const uint8_t* tile = a.pool + ((size_t)a.pool_ids[i] * a.num_kv_heads + h) * T::kBytes;
  uint16_t* to = (is_v ? a.v_out : a.k_out) + ((size_t)a.ids[i] * a.num_kv_heads + h) * 16 * D;
  const int part = R::part(lane);
  u32x2 c[R::kRows];
  int byte[R::kRows];
#pragma unroll
  for (int k = 0; k < R::kRows; ++k) {
    const int key = R::first(lane) + k;
    c[k] = u32x2{};
    if (!is_v) {
      const uint8_t* at = tile + key * T::kRowBytes + part * kBits;
      if constexpr (kBits == 4) c[k][0] = *reinterpret_cast<const uint32_t*>(at);
      else c[k] = *reinterpret_cast<const u32x2*>(at);
      byte[k] = tile[T::kKScales + key * T::kGroups + part / 4];
    } else {
      if constexpr (D == 128) {
        const uint8_t* at = tile + T::kV + (part * 16 + key) * T::kPartBytes;
        if constexpr (kBits == 4) c[k][0] = *reinterpret_cast<const uint32_t*>(at);
        else c[k] = *reinterpret_cast<const u32x2*>(at);
      } else {
        const uint8_t* at = tile + T::kV + (2 * part * 16 + key) * T::kPartBytes;
        if constexpr (kBits == 4)
          c[k][0] = *reinterpret_cast<const uint16_t*>(at) |
                    (uint32_t)*reinterpret_cast<const uint16_t*>(at + 16 * T::kPartBytes) << 16;
        else
          c[k] = u32x2{*reinterpret_cast<const uint32_t*>(at),
                       *reinterpret_cast<const uint32_t*>(at + 16 * T::kPartBytes)};
      }
      byte[k] = tile[T::kVScales + part / 4 * 16 + key];
    }
  }
#pragma unroll
  for (int k = 0; k < R::kRows; ++k) {
    const float scale = scale_of(byte[k]);
    u32x4 x;
#pragma unroll
    for (int p = 0; p < 4; ++p) x[p] = read_pair<kBits>(c[k][kBits == 4 ? 0 : p / 2], scale, kBits == 4 ? p : p % 2);
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to + (R::first(lane) + k) * D + 8 * part));
  }
}

template <template <int, int> class F>
hipError_t by_format(int head_dim, int bits, const QuantCopyLaunch& a, long long units, hipStream_t stream) {
  const dim3 grid((unsigned)((units + kWaves - 1) / kWaves)), block(kThreads);
  if (head_dim == 64) {
    if (bits == 4) hipLaunchKernelGGL((F<64, 4>::kernel), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((F<64, 8>::kernel), grid, block, 0, stream, a);
  } else {
    if (bits == 4) hipLaunchKernelGGL((F<128, 4>::kernel), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((F<128, 8>::kernel), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

template <int D, int kBits>
struct Write {
  static constexpr auto kernel = kv_write_quant_kernel<D, kBits>;
};
template <int D, int kBits>
struct Quantize {
  static constexpr auto kernel = kv_quantize_kernel<D, kBits>;
};
template <int D, int kBits>
struct Dequantize {
  static constexpr auto kernel = kv_dequantize_kernel<D, kBits>;
};

}  // namespace

long long quant_tile_bytes(int head_dim, int bits) {
  return 2LL * 16 * (head_dim * bits / 8 + head_dim / kScaleGroup);
}

bool quant_copy_fits(long long n, int num_kv_heads, bool tokens) {
  const double units = 2.0 * num_kv_heads * (double)(tokens ? (n + 15) / 16 : n);
  return launch_fits((units + kWaves) / kWaves, kThreads);
}

hipError_t launch_kv_write_quant(const QuantCopyLaunch& a, hipStream_t stream) {
  return by_format<Write>(a.head_dim, a.bits, a, 2LL * a.num_kv_heads * ((a.n + 15LL) / 16), stream);
}

hipError_t launch_kv_quantize(const QuantCopyLaunch& a, hipStream_t stream) {
  return by_format<Quantize>(a.head_dim, a.bits, a, 2LL * a.num_kv_heads * a.n, stream);
}

hipError_t launch_kv_dequantize(const QuantCopyLaunch& a, hipStream_t stream) {
  return by_format<Dequantize>(a.head_dim, a.bits, a, 2LL * a.num_kv_heads * a.n, stream);
}

}  // namespace cs
