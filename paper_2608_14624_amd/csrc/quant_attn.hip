// Attention over a KV pool held in 4 or 8 bits, for gfx950: decode (one token per sequence) and
// prefill (suffix rows over a prefix and their own keys).
//
//   out = sum_j softmax_j(scale * q . K_j) V_j,   K, V the values of the pool's codes
//
// With S^T = K Q^T and O^T = V^T P^T, S^T leaves the matrix unit in the very registers that P^T
// enters it from: a lane's keys of S^T are the ones it is to supply of P^T, in the order that the
// V^T operand takes them in too, and the tile's layout (quant_tile.h) gives K and V to the lanes
// that need them.  Decode works on 16 rows (the heads of a KV head), each wave on
// keys of its own; prefill works on 32 rows a wave and shares conversions through LDS.
// K and V are converted to bf16, V two features of a key at a time, which two byte permutes then pair
// up by keys.  The unit's products of 4- and 8-bit codes (v_mfma_scale_f32_*_f8f6f4) would take K as it
// is, but where an operand is E4M3 they sum the 32 products of a group without what lies 2^14 below the
// largest of them: with Q in two E4M3 parts, logits beside a product of 4096 were off by 0.1.  Q in four E2M3
// parts, whose sums with E2M1 codes are exact, takes as long as the conversions (4 x 512 rows on 4096 keys,
// 64 / 8 heads of 128, 4 bits: 260 us and 264; with the two E4M3 parts 242).
//
// The reference that the exponentials are relative to follows the logits only when the weights of a
// lane's keys have become 2^16 times as large as it left them: bf16 holds numbers of any size, and most
// steps rescale nothing, look for no maximum and exchange nothing between lanes.
#include "decode_common.h"
#include "internal.h"
#include "quant_tile.h"

#include <math.h>

#include <type_traits>

namespace cs {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;             // of a work-group, both kernels
constexpr int kThreads = 64 * kWaves;
// The sum of a lane's weights of 32 keys at which their reference moves, and how far above the largest
// logit it goes then.  A row's weights of n keys add up to n / 8 * kLargeSum at most, below 1 for every
// length, so that O, which is relative to the same reference, holds what V holds, up to 448 * 2^119.  (Weights
// up to 2^16 took sums past float32 from V's of 2^112 on.)  The price is at the other end: weights of
// 2^-45 on leave 2^-126 for V's below 2^-64 to lose bits in.
constexpr float kLargeSum = 0x1p-28f;
constexpr float kReferenceAbove = 44.f;
// Past this a reference is no longer a whole number of any size, and a logit's product with the scale,
// which the weights take unrounded, may be off the rounded one that the reference was found from by more
// than float32's exponents: from 2^31 on the largest logit would weigh 2^128 or 2^-128
constexpr float kFarReference = 0x1p24f;
// The reference of rows that have seen no key: about the lowest number, so that masked logits
// (-inf) weigh 0 and not NaN, and every other one is above it
constexpr float kLowest = -0x1.fffffp127f;

struct QuantParams {
  const uint16_t* q;
  const uint8_t* pool;
  const int32_t* block_tables;
  const int32_t* lens;
  const int32_t* cu_q_lens;
  uint16_t* out;
  int batch;
  int max_blocks_per_seq;
  int num_q_heads;
  int num_kv_heads;
  int group;
  float scale_log2;
  float* ws_o;
  float* ws_ml;
  int ranges;               // decode: work-groups per KV head
  long long rows;           // partial results per query head
  int parts;                // prefill: key parts
  int tiles;
  int total_q;
};

// ---------------------------------------------------------------------------
// Query rows

// 16 rows as the B operand: lane l holds row l & 15 (`row`, null: zeros), quarter l >> 4.
template <int D>
struct Rows16 {
  bf16x8 q[D / 32];
  __device__ __forceinline__ void load(const uint16_t* row, int lane) {
    // step s of the contracted index: features (D / 4) qd + 8 s .. + 7, as K's lanes hold them
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      q[s] = bf16x8{};
      if (row != nullptr) q[s] = *reinterpret_cast<const bf16x8*>(row + D / 4 * (lane >> 4) + 8 * s);
    }
  }
};

// 32 rows as the B operand of 32 x 32 products: lane l holds row l & 31, half l >> 5.
template <int D>
struct Rows32 {
  bf16x8 q[D / 16];
  __device__ __forceinline__ void load(const uint16_t* row, int lane) {
    // step s of the contracted index: features (D / 2) half + 8 s .. + 7, as K's lanes take them
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      q[s] = bf16x8{};
      if (row != nullptr) q[s] = *reinterpret_cast<const bf16x8*>(row + D / 2 * (lane >> 5) + 8 * s);
    }
  }
};

// ---------------------------------------------------------------------------
// Keys

// The codes and scales of a block's 16 keys as a lane needs them.
template <int D, int kBits>
struct Block {
  using T = QuantTile<D, kBits>;
  static constexpr int kKWords = D / 4 * kBits / 32;           // a lane's codes of K, in words
  static constexpr int kVWords = T::kPartBytes;                // of V: 4 keys of kPartBytes
  uint32_t k[kKWords];
  uint32_t v[kVWords];
  int ks;
  uint32_t vs;

  template <int kPolicy, int kWords>
  __device__ __forceinline__ static void load_words(uint32_t (&to)[kWords], __amdgpu_buffer_rsrc_t rs, int off) {
    if constexpr (kWords == 2) {
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, kPolicy));
      to[0] = x[0];
      to[1] = x[1];
    } else {
#pragma unroll
      for (int w = 0; w < kWords; w += 4) {
        const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off + 4 * w, 0, kPolicy));
#pragma unroll
        for (int i = 0; i < 4; ++i) to[w + i] = x[i];
      }
    }
  }

  // Block `id` of the KV head whose tiles `base` starts at, `stride` bytes apart.  The
  // descriptor of a negative id is empty: zeros, and nothing outside the pool is read.
  __device__ __forceinline__ static __amdgpu_buffer_rsrc_t tile(const uint8_t* base, size_t stride, int id) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)id * stride), (short)0, id < 0 ? 0 : T::kBytes,
                                             kRawBufferWord3);
  }
  template <int kPolicy = 0>
  __device__ __forceinline__ void load_keys(__amdgpu_buffer_rsrc_t rs, int lane) {
    const int key = lane & 15, qd = lane >> 4;
    const int k_off = key * T::kRowBytes + T::kRowBytes / 4 * qd;
    const int ks_off = T::kKScales + key * T::kGroups + qd * T::kGroups / 4;
    load_words<kPolicy>(k, rs, k_off);
    ks = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_off, 0, 0);
  }
  template <int kPolicy = 0>
  __device__ __forceinline__ void load_values(__amdgpu_buffer_rsrc_t rs, int lane) {
    const int c = lane & 15, qd = lane >> 4;
    load_words<kPolicy>(v, rs, T::kV + (c * 16 + 4 * qd) * T::kPartBytes);
    vs = __builtin_amdgcn_raw_buffer_load_b32(rs, T::kVScales + c * T::kPart / kScaleGroup * 16 + 4 * qd, 0, 0);
  }

  // The same by whole lines, where a key's codes, and those of a group of V, are lines of 128 bytes: lane
  // l holds bytes 16 (l % 8) .. + 15 of lines l / 8 and 8 + l / 8 of K and of V, until `arrange`.  (The
  // loads above have 16 neighbouring lanes take 16 bytes of as many lines, and a compute unit then
  // reads 16 bytes a clock.  us a call: the 61 sequences of the decode's comment 96 so and 65 by lines, the
  // 128 at 8 bits 350 and 320.  With rows of 64 bytes there was nothing to gain.)
  static constexpr bool kLines = T::kRowBytes == 128;
  template <int kPolicy = 0>
  __device__ __forceinline__ void load_lines(__amdgpu_buffer_rsrc_t rs, int lane) {
    const int key = lane & 15, qd = lane >> 4;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const u32x4 a = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, 1024 * w + 16 * lane, 0, kPolicy));
      const u32x4 b = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, T::kV + 1024 * w + 16 * lane, 0, kPolicy));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k[4 * w + i] = a[i];
        v[4 * w + i] = b[i];
      }
    }
    ks = __builtin_amdgcn_raw_buffer_load_b8(rs, T::kKScales + key * T::kGroups + qd, 0, 0);
    vs = __builtin_amdgcn_raw_buffer_load_b32(rs, T::kVScales + key / 4 * 16 + 4 * qd, 0, 0);
  }
  // ... through 4096 bytes of LDS that only this wave uses (its accesses are in order).  Chunk c of line
  // r stands at c ^ (r & 7), so that eight lanes' chunks are in different banks both ways.
  __device__ __forceinline__ void arrange(uint8_t* lds, int lane) {
    uint8_t* to = lds + lane / 8 * 128 + (lane % 8 ^ lane / 8) * 16;
    const int from = (lane & 15) * 128 + (2 * (lane >> 4) ^ (lane & 7)) * 16;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      *reinterpret_cast<u32x4*>(to + 1024 * w) = u32x4{k[4 * w], k[4 * w + 1], k[4 * w + 2], k[4 * w + 3]};
      *reinterpret_cast<u32x4*>(to + 2048 + 1024 * w) = u32x4{v[4 * w], v[4 * w + 1], v[4 * w + 2], v[4 * w + 3]};
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(lds + (from ^ 16 * w));
      const u32x4 b = *reinterpret_cast<const u32x4*>(lds + 2048 + (from ^ 16 * w));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k[4 * w + i] = a[i];
        v[4 * w + i] = b[i];
      }
    }
  }

  // What stands behind `n` keys of the block is not the sequence's: V there becomes zero (its
  // weights are 0, but 0 times a NaN is NaN).
  __device__ __forceinline__ void cut_values(int n, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * (lane >> 4) + i >= n) {
        vs = (vs & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
        // (key i's codes: kPartBytes of them)
        if constexpr (T::kPartBytes == 2) {
          v[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
        } else {
#pragma unroll
          for (int w = 0; w < T::kPartBytes / 4; ++w) v[i * (T::kPartBytes / 4) + w] = 0;
        }
      }
  }

  // The lane's features 8 i .. + 7 of its key as bf16
  __device__ __forceinline__ u32x4 key_features(int i, float scale) const {
    if constexpr (kBits == 4) {
      return u32x4{read_pair<4>(k[i], scale, 0), read_pair<4>(k[i], scale, 1), read_pair<4>(k[i], scale, 2),
                   read_pair<4>(k[i], scale, 3)};
    } else {
      return u32x4{read_pair<8>(k[2 * i], scale, 0), read_pair<8>(k[2 * i], scale, 1),
                   read_pair<8>(k[2 * i + 1], scale, 0), read_pair<8>(k[2 * i + 1], scale, 1)};
    }
  }

  // S^T of the block's keys and 16 rows: lane l has row l & 15 and keys 4 (l >> 4) .. + 3
  __device__ __forceinline__ f32x4 logits(const Rows16<D>& rows) const {
    f32x4 s = f32x4{};
    const float scale = scale_of(ks);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, key_features(i, scale)), rows.q[i], s, 0,
                                                  0, 0);
    return s;
  }

  // The lane's four keys' features kPart c + t (c = l & 15), t = 2 pair in f[0] and 2 pair + 1 in
  // f[1]: half of a V^T fragment
  __device__ __forceinline__ void values(int pair, const float (&scale)[4], u32x2 (&f)[2]) const {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kBits == 4) {
        const int byte = i * T::kPartBytes + pair;       // of the lane's codes
        x[i] = read_pair<4>(v[byte / 4], scale[i], byte % 4);
      } else {
        const int half = i * T::kPartBytes / 2 + pair;
        x[i] = read_pair<8>(v[half / 2], scale[i], half % 2);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f[0][i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
      f[1][i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
    }
  }

  __device__ __forceinline__ void value_scales(float (&scale)[4]) const {
    scale[0] = __builtin_bit_cast(float, (vs & 0xffu) << 23);
    scale[1] = __builtin_bit_cast(float, (vs & 0xff00u) << 15);
    scale[2] = __builtin_bit_cast(float, (vs & 0xff0000u) << 7);
    scale[3] = __builtin_bit_cast(float, (vs & 0xff000000u) >> 1);
  }
};

// 32 keys: two blocks, whose halves of a V^T fragment make one
template <int D, int kBits>
struct Unit {
  Block<D, kBits> b[2];
  // kOnce: no other sequence is known to read the blocks, so they need not stay in the caches
  template <bool kOnce>
  __device__ __forceinline__ void load(const uint8_t* base, size_t stride, int id0, int id1, int lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __amdgpu_buffer_rsrc_t rs = Block<D, kBits>::tile(base, stride, i ? id1 : id0);
      if constexpr (Block<D, kBits>::kLines) {
        b[i].template load_lines<kOnce ? kNonTemporal : 0>(rs, lane);
      } else {
        b[i].template load_keys<kOnce && kBits == 4 ? kNonTemporal : 0>(rs, lane);
        b[i].template load_values<kOnce ? kNonTemporal : 0>(rs, lane);
      }
    }
  }
  // `lds`: kArea bytes that only this wave uses
  static constexpr int kArea = Block<D, kBits>::kLines ? 2 * 4096 : 0;
  __device__ __forceinline__ void arrange(uint8_t* lds, int lane) {
    if constexpr (Block<D, kBits>::kLines) {
      b[0].arrange(lds, lane);
      b[1].arrange(lds + 4096, lane);
    }
  }
  __device__ __forceinline__ void cut_values(int n, int lane) {
    b[0].cut_values(n, lane);
    b[1].cut_values(n - 16, lane);
  }
};

// ---------------------------------------------------------------------------
// The softmax of a tile's rows over the keys seen so far, the rows 16 (a lane has four keys of
// every block) or 32 (eight).  l is of the lane's own keys.  Weights are 2^(s c - m) with m a
// whole number, so that moving m is exact.
template <int kRows>
struct Softmax {
  typedef float Logits __attribute__((ext_vector_type(kRows / 2)));       // of 32 keys
  float m = kLowest, l = 0.f;
  float limit = -1.f;       // kLargeSum, or below every sum while a row's m is past kFarReference; the wave's

  // Logits from .. to - 1 as weights, rounded to bf16 as operands; sum and theirs
  __device__ __forceinline__ float weigh(const Logits& s, float c, bf16x8 (&p)[kRows / 16], float sum = 0.f,
                                         int from = 0, int to = kRows / 2) const {
#pragma unroll
    for (int i = from; i < to; i += 2) {
      bf16_pair e;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        e[k] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i + k], c, -m));
        p[i / 8][i % 8 + k] = e[k];
      }
      sum = __builtin_amdgcn_fdot2_f32_bf16(e, bf16_pair{(__bf16)1.f, (__bf16)1.f}, sum, false);
    }
    return sum;
  }

  // Adds the weights p of logits s to l, by their sum; where one is too large (the sum finds it as
  // well as a maximum would, and is needed) m moves to its place above the largest logit, what there is
  // so far (o) with it, and the weights are made anew.  Rows with a reference that is far from 0 always
  // come here: their weights are of the rounded products.
  template <int kWords, typename O>
  __device__ __forceinline__ void add(float sum, const Logits& s, float c, O (&o)[kWords], bf16x8 (&p)[kRows / 16]) {
    if (__builtin_amdgcn_ballot_w64(sum > limit) != 0) {
      float top = s[0];
#pragma unroll
      for (int i = 1; i < kRows / 2; ++i) top = fmaxf(top, s[i]);
      float a, b;
      swap32(top, a, b);
      top = kRows == 16 ? quad_max(top) : fmaxf(a, b);
      const float m_new = fmaxf(m, ceilf(top * c) + kReferenceAbove);
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < kWords; ++t) o[t] *= alpha;
      sum = weigh(s, c, p);
      const bool is_far = fabsf(m) > kFarReference;
      limit = kLargeSum;
      if (__builtin_amdgcn_ballot_w64(is_far) != 0) {
#pragma clang fp contract(off)
        limit = -1.f;
        float far_sum = 0.f;
#pragma unroll
        for (int i = 0; i < kRows / 2; ++i) {
          const float x = s[i] * c;
          const __bf16 e = (__bf16)__builtin_amdgcn_exp2f(x - m);
          if (is_far) p[i / 8][i % 8] = e;
          far_sum += (float)e;
        }
        if (is_far) sum = far_sum;
      }
    }
    l += sum;
  }
};

// A unit's keys added to 16 rows, V converted as it is needed (decode); of the keys the rows see the
// first `seen`.  Lane l has of row l & 15 O's features D / 4 qd + D / 16 r + t in o[t][r].
template <int D, int kBits>
__device__ __forceinline__ void add_unit(Softmax<16>& soft, f32x4 (&o)[D / 16], const Unit<D, kBits>& u,
                                         const Rows16<D>& rows, float c, int seen, int lane) {
  Softmax<16>::Logits s;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const f32x4 x = u.b[b].logits(rows);
#pragma unroll
    for (int r = 0; r < 4; ++r) s[4 * b + r] = x[r];
  }
  if (seen < kUnitKeys) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 16 * (i / 4) + 4 * (lane >> 4) + i % 4 < seen ? s[i] : -INFINITY;
  }
  bf16x8 p[1];
  const float sum = soft.weigh(s, c, p);
  soft.add(sum, s, c, o, p);
  float scale[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) u.b[b].value_scales(scale[b]);
#pragma unroll
  for (int t = 0; t < D / 16; t += 2) {
    u32x2 f[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) u.b[b].values(t / 2, scale[b], f[b]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 a = {f[0][i][0], f[0][i][1], f[1][i][0], f[1][i][1]};
      o[t + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p[0], o[t + i], 0, 0, 0);
    }
  }
}

// ---------------------------------------------------------------------------
// Decode.  The batch's keys are counted in units of 32 and dealt to `ranges` work-groups per KV
// head in equal contiguous ranges.  A work-group's waves take the units of a piece (a sequence's
// part of the range) in turn and merge in LDS; a sequence cut over several ranges leaves partial
// results (O relative to m, m, and l) that a second kernel merges.  Bound by HBM: 128 sequences of 4.2k-10.8k
// keys, 32 / 8 heads of 128, take 173 us at 4 bits (1.08 GB, 6.2 TB/s), 320 at 8 (6.5).  Where sequences
// share anchors, by conversions and products: 64 / 8 heads, 61 sequences, 8 bits, 65 us (73 where the caches
// are cold), of which all but the loads 52; with every anchor in L2 61.

__device__ __forceinline__ int total_units(const QuantParams& p, int lane) {
  int total = 0;
  for (int s = 0; s < p.batch; s += 64) total += wave_total(s + lane < p.batch ? units_of(p.lens[s + lane]) : 0);
  return total;
}

__device__ __forceinline__ int units_per_range(const QuantParams& p, int total) {
  return max((int)(((unsigned)total + p.ranges - 1) / (unsigned)p.ranges), kWaves);
}

template <int D>
struct DecodeLds {
  float o[kWaves][kMaxGroup][D + 4];
  float2 ml[kWaves][kMaxGroup];
};

// How many sequences hold the block at index 31 that the one before them holds: a batch's agents'
// sequences usually stand together, and a prefix that short is not worth asking for.  Where they do not
// stand together their blocks are loaded as read once.  us a call by agents and in random order: the 61
// sequences of 4 agents below, three states in turn, 79 and 84 at 8 bits, 51 and 52 at 4; 128 of 8 agents, 32 / 8
// heads of 64, 8 bits, 60 and 65.  Asking for every pair among 64 sequences took 10 us more in any order.
constexpr int kProbeBlock = 31;
__device__ __forceinline__ int count_sharing(const QuantParams& p, int lane) {
  int count = 0;
  for (int s = 0; s < p.batch; s += 63) {      // (lane 0: the sequence before the 63)
    const int i = s + lane - 1;
    int id = -1 - lane;
    if (i >= 0 && i < p.batch && p.lens[i] > kProbeBlock * kBlock)
      id = p.block_tables[(size_t)i * p.max_blocks_per_seq + kProbeBlock];
    const int last = __shfl_up(id, 1);
    count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane > 0 && id == last));
  }
  return count;
}

// Units that a wave's registers hold, one of them being attended while the others are on their way,
// and work-groups per compute unit, to which a decode's keys are dealt: all run at once.  us a call
// of 128 sequences of 4.2k-10.8k keys, 32 / 8 heads of 128, at 4 bits: 4 units and 2 work-groups 175, 3 and 2
// 177, 6 and 2 178, 2 and 3 179, 3 and 3 183; at 8 bits 3 and 2 320, 2 and 2 320, 2 and 3 336.
constexpr int decode_depth(int head_dim, int bits) { return head_dim == 128 && bits == 8 ? 3 : 4; }
constexpr int kDecodeGroupsPerCu = 2;
// Blocks are loaded as read once (non-temporal) unless at least one sequence in kSharingPart shares
// them, in launches of at least kSharedUnits units a work-group; in smaller ones the answer is not worth
// waiting for.  us a call so and with ordinary loads: those 128 sequences at 4 bits 173 and 200, at 8 bits 320 and
// 363; 61 sequences of 4 agents with 4096 shared keys and 100-3000 of their own, 64 / 8 heads, 52 and 49 at 4
// bits, 84 and 65 at 8.  (Pieces cut at the same positions of all sequences, dealt so that the
// work-groups that run at one time share them, raised the L2's hits from 49% to 68% there, but took 108 us
// where 96 had been.)
constexpr int kSharingPart = 4;
constexpr int kSharedUnits = 16;

template <int D, int kBits>
__global__ __launch_bounds__(kThreads, kDecodeGroupsPerCu) void quant_decode_kernel(QuantParams p) {
  constexpr int kDepth = decode_depth(D, kBits);
  using T = QuantTile<D, kBits>;
  __shared__ DecodeLds<D> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // a wave's part of `o`, which it writes after its last unit, and others read between two barriers
  static_assert(sizeof(sm.o[0]) >= Unit<D, kBits>::kArea, "a unit is arranged there");
  uint8_t* area = reinterpret_cast<uint8_t*>(sm.o[wave]);
  const int g = blockIdx.x % p.num_kv_heads;
  const int w = blockIdx.x / p.num_kv_heads;
  const ScalarInts lens = (ScalarInts)p.lens;
  const int total = total_units(p, lane);
  const int per = units_per_range(p, total);
  if ((long long)w * per >= total) return;
  const int u0 = w * per;
  int left = min(per, total - u0);
  // the sequence that holds unit u0
  int r = 0, x = 0;
  {
    int first = 0;
    for (int s = 0;; s += 64) {
      const int n = s + lane < p.batch ? units_of(p.lens[s + lane]) : 0;
      const int incl = wave_scan(n);
      const unsigned long long past = __builtin_amdgcn_ballot_w64(first + incl > u0);
      if (past != 0) {
        const int at = __builtin_ctzll(past);
        r = s + at;
        x = u0 - first - __builtin_amdgcn_readlane(incl - n, at);
        break;
      }
      first += __builtin_amdgcn_readlane(incl, 63);
    }
  }
  const size_t stride = (size_t)p.num_kv_heads * T::kBytes;
  const uint8_t* base = p.pool + (size_t)g * T::kBytes;
  const int j = lane & 15;
  const float c = p.scale_log2;
  const bool shared = total >= kSharedUnits * p.ranges && p.batch > 1 && p.max_blocks_per_seq > kProbeBlock &&
                      kSharingPart * count_sharing(p, lane) >= p.batch;
  auto run = [&](auto once) __attribute__((always_inline)) {
    constexpr bool kOnce = decltype(once)::value;
    for (;;) {
      const int len = lens[r];
      const int n = units_of(len);
      const int xe = min(n, x + left);
      const bool whole = x == 0 && xe == n;
      left -= xe - x;
      const ScalarInts table = (ScalarInts)(p.block_tables + (size_t)r * p.max_blocks_per_seq);
      const int last = (len - 1) / kBlock;
      Rows16<D> rows;
      rows.load(j < p.group ? p.q + ((size_t)r * p.num_q_heads + g * p.group + j) * D : nullptr, lane);
      Softmax<16> soft;
      f32x4 o[D / 16];
#pragma unroll
      for (int t = 0; t < D / 16; ++t) o[t] = f32x4{};
      Unit<D, kBits> ring[kDepth];
      int id0 = 0, id1 = 0;
      auto ids_of = [&](int unit) {
        id0 = table[kUnitBlocks * unit];
        id1 = table[min(kUnitBlocks * unit + 1, last)];
      };
      int y = x + wave;
      if (y < xe) ids_of(y);
#pragma unroll
      for (int d = 0; d < kDepth; ++d) {
        if (y + d * kWaves >= xe) break;
        ring[d].template load<kOnce>(base, stride, id0, id1, lane);
        if (y + (d + 1) * kWaves < xe) ids_of(y + (d + 1) * kWaves);
      }
      while (y < xe) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d, y += kWaves) {
          if (y >= xe) break;
          const int seen = len - y * kUnitKeys;
          ring[d].arrange(area, lane);
          if (seen < kUnitKeys) ring[d].cut_values(seen, lane);
          add_unit<D, kBits>(soft, o, ring[d], rows, c, seen, lane);
          if (y + kDepth * kWaves < xe) {
            ring[d].template load<kOnce>(base, stride, id0, id1, lane);
            if (y + (kDepth + 1) * kWaves < xe) ids_of(y + (kDepth + 1) * kWaves);
          }
        }
      }
      const float l = quad_sum(soft.l);
      if (j < p.group) {
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
          for (int t = 0; t < D / 16; t += 4)
            *reinterpret_cast<f32x4*>(&sm.o[wave][j][D / 4 * (lane >> 4) + D / 16 * rr + t]) =
                f32x4{o[t][rr], o[t + 1][rr], o[t + 2][rr], o[t + 3][rr]};
        if (lane < 16) sm.ml[wave][j] = make_float2(soft.m, l);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < p.group * (D / 4); i += kThreads) {
        const int hj = i / (D / 4), d = i % (D / 4) * 4;
        float m = sm.ml[0][hj].x;
#pragma unroll
        for (int k = 1; k < kWaves; ++k) m = fmaxf(m, sm.ml[k][hj].x);
        float den = 0.f;
        f32x4 acc = f32x4{};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
          const float wt = __builtin_amdgcn_exp2f(sm.ml[k][hj].x - m);
          den = __builtin_fmaf(wt, sm.ml[k][hj].y, den);
          const f32x4 o = *reinterpret_cast<const f32x4*>(&sm.o[k][hj][d]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(wt, o[e], acc[e]);
        }
        if (whole) {
          bf16x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[e] / den);
          *reinterpret_cast<uint2*>(p.out + ((size_t)r * p.num_q_heads + g * p.group + hj) * D + d) =
              __builtin_bit_cast(uint2, o);
        } else {
          const size_t at = ((size_t)g * p.rows + r + w) * p.group + hj;
          *reinterpret_cast<f32x4*>(p.ws_o + at * D + d) = acc;
          if (d == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * at) = make_float2(m, den);
        }
      }
      if (left <= 0) return;
      do ++r;
      while (lens[r] <= 0);
      x = 0;
      __syncthreads();
    }
  };
  if (shared) run(std::false_type{});
  else run(std::true_type{});
}

// One work-group per (sequence, KV head) merges what the ranges left of it.
template <int D>
__global__ __launch_bounds__(kMergeThreads) void quant_decode_merge_kernel(QuantParams p) {
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads;
  const int lane = threadIdx.x & 63;
  int total = 0, before = 0;
  for (int s = 0; s < p.batch; s += 64) {
    const int n = s + lane < p.batch ? units_of(p.lens[s + lane]) : 0;
    total += wave_total(n);
    before += wave_total(s + lane < r ? n : 0);
  }
  const int per = units_per_range(p, total);
  const int n = units_of(p.lens[r]);
  const int w0 = (unsigned)before / (unsigned)per;
  const int pieces = n == 0 ? 0 : (int)((unsigned)(before + n - 1) / (unsigned)per) - w0 + 1;
  if (pieces == 1) return;
  const size_t first = ((size_t)g * p.rows + r + w0) * p.group;
  merge_pieces<D>(
      p.ws_o, p.ws_ml, p.group, 1.f, [&](int) { return pieces; },
      [&](int hj, int k) { return first + (size_t)k * p.group + hj; },
      [&](int hj, int d, bf16x4 o) {
        *reinterpret_cast<uint2*>(p.out + ((size_t)r * p.num_q_heads + g * p.group + hj) * D + d) =
            __builtin_bit_cast(uint2, pieces == 0 ? bf16x4{} : o);
      });
}

// ---------------------------------------------------------------------------
// Prefill.  Rows of a KV head are (token, query head of it), heads fastest; a wave takes 32 of them,
// or at D = 64, where the launch fills the device so, 64 (kTiles).  A work-group's steps are 64
// keys: each wave reads one of the four blocks ahead into registers, and a step later leaves it in
// LDS as all waves then take it, K and V as bf16 fragments, so that a conversion is done once for the
// work-group's rows.  A step's buffer is written while the other one is read: one barrier a step.
//
// Within a wave the logits of the next 32 keys, the weights of the present ones and the values of the
// last 32 stand side by side, so that the matrix unit's work does not depend on the vector unit's.
// Several parts of a tile's keys on as many work-groups leave partial results.
//
// us a call: 64 / 8 heads of 128, 4 x (4096 + 512), 264 at 4 bits (1.11 PFLOP/s; a large bf16 product of
// the library reaches 1.24), 286 at 8; heads of 64 149 and 152; 32 / 8 heads, 16 ragged invocations, 8 bits
// 1005 (0.93).
// Bound by the step's own work: the 264 are 249 without the exponentials, 225 without the conversions and
// their stores, 215 without LDS reads, and 203 without the products.  Each wave converting all for itself
// took 317 and 2850; 16 x 16 products, three waves a SIMD and, at D = 128, 64 rows a wave (O in
// accumulation registers) were as fast or slower; loads one more step ahead, the rows' all at once, and K's
// fragments read a chunk ahead like V's are within 1% both ways.  Of a small launch
// (83 rows x 32 / 8 heads on 3094 keys, 21 us in this kernel) a wave alone on its SIMD takes 1.3 us a
// step, 6 to get to the second step, and 4 to store its partial results.

constexpr int kStepBlocks = kWaves;
constexpr int kStepKeys = 16 * kStepBlocks;

// What a step's buffer holds: step x computes the logits of blocks 4 x + 2 .. 4 x + 5 and adds the
// values of blocks 4 x - 2 .. 4 x + 1.
template <int D, int kBits>
struct PrefillLds {
  // fragments of K, 16 keys, and of V^T
  u32x4 k[2][kStepBlocks][D / 32][64];
  u32x4 v[2][kStepBlocks][D / 32][64];
};

template <int D, int kBits, int kTiles>
__global__ __launch_bounds__(kThreads, kTiles == 1 ? 2 : 1) void quant_prefill_kernel(QuantParams p) {
  using T = QuantTile<D, kBits>;
  constexpr int kWaveRows = 32 * kTiles;
  constexpr int kTileRows = kWaves * kWaveRows;
  __shared__ PrefillLds<D, kBits> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ScalarInts prefix = (ScalarInts)p.lens;
  const ScalarInts cu = (ScalarInts)p.cu_q_lens;
  unsigned at = blockIdx.x;
  const int g = at % p.num_kv_heads;
  at /= p.num_kv_heads;
  const int part = at % p.parts;
  at /= p.parts;
  // an invocation's tiles one after another, those with the most keys first: the work-groups that
  // run at one time read few sequences' keys, which their L2 holds
  const int tile = p.tiles - 1 - at % p.tiles;
  const int r = at / p.tiles;
  const int q0 = cu[r];
  const int tokens = cu[r + 1] - q0;
  const unsigned group = p.group;
  const int n_rows = tokens * p.group;
  const int tile0 = tile * kTileRows;
  if (tile0 >= n_rows) return;
  const int before = prefix[r];
  const int len = before + tokens;
  // tokens of the wave's first and last row
  const int row0 = tile0 + wave * kWaveRows;
  const int t0 = (unsigned)min(row0, n_rows - 1) / group;
  const int t1 = (unsigned)(min(row0 + kWaveRows, n_rows) - 1) / group;
  // steps of the keys that the tile's rows see, this part's
  const int tile_t1 = (unsigned)(min(tile0 + kTileRows, n_rows) - 1) / group;
  const unsigned steps = (unsigned)(before + tile_t1) / kStepKeys + 1;
  const int x0 = steps * part / (unsigned)p.parts;
  const int xe = steps * (part + 1) / (unsigned)p.parts;

  const size_t stride = (size_t)p.num_kv_heads * T::kBytes;
  const uint8_t* base = p.pool + (size_t)g * T::kBytes;
  const float c = p.scale_log2;
  const ScalarInts table = (ScalarInts)(p.block_tables + (size_t)r * p.max_blocks_per_seq);
  const int last = (len - 1) / kBlock;
  // The wave's blocks of a step: in registers, and a step later in the step's buffer.  Blocks outside
  // the part are read but not used; before its beginning (where weights are 0) V is zeros.
  Block<D, kBits> block;
  auto load = [&](int key_step, int value_step) __attribute__((always_inline)) {
    const int b = kStepBlocks * value_step - 2 + wave;
    const int k_id = table[max(0, min(kStepBlocks * key_step + 2 + wave, last))];
    const int v_id = b < kStepBlocks * x0 ? -1 : table[min(b, last)];
    block.load_keys(Block<D, kBits>::tile(base, stride, k_id), lane);
    block.load_values(Block<D, kBits>::tile(base, stride, v_id), lane);
  };
  auto store_keys = [&](int step) __attribute__((always_inline)) {
    // lane (key, qd)'s features D / 4 qd + 8 i .. + 7: step s of the products, half h of the wave
    const float scale = scale_of(block.ks);
    const int qd = lane >> 4;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int step8 = qd % 2 * (D / 32) + i;
      (&sm.k[step & 1][wave][0][0])[(step8 * 2 + qd / 2) * 16 + (lane & 15)] = block.key_features(i, scale);
    }
  };
  // Of a 32 x 16 fragment of V^T lane l holds feature group l & 31, D / 32 features each in as many
  // fragments, and of the block's keys 4 h .. + 3 and 8 + 4 h .. + 3, h = l >> 5, as P's lanes do.
  const int v_lane = (lane >> 4 & 1) * 32 + 2 * (lane & 15);
  const int v_half = lane >> 5;
  float v_scale[4];
  // features 2 pair and 2 pair + 1 of the lane's D / 16
  auto store_values = [&](int step, int pair) __attribute__((always_inline)) {
    u32x2 f[2];
    block.values(pair, v_scale, f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = 2 * pair + i;
      *(reinterpret_cast<u32x2*>(&sm.v[step & 1][wave][t % (D / 32)][v_lane + t / (D / 32)]) + v_half) = f[i];
    }
  };
  auto cut_values = [&](int step) __attribute__((always_inline)) {
    const int n = len - step * kStepKeys + 16 * (2 - wave);
    if (n < 16) block.cut_values(n, lane);
    block.value_scales(v_scale);
  };

  if (x0 < xe) load(x0 - 1, x0);
  Rows32<D> rows[kTiles];
#pragma unroll
  for (int x = 0; x < kTiles; ++x) {
    const int row = row0 + 32 * x + (lane & 31);
    const int t = (unsigned)row / group;
    const long long q_row = (long long)(q0 + t) * p.num_q_heads + g * p.group + (row - t * p.group);
    rows[x].load(row < n_rows ? p.q + q_row * D : nullptr, lane);
  }
  // lane l has of row l & 31 and with h = l >> 5 the weights of keys 8 i + 4 h .. + 3 and O's
  // features of groups 8 i + 4 h .. + 3, i < 4
  typedef typename Softmax<32>::Logits Logits;
  Softmax<32> soft[kTiles];
  Logits o[kTiles][D / 32];
#pragma unroll
  for (int x = 0; x < kTiles; ++x)
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[x][i] = Logits{};
  auto barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // of the buffer's blocks 2 half and 2 half + 1
  const int key = lane & 15, k_block = lane >> 4 & 1, k_half = lane >> 5;
  // The work of half a step comes in chunks, each of two products for the logits and two for the values.
  constexpr int kChunks = D / 32;
  struct Keys {
    u32x4 w[2 * kChunks];
  };
  auto read_keys = [&](int step, int half) __attribute__((always_inline)) {
    const int buf = step & 1, b = 2 * half + k_block;
    Keys k;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) k.w[i] = (&sm.k[buf][b][0][0])[(2 * i + k_half) * 16 + key];
    return k;
  };
  auto add_logits = [&](int chunk, const Keys& k, Logits (&s)[kTiles]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 2 * chunk; e < 2 * chunk + 2; ++e) {
      const u32x4 a = k.w[e];
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), rows[x].q[e], s[x], 0, 0, 0);
    }
  };
  auto read_values = [&](int step, int half, int i) {
    return __builtin_bit_cast(bf16x8, sm.v[step & 1][2 * half + i / (D / 32)][i % (D / 32)][lane]);
  };
  auto add_values = [&](int i, const bf16x8& f, const bf16x8 (&w)[kTiles][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
      o[x][i % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, w[x][i / (D / 32)], o[x][i % (D / 32)], 0, 0, 0);
  };
  // Half a step: from the logits s of 32 keys their weights w; beside that the logits of the next
  // 32 and the values of the last 32, and the wave's share of the next step's buffer
  auto half_step = [&](int x, int half, Logits (&s)[kTiles], Logits (&next)[kTiles], const bf16x8 (&last_w)[kTiles][2],
                       bf16x8 (&w)[kTiles][2]) __attribute__((always_inline)) {
    const int key0 = x * kStepKeys + 32 * half;
    if (key0 + 32 > before + t0 + 1) {
#pragma unroll
      for (int y = 0; y < kTiles; ++y) {
        // keys that the row sees (found anew here: few steps are masked, and registers are short)
        int first = row0 + 32 * y;
        asm volatile("" : "+s"(first));
        const int end = before + min((int)((unsigned)(first + (lane & 31)) / group), t1) + 1;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[y][i] = key0 + 8 * (i / 4) + 4 * k_half + i % 4 < end ? s[y][i] : -INFINITY;
      }
    }
    // Chunk by chunk, so that a fragment is read one chunk before its products and few are held at a
    // time (the order within a chunk makes no difference that was measured)
    __builtin_amdgcn_sched_barrier(0);
    const Keys keys = read_keys(x, half);
    bf16x8 f[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) f[0][i] = read_values(x, half, i);
    float sum[kTiles];
#pragma unroll
    for (int y = 0; y < kTiles; ++y) {
      next[y] = Logits{};
      sum[y] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      if (k + 1 < kChunks) {
#pragma unroll
        for (int i = 0; i < 2; ++i) f[(k + 1) % 2][i] = read_values(x, half, 2 * (k + 1) + i);
      }
      if (half == 0 && k == 0) store_keys(x + 1);
      if (k % 2 == 1) store_values(x + 1, half * (D / 64) + k / 2);
#pragma unroll
      for (int y = 0; y < kTiles; ++y)
        sum[y] = soft[y].weigh(s[y], c, w[y], sum[y], 16 / kChunks * k, 16 / kChunks * (k + 1));
      add_logits(k, keys, next);
#pragma unroll
      for (int i = 0; i < 2; ++i) add_values(2 * k + i, f[k % 2][i], last_w);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int y = 0; y < kTiles; ++y) asm volatile("" : "+v"(next[y]));
#pragma unroll
    for (int y = 0; y < kTiles; ++y) soft[y].add(sum[y], s[y], c, o[y], w[y]);
  };
  if (x0 < xe) {
    Logits s0[kTiles], s1[kTiles];
    bf16x8 w0[kTiles][2], w1[kTiles][2] = {};
    store_keys(x0 - 1);
    cut_values(x0);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) store_values(x0, i);
    barrier();
    block.load_keys(Block<D, kBits>::tile(base, stride, table[min(kStepBlocks * x0 + 2 + wave, last)]), lane);
    const Keys keys = read_keys(x0 - 1, 1);
#pragma unroll
    for (int y = 0; y < kTiles; ++y) s0[y] = Logits{};
#pragma unroll
    for (int k = 0; k < kChunks; ++k) add_logits(k, keys, s0);
    store_keys(x0);
    load(x0 + 1, x0 + 1);
    for (int x = x0; x < xe; ++x) {
      // step x is in LDS, and no wave reads the other buffer any more
      barrier();
      cut_values(x + 1);
      half_step(x, 0, s0, s1, w1, w0);
      half_step(x, 1, s1, s0, w0, w1);
      load(x + 2, x + 2);
    }
    barrier();
#pragma unroll
    for (int i = 0; i < 2 * kChunks; ++i) add_values(i, read_values(xe, 0, i), w1);
  }
#pragma unroll
  for (int x = 0; x < kTiles; ++x) {
    float la, lb;
    swap32(soft[x].l, la, lb);
    const float l = la + lb;
    int row = row0 + 32 * x;
    asm volatile("" : "+s"(row));
    row += lane & 31;
    if (row >= n_rows) continue;
    const int t = (unsigned)row / group;
    const long long q_row = (long long)(q0 + t) * p.num_q_heads + g * p.group + (row - t * p.group);
    // D / 8 neighbouring features for each i, feature k of them in o[k % (D / 32)]
    if (p.parts == 1) {
      const float inv_l = 1.f / l;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < D / 8; k += 8) {
          bf16x8 y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (__bf16)(o[x][(k + e) % (D / 32)][4 * i + (k + e) / (D / 32)] * inv_l);
          *reinterpret_cast<bf16x8*>(p.out + q_row * D + D / 4 * i + D / 8 * k_half + k) = y;
        }
    } else {
      const size_t to = (size_t)part * p.total_q * p.num_q_heads + q_row;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < D / 8; k += 4) {
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = o[x][(k + e) % (D / 32)][4 * i + (k + e) / (D / 32)];
          *reinterpret_cast<f32x4*>(p.ws_o + to * D + D / 4 * i + D / 8 * k_half + k) = y;
        }
      if (lane < 32) *reinterpret_cast<float2*>(p.ws_ml + 2 * to) = make_float2(soft[x].m, l);
    }
  }
}

// A thread merges 4 features of a (token, query head) row.
template <int D>
__global__ __launch_bounds__(kThreads) void quant_prefill_merge_kernel(QuantParams p) {
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long n = (long long)p.total_q * p.num_q_heads;
  const long long row = i / (D / 4);
  const int d = (int)(i % (D / 4)) * 4;
  if (row >= (long long)p.cu_q_lens[p.batch] * p.num_q_heads) return;
  float m = -INFINITY, den = 0.f;
  f32x4 acc = f32x4{};
  for (int k0 = 0; k0 < p.parts; k0 += kMergeStep) {
    float2 ml[kMergeStep];
    f32x4 o[kMergeStep];
#pragma unroll
    for (int k = 0; k < kMergeStep; ++k) {
      ml[k] = make_float2(-INFINITY, 0.f);
      o[k] = f32x4{};
      if (k0 + k >= p.parts) continue;
      const size_t at = (size_t)((k0 + k) * n + row);
      ml[k] = *reinterpret_cast<const float2*>(p.ws_ml + 2 * at);
      o[k] = *reinterpret_cast<const f32x4*>(p.ws_o + at * D + d);
    }
    float m_new = m;
#pragma unroll
    for (int k = 0; k < kMergeStep; ++k) m_new = fmaxf(m_new, ml[k].x);
    const float alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    den *= alpha;
    acc *= alpha;
#pragma unroll
    for (int k = 0; k < kMergeStep; ++k) {
      const float wt = __builtin_amdgcn_exp2f(ml[k].x - m);
      den = __builtin_fmaf(wt, ml[k].y, den);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(wt, o[k][e], acc[e]);
    }
  }
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(acc[e] / den);
  *reinterpret_cast<uint2*>(p.out + row * D + d) = __builtin_bit_cast(uint2, y);
}

QuantParams params_of(const QuantAttnLaunch& a) {
  QuantParams p = {};
  p.q = a.q;
  p.pool = a.pool;
  p.block_tables = a.block_tables;
  p.lens = a.lens;
  p.cu_q_lens = a.cu_q_lens;
  p.out = a.out;
  p.batch = a.batch;
  p.max_blocks_per_seq = a.max_blocks_per_seq;
  p.num_q_heads = a.num_q_heads;
  p.num_kv_heads = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.scale_log2 = a.scale * kLog2e;
  p.total_q = a.total_q;
  return p;
}

template <int D, int kBits>
hipError_t decode(const QuantParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((quant_decode_kernel<D, kBits>), dim3((unsigned)p.ranges * p.num_kv_heads), dim3(kThreads), 0,
                     stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(quant_decode_merge_kernel<D>, dim3((unsigned)p.batch * p.num_kv_heads), dim3(kMergeThreads), 0,
                     stream, p);
  return hipGetLastError();
}

template <int D, int kBits>
hipError_t prefill(const QuantParams& p, int wave_tiles, long long grid, hipStream_t stream) {
  if (D == 64 && wave_tiles == 2)
    hipLaunchKernelGGL((quant_prefill_kernel<64, kBits, 2>), dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL((quant_prefill_kernel<D, kBits, 1>), dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  const long long threads = (long long)p.total_q * p.num_q_heads * (D / 4);
  hipLaunchKernelGGL(quant_prefill_merge_kernel<D>, dim3((unsigned)((threads + kThreads - 1) / kThreads)),
                     dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

QuantDecodeGeometry quant_decode_geometry(int batch, int max_seq_len, int num_q_heads, int num_kv_heads,
                                          int head_dim, int cus) {
  QuantDecodeGeometry geo = {};
  const double units = (double)((max_seq_len + 31LL) / 32);
  const double most = batch * units;
  geo.ranges = (kDecodeGroupsPerCu * cus + num_kv_heads - 1) / num_kv_heads;
  if (most < geo.ranges) geo.ranges = most < 1 ? 1 : (int)most;
  geo.rows = (long long)geo.ranges + batch;
  geo.bytes = geo.rows * num_q_heads * (head_dim + 2) * (long long)sizeof(float);
  // (units are counted in 32 bits, 64 sequences' at a time)
  geo.fits = launch_fits((double)geo.ranges * num_kv_heads, kThreads) &&
             launch_fits((double)batch * num_kv_heads, kMergeThreads) && (batch + 63.0) * units < 0x1p31;
  return geo;
}

hipError_t launch_quant_decode(const QuantAttnLaunch& a, const QuantDecodeGeometry& geo, hipStream_t stream) {
  QuantParams p = params_of(a);
  p.ranges = geo.ranges;
  p.rows = geo.rows;
  p.ws_o = a.workspace;
  p.ws_ml = a.workspace + geo.rows * a.num_q_heads * a.head_dim;
  if (a.head_dim == 64) return a.bits == 4 ? decode<64, 4>(p, stream) : decode<64, 8>(p, stream);
  return a.bits == 4 ? decode<128, 4>(p, stream) : decode<128, 8>(p, stream);
}

constexpr int kPrefillMaxParts = 16;
// Fewest steps of a part of the longest sequence.  A part's work-group takes about 10 us besides its steps of
// 1.3 (6 to the second step, 4 to store), and the merge launch 4.5 once.  us a call of 83 rows x 32 / 8 heads on 3094
// keys with 3, 4, 6, 8, 12 and 24: 29, 29.6, 25.5, 25.7, 28 and 38.
constexpr int kPrefillPartSteps = 6;

QuantPrefillGeometry quant_prefill_geometry(int batch, int total_q, int max_q_len, int max_kv_len,
                                            int num_q_heads, int num_kv_heads, int head_dim, int cus) {
  QuantPrefillGeometry geo = {};
  const long long group = num_q_heads / num_kv_heads;
  // work-groups there are at most: of the longest suffix, or as many as the rows of all make
  auto tiles_of = [&](int wave_tiles) {
    const long long rows = 32 * kWaves * wave_tiles;
    const double longest = (double)((max_q_len * group + rows - 1) / rows) * batch;
    const double all = (double)total_q * group / rows + batch;
    return num_kv_heads * (longest < all ? longest : all);
  };
  geo.wave_tiles = head_dim == 64 && tiles_of(2) >= cus ? 2 : 1;
  const long long rows = 32 * kWaves * geo.wave_tiles;
  geo.tiles = (max_q_len * group + rows - 1) / rows;
  const double tiles = tiles_of(geo.wave_tiles);
  long long parts = tiles > 0 ? (long long)(2 / geo.wave_tiles * cus / tiles) : 1;
  const long long steps = (max_kv_len + kStepKeys - 1LL) / kStepKeys;
  if (parts > steps / kPrefillPartSteps) parts = steps / kPrefillPartSteps;
  if (parts > kPrefillMaxParts) parts = kPrefillMaxParts;
  geo.parts = parts < 1 ? 1 : (int)parts;
  const double grid = (double)geo.tiles * batch * num_kv_heads * geo.parts;
  // (an invocation's rows of a KV head, and its keys up to the end of the step after next, are counted
  // in 32 bits)
  geo.fits = launch_fits(grid, kThreads) && max_q_len * group < 0x7fffff00LL && max_kv_len < 0x7fffff00LL &&
             (geo.parts == 1 || launch_fits((double)total_q * num_q_heads * (head_dim / 4) / kThreads + 1, kThreads));
  if (!geo.fits) return geo;
  geo.grid = (long long)grid;
  if (geo.parts > 1)
    geo.bytes = (long long)geo.parts * total_q * num_q_heads * (head_dim + 2) * (long long)sizeof(float);
  return geo;
}

hipError_t launch_quant_prefill(const QuantAttnLaunch& a, const QuantPrefillGeometry& geo, hipStream_t stream) {
  QuantParams p = params_of(a);
  p.parts = geo.parts;
  p.tiles = (int)geo.tiles;
  p.ws_o = a.workspace;
  p.ws_ml = a.workspace + (long long)geo.parts * a.total_q * a.num_q_heads * a.head_dim;
  auto* run = a.head_dim == 64 ? (a.bits == 4 ? prefill<64, 4> : prefill<64, 8>)
                               : (a.bits == 4 ? prefill<128, 4> : prefill<128, 8>);
  return run(p, geo.wave_tiles, geo.grid, stream);
}

}  // namespace cs
