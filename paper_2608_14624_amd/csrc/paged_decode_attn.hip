// Paged decode attention for gfx950: one new token per sequence attends over
// all keys of its sequence in the paged pool.
//
// This is the one-token case of the prefix-reuse attention (arXiv
// 2608.14624, Sec. 2.1: a request reuses the cached KV of its prefix; the
// per-turn latency the paper reports includes the decode that follows the
// prefill, Sec. 5): the query of sequence r is its last position L_r - 1 and
// sees every key 0 .. L_r - 1.  Decode reads each key once per KV head and
// does G = Hq / Hkv dot products with it, so it is bound by HBM bandwidth,
// not by the matrix cores.
//
// Kernel design
//   * One work-group = W wave64s = one (sequence, KV head), W = 12 (4 in
//     cascade mode); the G query heads of the group are the N = 16 columns
//     of v_mfma_f32_16x16x32_bf16 (G <= 16).
//   * The W waves split the key range in 32-key chunks (wave w takes chunks
//     w, w+W, ...) and run independent online softmaxes, so there is no
//     synchronisation in the loop; the W partial results are merged in LDS
//     at the end (log-sum-exp weights), so no workspace is needed.
//   * S^T = K Q^T with K fragments loaded from HBM straight into the MFMA A
//     operand (16 B per lane), Q^T kept in VGPRs.  O^T = V^T P^T reads V^T
//     with ds_read_b64_tr_b16 from a per-wave LDS tile that the wave itself
//     wrote (LDS operations of one wave complete in order, so no barrier).
//   * The K/V loads of a wave's next chunk are issued before the math of the
//     current one, so each wave keeps 16 KiB in flight.
//   * Work-groups are ordered KV head fastest, so each XCD serves one head.
//
// Cascade mode (the launches that cascade_ranges.hip does not take): a sequence
// belongs to a group whose shared prefix (its first
// shared_len keys) is attended by the stacked prefill kernel, which leaves
// one partial result (O relative to its running max m, the max m and the sum
// l) per 1024-key chunk in a workspace.  Here a work-group takes one KV head
// and one 1024-key segment of a sequence's own keys shared_len .. L - 1, so
// a long history spreads over several work-groups, and leaves its partial
// in the workspace too; cascade_merge_kernel then combines every partial of
// a row with log-sum-exp weights exp2((m_i - max) * c).
#include "decode_common.h"
#include "internal.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace cs {
namespace {

// waves per work-group: 12 for plain decode (one work-group fills a CU at
// three waves per SIMD, so a CU's last, longest sequence runs on all of its
// wave slots instead of a third of them), 4 for the cascade's 1024-key
// segments
constexpr int kDecodeWaves = 12;
constexpr int kCascadeWaves = 4;
constexpr int kThreads = 256;        // the merge kernel
// plain decode batches up to this size run longest sequence first
constexpr int kLptMaxBatch = 1024;

// What a decode launch attends over: all keys of a sequence; its own keys past a shared
// prefix (the cascade's rest); those under a window and the first few (sinks); or all of
// them, adding every key's attention weight to its score.
enum class Keys { kAll, kCascade, kWindow, kScored };

struct DecParams {
  const uint16_t* q;          // [B][Hq][D]
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* block_tables;
  const int32_t* seq_lens;
  uint16_t* out;              // [B][Hq][D]
  int max_blocks_per_seq;
  int num_q_heads;
  int num_kv_heads;
  int group;
  float scale_log2;
  // decode in ranges (decode_ranges_kernel): work-groups per KV head, partials
  // per KV head in ws_o / ws_ml, and the plan ({aligned, units per piece})
  int ranges;
  int aligned_ranges;
  int slots;
  int2* plan;
  // cascade mode only
  const int32_t* cu_groups;     // [num_groups + 1], cu_groups[0] = 0, last = batch
  const int32_t* shared_lens;   // [num_groups]
  int num_groups;
  int batch;
  int chunk_keys;               // keys per partial of the shared prefix
  int chunks;                   // shared-prefix partials per row (upper bound)
  int segments;                 // own-key partials per row (upper bound)
  float* ws_o;                  // [chunks + segments][batch * num_q_heads][D]
  float* ws_ml;                 // [chunks + segments][batch * num_q_heads][2]
  int ws_rows;
  // Keys::kWindow
  int window;
  int sinks;
  // Keys::kScored: a sequence's logits from the unit of its first scored key on,
  // [batch][num_kv_heads][logit_units][8 quads of keys][group][4]
  const int32_t* score_from;
  float* score_pool;            // [num_blocks][num_kv_heads][16]
  float decay;
  float* logits;
  int logit_units;
  int lds_units;                // of these, the ones that decode_scores_pair_kernel keeps in LDS
};

// The units of a sequence of len keys that its query sees, as a list: under a window
// those with a key below `sinks` or from `lo` on, unit x of the list being the
// sequence's unit x or (past the sinks) x + skip; else all of them.
template <Keys kKeys>
struct SeenUnits {
  int sinks, lo, sink_units, skip;
  __device__ __forceinline__ SeenUnits(const DecParams& p, int len) {
    if constexpr (kKeys == Keys::kWindow) {
      sinks = min(p.sinks, len);
      lo = max(0, len - p.window);
      sink_units = units_of(sinks);
      skip = max(0, lo / kUnitKeys - sink_units);
    }
  }
  __device__ __forceinline__ int count(int len) const {
    if constexpr (kKeys == Keys::kWindow) return units_of(len) - skip;
    else return units_of(len);
  }
  __device__ __forceinline__ int unit(int x) const {
    if constexpr (kKeys == Keys::kWindow) return x < sink_units ? x : x + skip;
    else return x;
  }
  __device__ __forceinline__ bool key(int k) const {
    if constexpr (kKeys == Keys::kWindow) return k >= lo || k < sinks;
    else return true;
  }
  // no key of pool block b is seen: its table entry is not read
  __device__ __forceinline__ bool hidden(int b) const {
    if constexpr (kKeys == Keys::kWindow) return b * kBlock >= sinks && (b + 1) * kBlock <= lo;
    else return false;
  }
  // V rows of hidden keys in a unit's LDS tile as zeros (0 times a NaN there is NaN)
  template <int D>
  __device__ __forceinline__ void zero_hidden(int lane, int key0, uint16_t* tile) const {
    if constexpr (kKeys == Keys::kWindow) {
      if (key0 < lo && key0 + kUnitKeys > sinks) {
#pragma unroll
        for (int v = 0; v < kChunk * D / 8 / 64; ++v) {
          const int cc = lane + 64 * v;
          if (!key(key0 + cc / (D / 8)))
            *reinterpret_cast<bf16x8*>(&tile[(cc / (D / 8)) * v_tile_stride(D) + (cc % (D / 8)) * 8]) = bf16x8{};
        }
      }
    }
  }
};

template <Keys kKeys>
__device__ __forceinline__ int seen_units(const DecParams& p, int len) {
  return SeenUnits<kKeys>(p, len).count(len);
}

// Where the lane's four logits (quad mt * 4 + qd, head j of the group) of a unit are
// kept, or null: a unit before the first scored key, or past the bound of their number.
__device__ __forceinline__ float* logits_at(const DecParams& p, int r, int g, int unit, int from_unit) {
  const int u = unit - from_unit;
  if (u < 0 || u >= p.logit_units) return nullptr;
  return p.logits + (((size_t)r * p.num_kv_heads + g) * p.logit_units + u) * (size_t)(kUnitKeys * p.group);
}
__device__ __forceinline__ void keep_logits(const DecParams& p, float* unit_logits, int lane, const f32x4 (&s)[2]) {
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
    *reinterpret_cast<f32x4*>(unit_logits + 4 * ((4 * mt + (lane >> 4)) * p.group + (lane & 15))) = s[mt];
}

// Units whose logits a wave of decode_ranges_kernel stages in LDS before it stores them:
// 128 sequences of 4.2k-10k keys 806 us without, 751 with 4 units, 747 with 8, 743 with 16.
constexpr int kStagedUnits = 8;

// The weights of four keys, of the group's heads together, from their logits ([group][4]).
// stat: m c and 1 / l of every head.
__device__ __forceinline__ f32x4 quad_weights(const DecParams& p, const float2* stat, const float* logits) {
  f32x4 w = f32x4{};
  for (int j = 0; j < p.group; ++j) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(logits + 4 * j);
    const float2 st = stat[j];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(x[e], p.scale_log2, -st.x)), st.y, w[e]);
  }
  return w;
}

// The scores of the keys key .. key + 3 with the weights added; those not scored as they
// were.  The query's own key is new in this step: what its slot held is another key's.
__device__ __forceinline__ f32x4 quad_scores(const DecParams& p, f32x4 old, f32x4 w, int key, int from, int len) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float kept = key + e == len - 1 ? 0.f : p.decay * old[e];
    w[e] = key + e >= from && key + e < len ? kept + w[e] : old[e];
  }
  return w;
}

// The first scored key of sequence r, its length if there is none (score_from may be any number
// from 0 on, and what follows adds to it).
__device__ __forceinline__ int first_scored(const DecParams& p, int r, int len) {
  return min(max(0, p.score_from[r]), len);
}

__device__ __forceinline__ float* score_at(const DecParams& p, int id, int g, int key) {
  return p.score_pool + ((size_t)id * p.num_kv_heads + g) * kBlock + key % kBlock;
}

// first key of sequence r that its group does not share
__device__ __forceinline__ int shared_len_of(const DecParams& p, int r) {
  int lo = 0, hi = p.num_groups - 1;   // the last group gr with cu_groups[gr] <= r
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.cu_groups[mid] <= r) lo = mid; else hi = mid - 1;
  }
  return p.shared_lens[lo];
}

template <int D, int W>
struct DecLds {
  static constexpr int vStride = v_tile_stride(D);
  union {
    uint16_t v[W][kChunk * vStride];
    struct {
      float m[W][kMaxGroup];
      float l[W][kMaxGroup];
      float o[W][kMaxGroup][D];
    } merge;
  };
};

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

template <int D, Keys kKeys>
__global__ __launch_bounds__(64 * (kKeys == Keys::kCascade ? kCascadeWaves : kDecodeWaves)) void paged_decode_attn_kernel(
    DecParams p) {
  constexpr bool kCascade = kKeys == Keys::kCascade;
  constexpr int kWaves = kCascade ? kCascadeWaves : kDecodeWaves;
  constexpr int kWGThreads = 64 * kWaves;
  __shared__ DecLds<D, kWaves> sm;
  constexpr int vStride = DecLds<D, kWaves>::vStride;
  constexpr int DC = D / 32;         // 32-wide k-steps of the QK^T product
  constexpr int DT = D / 16;         // 16-row output tiles over the head dim
  constexpr int kRowChunks = D / 8;  // 16-byte chunks per key row
  constexpr int kVLoads = kChunk * kRowChunks / 64;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15;           // MFMA column: query head within the group
  const int qd = lane >> 4;          // lane group: k-slots 8*qd .. +7

  const int g = blockIdx.x % p.num_kv_heads;
  int r, seg = 0;
  if constexpr (kCascade) {
    r = (blockIdx.x / p.num_kv_heads) % p.batch;
    seg = blockIdx.x / p.num_kv_heads / p.batch;
  } else {
    // Longest sequence first: the work-groups of one wave of dispatch take
    // the sequences of ranks w / num_kv_heads in decreasing length (ties by
    // index), so the last of the launch's rounds holds the shortest ones
    // and the CUs run out of work together.  Every work-group ranks the
    // lengths itself (each thread a few candidates against all of them, in
    // LDS): the order is a permutation whatever the lengths hold, so every
    // (sequence, head) is still computed exactly once, and each output is
    // the same as in any other order.
    // (Under a window the sequences' work is about the same.)
    r = blockIdx.x / p.num_kv_heads;
    if (kKeys != Keys::kWindow && p.batch <= kLptMaxBatch) {
      __shared__ int lens[kLptMaxBatch];
      __shared__ int pick;
      for (int s = threadIdx.x; s < p.batch; s += kWGThreads) lens[s] = p.seq_lens[s];
      if (threadIdx.x == 0) pick = r;
      __syncthreads();
      for (int s = threadIdx.x; s < p.batch; s += kWGThreads) {
        const int ls = lens[s];
        int rank = 0;
        for (int t = 0; t < p.batch; ++t) {
          const int lt = lens[t];
          rank += (lt > ls) || (lt == ls && t < s);
        }
        if (rank == r) pick = s;
      }
      __syncthreads();
      r = pick;
    }
  }
  const int L = p.seq_lens[r];
  int start = 0;       // keys start .. end - 1 are this work-group's
  int end = L;
  if constexpr (kCascade) {
    start = shared_len_of(p, r) + seg * kCascadeSegmentKeys;
    end = min(L, start + kCascadeSegmentKeys);
    if (start >= end) return;          // nothing of this sequence's own here
  }
  const int n_blk = (end + kBlock - 1) / kBlock;
  const SeenUnits<kKeys> seen(p, L);
  const int first_chunk = start / kChunk;
  const int ch_end = kKeys == Keys::kWindow ? seen.count(L) : (end + kChunk - 1) / kChunk;
  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const uint16_t* kbase = p.k_pool + (size_t)g * tile_elems;
  const uint16_t* vbase = p.v_pool + (size_t)g * tile_elems;
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(p.block_tables +
                                                          (size_t)r * p.max_blocks_per_seq);

  // ---- Q^T operand: column j = query head g*G + j, dims 32*dc + 8*qd .. +7
  const bool head_valid = j < p.group;
  const int h = g * p.group + (head_valid ? j : 0);
  bf16x8 qreg[DC];
#pragma unroll
  for (int dc = 0; dc < DC; ++dc) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (head_valid)
      v = *reinterpret_cast<const uint4*>(p.q + ((size_t)r * p.num_q_heads + h) * D + 32 * dc + 8 * qd);
    qreg[dc] = as_bf16x8(v);
  }

  // ---- loads of one chunk: K fragments (A operand) and V rows (to LDS) --
  uint4 kreg[2][DC];
  uint4 vreg[kVLoads];
  auto load_chunk = [&](int ch) {
    const int b0 = 2 * seen.unit(ch);
    const int id0 = b0 < n_blk && !seen.hidden(b0) ? bt[b0] : -1;
    const int id1 = b0 + 1 < n_blk && !seen.hidden(b0 + 1) ? bt[b0 + 1] : -1;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int id = mt ? id1 : id0;
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) {
        kreg[mt][dc] = make_uint4(0, 0, 0, 0);
        if (id >= 0)
          kreg[mt][dc] = *reinterpret_cast<const uint4*>(kbase + (size_t)id * slot_elems + j * D + 32 * dc + 8 * qd);
      }
    }
#pragma unroll
    for (int u = 0; u < kVLoads; ++u) {
      const int c = lane + 64 * u;
      const int key = c / kRowChunks;           // 0..31, uniform block per u
      const int id = key < kBlock ? id0 : id1;
      vreg[u] = make_uint4(0, 0, 0, 0);
      if (id >= 0)
        vreg[u] = *reinterpret_cast<const uint4*>(vbase + (size_t)id * slot_elems + (key % kBlock) * D + (c % kRowChunks) * 8);
    }
  };

  const uint16_t* vt = sm.v[wave];
  f32x4 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{};
  float m_run = -INFINITY;
  float l_run = 0.f;
  const float c = p.scale_log2;

  int ch = first_chunk + wave;
  if (ch < ch_end) load_chunk(ch);
  for (; ch < ch_end; ch += kWaves) {
    // V rows of this chunk into the wave's LDS tile
#pragma unroll
    for (int u = 0; u < kVLoads; ++u) {
      const int cc = lane + 64 * u;
      *reinterpret_cast<uint4*>(&sm.v[wave][(cc / kRowChunks) * vStride + (cc % kRowChunks) * 8]) = vreg[u];
    }
    // rows past the end of the sequence (inside its last block) overwritten
    // with zeros: their probabilities are 0, but 0 times a stale NaN or Inf
    // in the pool is NaN
    const int kbase_idx = seen.unit(ch) * kChunk;
    seen.template zero_hidden<D>(lane, kbase_idx, sm.v[wave]);
    if (kbase_idx + kChunk > end) {
#pragma unroll
      for (int u = 0; u < kVLoads; ++u) {
        const int cc = lane + 64 * u;
        if (kbase_idx + cc / kRowChunks >= end)
          *reinterpret_cast<uint4*>(&sm.v[wave][(cc / kRowChunks) * vStride + (cc % kRowChunks) * 8]) =
              make_uint4(0, 0, 0, 0);
      }
    }
    // S^T = K Q^T: two 16-key tiles
    f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int dc = 0; dc < DC; ++dc)
        s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kreg[mt][dc]), qreg[dc], s[mt], 0, 0, 0);
    if (ch + kWaves < ch_end) load_chunk(ch + kWaves);     // in flight during the math

    // mask keys past the end; register r of tile mt holds key 32*ch + 16*mt + 4*qd + r
    float mloc = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int key = kbase_idx + 16 * mt + 4 * qd + rr;
        s[mt][rr] = (key < end && key >= start && seen.key(key)) ? s[mt][rr] : -INFINITY;
        mloc = fmaxf(mloc, s[mt][rr]);
      }
    mloc = fmaxf(mloc, __shfl_xor(mloc, 16));
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
    const float m_new = fmaxf(m_run, mloc);
    const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
    const float mc = m_new * c;
    bf16x8 pb;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][rr], c, -mc));
        pb[4 * mt + rr] = (__bf16)e;
        l_run += (float)pb[4 * mt + rr];
      }
    // O^T += V^T P^T
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_fragment<D>(vt, lane, dt), pb, oacc[dt], 0, 0, 0);
  }

  // ---- merge the waves' partial softmaxes -----------------------------
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  __syncthreads();                     // every wave is done with its V tile
  if (qd == 0) {
    sm.merge.m[wave][j] = m_run;
    sm.merge.l[wave][j] = l_run;
  }
  // accumulator register rr of tile dt holds dim 16*dt + 4*qd + rr of head j
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) sm.merge.o[wave][j][16 * dt + 4 * qd + rr] = oacc[dt][rr];
  __syncthreads();
  for (int idx = threadIdx.x; idx < p.group * D; idx += kWGThreads) {
    const int hj = idx / D;
    const int d = idx % D;
    const size_t row = (size_t)r * p.num_q_heads + g * p.group + hj;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, sm.merge.m[w][hj]);
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f((sm.merge.m[w][hj] - mx) * c);   // 0 for idle waves
      num += wt * sm.merge.o[w][hj][d];
      den += wt * sm.merge.l[w][hj];
    }
    if constexpr (kCascade) {
      // this segment's partial: O relative to mx, mx, and the sum
      const size_t widx = (size_t)(p.chunks + seg) * p.ws_rows + row;
      p.ws_o[widx * D + d] = num;
      if (d == 0) {
        p.ws_ml[2 * widx] = mx;
        p.ws_ml[2 * widx + 1] = den;
      }
    } else if constexpr (kKeys == Keys::kAll) {
      p.out[row * D + d] = __builtin_bit_cast(uint16_t, (__bf16)(num / den));
    } else {
      // a row of an empty sequence (a padded batch) is zero
      p.out[row * D + d] = __builtin_bit_cast(uint16_t, (__bf16)(L > 0 ? num / den : 0.f));
    }
  }
}

// ---- decode in ranges ----------------------------------------------------
//
// One wave per work-group, a few per CU, p.ranges of them per KV head whatever
// the batch holds.  The sequences' keys are counted in units of 32 (one chunk),
// and every wave works the plan out itself from the lengths (wave-wide scans),
// so the host needs no lengths and no tight bound of them.
//   * Nothing shared: the sequences' units are laid end to end in batch order
//     and dealt in equal contiguous ranges of ceil(total / ranges) units.
//   * Where enough of the batch shares prefixes (counted by the pool block at
//     index kProbeBlock of the block tables): every sequence is cut at the same
//     positions, multiples of ceil(total / (aligned_rounds ranges)) units, and the
//     waves take the first pieces of all sequences, then the second ones, ..., so
//     that sequences with the same blocks read them at about the same time and
//     most find them in L2.
// A piece of a sequence that is not the whole of it leaves a partial result (O
// relative to its running max m, the max m and the sum l) in a slot of the
// workspace, and decode_ranges_merge_kernel combines a sequence's pieces.  The
// slot of a contiguous piece is r + w (sequence r, range w: both grow from piece
// to piece, so slots are unique), of an aligned piece its index among all.
//
// What bounds it is HBM, and how it is asked: 4 KiB (block, head) tiles at
// scattered places.  More requests in flight than the memory needs make some
// waves starve (first loads served after 60 us of a 90 us launch) while the
// slowest range sets the time, and ordinary loads wash the whole stream through
// the last-level cache.  128 sequences of 6000-9000 keys, 32 / 8 heads of 128:
// twelve waves per CU as work-groups of four 659 us, with non-temporal loads
// 612, four single-wave work-groups per CU and non-temporal loads 574, three
// 571 (6.7 TB/s; one 12-wave work-group per sequence and KV head: 642).  Three
// per CU at head_dim 128 (two: 1% slower, five: 6%), four at 64, where a wave's
// chunk is half the bytes (three: 5% slower).  K and V both non-temporal is up
// to 4% faster than V alone, but 17% slower where the pools were written just
// before (4 GB of them: 875 us against 749; ordinary loads 797).  Sequences that
// share want ordinary loads and more waves, at head_dim 128 eight per CU with two
// pieces each (128 sequences of 8 agents 317 us, four and four 355), at 64, where
// a unit is half the bytes, sixteen with one (256 sequences of 8 agents, 8 / 2
// heads, 86 us; eight and two 97, one work-group per sequence and KV head 89).
//
// For sequences with blocks of their own the aligned pieces are the slower ones
// (many waves, ordinary loads): 128 of 6000-9000 keys, two of them on one anchor,
// 32 / 8 heads of 128, 592 us in ranges, 676 in pieces, one work-group each 648.
// And short launches lose in pieces what the order saves: the pieces' ends do not
// meet the work of the waves.  Pieces are therefore taken where at least a
// quarter of the sequences are on a block counted before (kSharingPart), and that
// share times the units of an equal range is at least kSharedUnits.  us a call,
// ranges and pieces, at share times units: 4 / 1 heads of 64, 128 sequences of one
// agent 18.5 and 22.7 (11), 500 of 16 45.3 and 48.3 (29), 256 of 8 61 and 54 (52);
// 8 / 2 of 64, 128 of one 25.1 and 26.4 (21), 500 of 16 68 and 61 (57), 128 of 64
// 32 and 38 (11); 32 / 8 of 64, 24 of 3 18.3 and 19.8 (11), 64 of 4 47.8 and 42.2
// (42); 32 / 8 of 128, 16 of 2 46.9 and 48.4 (31), 64 of 4 75 and 67 (56); of 128
// sequences of 6000-9000 keys 64 in pairs (a quarter counted: 67) 555 and 532 at
// 128, 269 and 281 at 64, and 48 in pairs 565 and 568, 273 and 302.
// Pieces per CU and KV head, and how many of them a wave takes:
constexpr int kAlignedPiecesPerCu = 16;
constexpr int aligned_rounds(int head_dim) { return head_dim == 64 ? 1 : 2; }
constexpr int kSharingPart = 4;
constexpr int kSharedUnits = 36;
constexpr int kProbeBlock = 31;
constexpr int kProbeTable = 2 * kRangeMaxBatch;
constexpr int kPlanRounds = kRangeMaxBatch / 64;

// f(0), f(1), ... over the rounds of 64 sequences that a batch takes, or up to
// twice as many (past the batch f has nothing to do): a small batch passes the
// code of the other rounds in one jump, where a test per round and loop took 1.3
// us of a 14 us call in instruction fetches.
template <int kFrom = 0, typename F>
__device__ __forceinline__ void plan_rounds(int batch, F&& f) {
  constexpr int kTo = kFrom == 0 ? 1 : 2 * kFrom;
#pragma unroll
  for (int i = kFrom; i < kTo; ++i) f(i);
  if constexpr (kTo < kPlanRounds) {
    if (batch > 64 * kTo) plan_rounds<kTo>(batch, f);
  }
}

// How many of the batch's sequences hold the pool block at index kProbeBlock that
// another one counted before them holds (one wave; ids: the lane's sequences',
// -1 where there is none): a hash table of the blocks in LDS, at most half full.
// The count is that of all less the different ones, so it does not depend on the
// order in which the lanes meet.
__device__ __forceinline__ int count_sharing(const int (&ids)[kPlanRounds], int batch, int lane, int* table) {
  for (int i = lane; i < kProbeTable; i += 64) table[i] = -1;
  __syncthreads();
  int dups = 0;
  plan_rounds(batch, [&](int i) __attribute__((always_inline)) {
    const int id = ids[i];
    bool dup = false;
    if (id >= 0) {
      unsigned h = ((unsigned)id * 2654435761u) >> 16;
      for (int tries = 0; tries < kProbeTable; ++tries) {
        h %= kProbeTable;
        const int old = atomicCAS(&table[h], -1, id);
        if (old == -1) break;
        if (old == id) {
          dup = true;
          break;
        }
        ++h;
      }
    }
    dups += __builtin_popcountll(__builtin_amdgcn_ballot_w64(dup));
  });
  __syncthreads();
  return dups;
}

// A position in a wave's list of pieces.
struct RangeCursor {
  int r;          // sequence
  int len;        // its keys
  int x, xe;      // unit within the sequence, end of the piece
  int slot;       // where the piece's partial goes; negative: the piece is the whole
                  // sequence (~ the slot its m and l go to where scores are asked)
  bool valid;
};

template <int D, Keys kKeys>
__global__ __launch_bounds__(64) void decode_ranges_kernel(DecParams p) {
  constexpr int vStride = v_tile_stride(D);
  constexpr int DC = D / 32;
  constexpr int DT = D / 16;
  constexpr int kVLoads = kChunk * D / 8 / 64;
  constexpr int kManyUnits = 0xffff;
  constexpr bool kScored = kKeys == Keys::kScored;
  __shared__ union {
    struct {
      uint16_t v[kChunk * vStride];
      uint16_t units[kRangeMaxBatch];    // of every sequence (kManyUnits: that many or more)
    };
    int probe[kProbeTable];
  } sm;

  extern __shared__ __attribute__((aligned(16))) float staged[];     // kScored: kStagedUnits units' logits
  const int lane = threadIdx.x;
  const int j = lane & 15;
  const int qd = lane >> 4;
  const int g = blockIdx.x % p.num_kv_heads;
  const int w = blockIdx.x / p.num_kv_heads;
  const ScalarInts lens_c = (ScalarInts)p.seq_lens;
  const ScalarInts from_c = (ScalarInts)p.score_from;

  // ---- the plan.  All lengths and probed blocks are asked for at once, and the
  // units then kept in LDS: read from memory again for every piece, a batch of
  // 256 spent longer on finding its last pieces than on a short piece itself.
  int n_of[kPlanRounds], ids_probed[kPlanRounds];
  const bool probes = p.batch > 1 && p.max_blocks_per_seq > kProbeBlock;
  plan_rounds(p.batch, [&](int i) __attribute__((always_inline)) {
    const int s = 64 * i + lane;
    n_of[i] = s < p.batch ? p.seq_lens[s] : 0;
    ids_probed[i] = probes && s < p.batch ? p.block_tables[(size_t)s * p.max_blocks_per_seq + kProbeBlock] : -1;
  });
  int total = 0, longest = 0;
  int unscored = 0;                      // units before the sequences' first scored keys
  plan_rounds(p.batch, [&](int i) __attribute__((always_inline)) {
    if (n_of[i] <= kProbeBlock * kBlock) ids_probed[i] = -1;      // an entry past its last block
    if (SeenUnits<kKeys>(p, n_of[i]).hidden(kProbeBlock)) ids_probed[i] = -1;
    n_of[i] = seen_units<kKeys>(p, n_of[i]);
    total += wave_total(n_of[i]);
    if constexpr (kScored) {
      const int s = 64 * i + lane;
      unscored += wave_total(s < p.batch ? units_of(min(p.score_from[s], n_of[i] * kUnitKeys)) : 0);
    }
    longest = max(longest, wave_max(n_of[i]));
  });
  bool aligned = false;
  if (p.batch > 1 && total >= kSharedUnits * p.ranges) {
    const int sharing = count_sharing(ids_probed, p.batch, lane, sm.probe);
    aligned = kSharingPart * sharing >= p.batch &&
              (long long)sharing * total >= (long long)kSharedUnits * p.batch * p.ranges;
    // What is scored is no other sequence's, so where scores are asked it is known how much
    // of the batch can be shared.  128 sequences of 8 agents, 1024 shared keys and 3200-9000
    // of their own: 772 us in pieces, 741 in ranges.
    if constexpr (kScored)
      aligned = aligned && (long long)kSharingPart * sharing * unscored >= (long long)p.batch * total;
  }
  plan_rounds(p.batch, [&](int i) __attribute__((always_inline)) {
    sm.units[64 * i + lane] = (uint16_t)min(n_of[i], kManyUnits);
  });
  __syncthreads();
  auto units_at = [&](int s) {           // of sequence s (a lane's), 0 past the batch
    if (s >= p.batch) return 0;
    const int n = sm.units[s];
    return n == kManyUnits ? seen_units<kKeys>(p, p.seq_lens[s]) : n;
  };
  const int ranges = aligned ? p.aligned_ranges : p.ranges;     // waves that take part
  // With few KV heads there are more waves than the merge has use for: few
  // sequences in pieces of one unit leave it hundreds of partials each.  Past
  // 16 pieces of the longest sequence a range has up to 4 units (8 / 1 heads,
  // one sequence of 7000 keys 27.3 -> 13.9 us, 3 of 2000-6000 23.3 -> 14.6; 8 of
  // 100-500 9.8 with 1, 11.3 with 4).  Aligned pieces are longer by their rule.
  const int shortest = min(4, ceil_div(longest, 16));
  const int per = max(max(1, shortest), ceil_div(total, aligned ? aligned_rounds(D) * ranges : ranges));
  if (blockIdx.x == 0 && lane == 0) *p.plan = make_int2(aligned, per);

  // the sequence's slots: its pieces are numbered from here
  auto piece_base = [&](int r) {
    int t = 0;
    for (int s = 0; s < r; s += 64) t += wave_total(s + lane < r ? ceil_div(units_at(s + lane), per) : 0);
    return t;
  };
  // aligned pieces in order of (piece, sequence): the wave's are w, w + ranges, ...
  int rank = 0, piece = 0;
  auto aligned_piece = [&](RangeCursor& c) {
    for (;; ++piece) {
      int count = 0;
      for (int s = 0; s < p.batch; s += 64)
        count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(units_at(s + lane) > piece * per));
      if (count == 0) {
        c.valid = false;
        return;
      }
      if (rank < count) break;
      rank -= count;
    }
    int before = 0;
    for (int s = 0; s < p.batch; s += 64) {
      const unsigned long long mask = __builtin_amdgcn_ballot_w64(units_at(s + lane) > piece * per);
      const int n = __builtin_popcountll(mask);
      if (rank < before + n) {
        const int mine = __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
        const bool hit = ((mask >> lane) & 1) && mine == rank - before;
        c.r = s + __builtin_ctzll(__builtin_amdgcn_ballot_w64(hit));
        break;
      }
      before += n;
    }
    c.len = lens_c[c.r];
    c.x = piece * per;
    const int n = seen_units<kKeys>(p, c.len);
    c.xe = min(n, c.x + per);
    const bool whole = n <= per;
    c.slot = whole && !kScored ? -1 : piece_base(c.r) + piece;
    if (kScored && whole) c.slot = ~c.slot;
    c.valid = true;
  };
  // contiguous ranges: `left` units of the range lie past the cursor's piece
  int left = 0;
  auto contiguous_piece = [&](RangeCursor& c) {      // from unit c.x of sequence c.r on
    const int n = seen_units<kKeys>(p, c.len);
    c.xe = min(n, c.x + left);
    left -= c.xe - c.x;
    c.slot = (c.x == 0 && c.xe == n) ? (kScored ? ~(c.r + w) : -1) : c.r + w;
    c.valid = true;
  };

  RangeCursor ids{};
  if (w >= ranges) return;
  if (aligned) {
    rank = w;
    aligned_piece(ids);
  } else {
    const int u = w * per;
    left = min(total, u + per) - u;
    if (left > 0) {
      int first = 0;                                    // first unit of sequence ids.r
      for (int s = 0;; s += 64) {
        const int n = units_at(s + lane);
        const int incl = wave_scan(n);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(first + incl > u);
        if (past != 0) {
          const int l = __builtin_ctzll(past);
          ids.r = s + l;
          first += __builtin_amdgcn_readlane(incl - n, l);
          break;
        }
        first += __builtin_amdgcn_readlane(incl, 63);
      }
      ids.len = lens_c[ids.r];
      ids.x = u - first;
      contiguous_piece(ids);
    }
  }
  if (!ids.valid) return;
  // the unit after the cursor's: in its piece, or the first of the next one
  auto advance = [&](RangeCursor& c, auto tag) {
    if (++c.x < c.xe) return;
    if constexpr (decltype(tag)::value) {
      rank += ranges;
      aligned_piece(c);
      return;
    }
    if (left <= 0) {
      c.valid = false;
      return;
    }
    do c.len = lens_c[++c.r];
    while (c.len <= 0);
    c.x = 0;
    contiguous_piece(c);
  };

  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const uint16_t* kbase = p.k_pool + (size_t)g * tile_elems;
  const uint16_t* vbase = p.v_pool + (size_t)g * tile_elems;
  const bool head_valid = j < p.group;
  const int h = g * p.group + (head_valid ? j : 0);
  const float c = p.scale_log2;
  // a unit whose logits are all -inf weighs 0 relative to this, not NaN
  const float lowest = lowest_reference(c);

  bf16x8 kreg[2][DC];
  bf16x8 vreg[kVLoads];
  // K fragments and V rows of the blocks id0, id1.  Where each block is read
  // once V is loaded non-temporally, so that half the stream leaves the
  // last-level cache alone
  auto load_chunk = [&](int id0, int id1, auto tag) {
    load_chunk_tiles<D, decltype(tag)::value ? 0 : kNonTemporal>(kbase, vbase, id0, id1, slot_elems, lane, kreg, vreg);
  };
  // block ids of a cursor's unit; past the sequence's end its last block again
  // (its keys there are masked, its V rows zeroed)
  auto ids_of = [&](const RangeCursor& cu, int& id0, int& id1) {
    const ScalarInts bt = (ScalarInts)(p.block_tables + (size_t)cu.r * p.max_blocks_per_seq);
    const SeenUnits<kKeys> seen(p, cu.len);
    int b0 = seen.unit(cu.x) * kUnitBlocks;
    int b1 = min(b0 + 1, (cu.len - 1) / kBlock);
    // (a hidden block stands for the unit's other one; its keys are masked, its V zeroed)
    const int hidden0 = seen.hidden(b0) ? b1 : b0;
    b1 = seen.hidden(b1) ? b0 : b1;
    b0 = hidden0;
    id0 = bt[b0];
    id1 = bt[b1];
  };
  bf16x8 qreg[DC];
  auto load_q = [&](int r) {
#pragma unroll
    for (int dc = 0; dc < DC; ++dc) {
      qreg[dc] = bf16x8{};
      if (head_valid)
        qreg[dc] = *reinterpret_cast<const bf16x8*>(p.q + ((size_t)r * p.num_q_heads + h) * D + 32 * dc + 8 * qd);
    }
  };

  f32x4 oacc[DT];
  float m_run, l_run;
  auto reset = [&]() {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{};
    m_run = -INFINITY;
    l_run = 0.f;
  };

  // three cursors: the unit being computed, the one whose loads are in flight
  // behind it, and the one whose block ids are being read
  auto run = [&](auto tag) __attribute__((always_inline)) {
    RangeCursor cur = ids;
    int id0, id1;
    ids_of(cur, id0, id1);
    load_q(cur.r);
    int from_unit = 0;                   // of the sequence's first scored key
    int n_staged = 0;                    // units staged in LDS, of one piece, and where they go
    float* staged_to = nullptr;
    bool piece_begins = false;           // the unit is the first of a piece that is not the wave's first
    auto store_staged = [&]() __attribute__((always_inline)) {
      for (int i = 4 * lane; i < n_staged * kUnitKeys * p.group; i += 4 * 64)
        *reinterpret_cast<f32x4*>(staged_to + i) = *reinterpret_cast<const f32x4*>(staged + i);
      n_staged = 0;
    };
    if constexpr (kScored) from_unit = max(0, from_c[cur.r]) / kUnitKeys;
    load_chunk(id0, id1, tag);
    reset();
    advance(ids, tag);
    RangeCursor nxt = ids;
    if (nxt.valid) ids_of(nxt, id0, id1);

    for (;;) {
      const SeenUnits<kKeys> seen(p, cur.len);
      const int key0 = seen.unit(cur.x) * kUnitKeys;
      store_v_tile<D>(vreg, lane, key0, cur.len, sm.v);
      seen.template zero_hidden<D>(lane, key0, sm.v);
      f32x4 s[2] = {f32x4{}, f32x4{}};
  #pragma unroll
      for (int mt = 0; mt < 2; ++mt)
  #pragma unroll
        for (int dc = 0; dc < DC; ++dc)
          s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kreg[mt][dc], qreg[dc], s[mt], 0, 0, 0);
      // Staged logits go out ahead of the next unit's loads: these are waited for in order,
      // so behind them the stores' way to memory would be waited for on top of theirs (747
      // us behind, 741 ahead).
      if constexpr (kScored) {
        if (n_staged == kStagedUnits || (n_staged > 0 && piece_begins)) store_staged();
      }
      // the next unit's loads, in flight during the math; block ids one further
      if (nxt.valid) {
        load_chunk(id0, id1, tag);
        advance(ids, tag);
        if (ids.valid) ids_of(ids, id0, id1);
      }
      float mloc = -INFINITY;
  #pragma unroll
      for (int mt = 0; mt < 2; ++mt)
  #pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const int key = key0 + 16 * mt + 4 * qd + rr;
          s[mt][rr] = key < cur.len && seen.key(key) ? s[mt][rr] : -INFINITY;
          mloc = fmaxf(mloc, s[mt][rr]);
        }
      if constexpr (kScored) {
        float* keep = logits_at(p, cur.r, g, cur.x, from_unit);
        if (keep != nullptr) {
          if (head_valid) keep_logits(p, staged + n_staged * kUnitKeys * p.group, lane, s);
          if (n_staged++ == 0) staged_to = keep;
        }
      }
      // A unit's probabilities are relative to its own maximum and its O is
      // rescaled in fp32: the largest of every 32 are then exact in bf16, where
      // against the running maximum of a whole range only a few were.  Relative
      // error against float64, 128 sequences of 4.2k-10.8k keys: 0.00227 with
      // running maxima, 0.00218 with one per wave of a 12-wave work-group, 0.00202
      // so, in the same time (the 64 FMAs of a unit hide behind its loads).
      const float m_unit = fmaxf(quad_max(mloc), lowest);
      const float m_new = fmaxf(m_run, m_unit);
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c);
      const float beta = __builtin_amdgcn_exp2f((m_unit - m_new) * c);
      m_run = m_new;
      const float mc = m_unit * c;
      bf16x8 pb;
      float l_unit = 0.f;
  #pragma unroll
      for (int mt = 0; mt < 2; ++mt)
  #pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][rr], c, -mc));
          pb[4 * mt + rr] = (__bf16)e;
          // (scores are sums of fp32 weights, which are normalised by a sum of such; the
          // output then divides rounded probabilities by the unrounded sum, which is as
          // close: 0.00202 relative to float64 both ways, 40 sequences of 5000 keys)
          l_unit += kScored ? e : (float)pb[4 * mt + rr];
        }
      l_run = __builtin_fmaf(l_run, alpha, l_unit * beta);
  #pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_fragment<D>(sm.v, lane, dt), pb, f32x4{}, 0, 0, 0);
  #pragma unroll
        for (int e = 0; e < 4; ++e) oacc[dt][e] = __builtin_fmaf(oacc[dt][e], alpha, o[e] * beta);
      }

      piece_begins = false;
      if (cur.x + 1 == cur.xe) {
        // the piece ends: lane (j, qd) holds dims 16 dt + 4 qd .. +3 of head j
        if (nxt.valid) load_q(nxt.r);
        l_run = quad_sum(l_run);
        if (head_valid) {
          if (cur.slot < 0) {
            uint16_t* orow = p.out + ((size_t)cur.r * p.num_q_heads + h) * D;
  #pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              bf16x4 o;
  #pragma unroll
              for (int e = 0; e < 4; ++e) o[e] = (__bf16)(oacc[dt][e] / l_run);
              *reinterpret_cast<uint2*>(orow + 16 * dt + 4 * qd) = __builtin_bit_cast(uint2, o);
            }
            if constexpr (kScored) {
              const size_t at = ((size_t)g * p.slots + ~cur.slot) * p.group + j;
              if (qd == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * at) = make_float2(m_run, l_run);
            }
          } else {
            const size_t at = ((size_t)g * p.slots + cur.slot) * p.group + j;
  #pragma unroll
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(p.ws_o + at * D + 16 * dt + 4 * qd) = oacc[dt];
            if (qd == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * at) = make_float2(m_run, l_run);
          }
        }
        if constexpr (kScored) {
          if (!nxt.valid && n_staged > 0) store_staged();
          piece_begins = true;
        }
        if (!nxt.valid) return;
        if constexpr (kScored) from_unit = max(0, from_c[nxt.r]) / kUnitKeys;
        reset();
      }
      cur = nxt;
      nxt = ids;
    }
  };
  if (aligned)
    run(std::true_type{});
  else
    run(std::false_type{});
}

// The pieces that decode_ranges_kernel left of sequence r: its first slot and their number.
template <Keys kKeys>
__device__ __forceinline__ int2 pieces_of(const DecParams& p, int r, int lane) {
  const int2 plan = *p.plan;
  const bool aligned = plan.x != 0;
  const int per = plan.y;
  // units before r, or (aligned) pieces before r
  int before = 0;
  for (int s = 0; s < r; s += 64) {
    const int x = s + lane < r ? seen_units<kKeys>(p, p.seq_lens[s + lane]) : 0;
    before += wave_total(aligned ? ceil_div(x, per) : x);
  }
  const int units = seen_units<kKeys>(p, p.seq_lens[r]);
  if (units == 0) return make_int2(0, 0);
  if (aligned) return make_int2(before, ceil_div(units, per));
  const int w0 = before / per;
  return make_int2(r + w0, (before + units - 1) / per - w0 + 1);
}

// Combines the pieces of a sequence and KV head into its output (a sequence of one
// piece has it already).  A sequence without keys gets NaN, as from one work-group per
// pair, or zeros where the call allows such rows.
template <int D, Keys kKeys>
__device__ __forceinline__ void merge_sequence(const DecParams& p, int g, int r, int2 piece) {
  if (piece.y == 1) return;
  const size_t base = ((size_t)g * p.slots + piece.x) * p.group;
  const size_t row = (size_t)r * p.num_q_heads + g * p.group;
  const bool empty = kKeys != Keys::kAll && piece.y == 0;
  merge_pieces<D>(
      p.ws_o, p.ws_ml, p.group, p.scale_log2, [&](int) { return piece.y; },
      [&](int hj, int k) { return base + (size_t)k * p.group + hj; },
      [&](int hj, int d, bf16x4 o) {
        *reinterpret_cast<uint2*>(p.out + (row + hj) * D + d) = __builtin_bit_cast(uint2, empty ? bf16x4{} : o);
      });
}

// One work-group per (sequence, KV head).
template <int D, Keys kKeys>
__global__ __launch_bounds__(kMergeThreads) void decode_ranges_merge_kernel(DecParams p) {
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads;
  merge_sequence<D, kKeys>(p, g, r, pieces_of<kKeys>(p, r, threadIdx.x & 63));
}

// The end of a decode in ranges that adds attention weights to scores: the first
// work-groups, one per (sequence, KV head), merge its pieces, and the others, one per
// kScoreKeys of its scored keys too, turn the logits that the ranges kept into weights.
// Every one of these finds the row statistics (m, l) itself from the pieces'.
constexpr int kScoreKeys = 4 * kMergeThreads;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void decode_scores_kernel(DecParams p) {
  const int lane = threadIdx.x & 63;
  const int pairs = p.batch * p.num_kv_heads;
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads % p.batch;
  if ((int)blockIdx.x < pairs) {
    merge_sequence<D, Keys::kScored>(p, g, r, pieces_of<Keys::kScored>(p, r, lane));
    return;
  }
  const int chunk = blockIdx.x / pairs - 1;
  const int len = p.seq_lens[r];
  const int from = first_scored(p, r, len);
  const long long first = from / kUnitKeys * kUnitKeys + (long long)chunk * kScoreKeys;
  if (from >= len || first >= len) return;
  const int2 piece = pieces_of<Keys::kScored>(p, r, lane);
  __shared__ float2 stat[kMaxGroup];
  const float c = p.scale_log2;
  for (int j = threadIdx.x >> 6; j < p.group; j += kMergeThreads / 64) {
    float m = -INFINITY, l = 0.f;
    for (int k = lane; k < piece.y; k += 64) {
      const size_t at = ((size_t)g * p.slots + piece.x + k) * p.group + j;
      const float2 ml = *reinterpret_cast<const float2*>(p.ws_ml + 2 * at);
      const float m_new = fmaxf(m, ml.x);
      l = l * __builtin_amdgcn_exp2f((m - m_new) * c) + ml.y * __builtin_amdgcn_exp2f((ml.x - m_new) * c);
      m = m_new;
    }
    float m_all = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, o));
    l = m == -INFINITY ? 0.f : l * __builtin_amdgcn_exp2f((m - m_all) * c);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
    if (lane == 0) stat[j] = make_float2(m_all * c, 1.f / l);
  }
  __syncthreads();
  const int key = (int)first + 4 * threadIdx.x;
  if (key + 3 < from || key >= len || (key - from / kUnitKeys * kUnitKeys) / kUnitKeys >= p.logit_units) return;
  f32x4* score = reinterpret_cast<f32x4*>(
      score_at(p, p.block_tables[(size_t)r * p.max_blocks_per_seq + key / kBlock], g, key));
  const f32x4 old = *score;
  const float* logits = logits_at(p, r, g, key / kUnitKeys, from / kUnitKeys) + 4 * (key / 4 % 8) * p.group;
  *score = quad_scores(p, old, quad_weights(p, stat, logits), key, from, len);
}

// Decode with scores, one work-group of four waves per (sequence, KV head): the waves take
// the sequence's units in turn and keep the logits of its scored keys in LDS (those past
// p.lds_units units in the workspace), so that its weights need no memory but the scores.
// Ranges have to write all logits, since a sequence's softmax is known only when all of
// its pieces are done, and the writes cost the stream of reads far more than their bytes:
// 128 sequences of 4.2k-10k keys, 32 / 8 heads of 128, 3.3 GB of K and V and 100 MB of logits,
// 748 us in ranges, 612 here (5.5 TB/s; five, six and eight waves 617, 625 and 638: what is
// read ahead is enough, and the V tiles of more waves leave the logits less room).
constexpr int kScoreWaves = 4;
constexpr int kScoreThreads = 64 * kScoreWaves;
constexpr int kScoreBatch = 256;        // longest sequence first up to this many
constexpr int kScoreQuads = 8;          // quads of keys per thread whose scores are loaded together
template <int D>
__global__ __launch_bounds__(kScoreThreads) void decode_scores_pair_kernel(DecParams p) {
  constexpr int DC = D / 32;
  constexpr int DT = D / 16;
  constexpr int kVLoads = kChunk * D / 8 / 64;
  __shared__ DecLds<D, kScoreWaves> sm;
  __shared__ float2 stat[kMaxGroup];
  __shared__ int lens[kScoreBatch];
  __shared__ int pick;
  extern __shared__ __attribute__((aligned(16))) float kept_logits[];     // [lds_units][8][group][4]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 15;
  const int qd = lane >> 4;
  const int g = blockIdx.x % p.num_kv_heads;
  int r = blockIdx.x / p.num_kv_heads;
  if (p.batch <= kScoreBatch) {
    // (the order of paged_decode_attn_kernel)
    for (int s = threadIdx.x; s < p.batch; s += kScoreThreads) lens[s] = p.seq_lens[s];
    __syncthreads();
    for (int s = threadIdx.x; s < p.batch; s += kScoreThreads) {
      const int mine = lens[s];
      int rank = 0;
      for (int t = 0; t < p.batch; ++t) rank += (lens[t] > mine) || (lens[t] == mine && t < s);
      if (rank == r) pick = s;
    }
    __syncthreads();
    r = pick;
  }
  r = __builtin_amdgcn_readfirstlane(r);
  const ScalarInts bt = (ScalarInts)(p.block_tables + (size_t)r * p.max_blocks_per_seq);
  const int len = __builtin_amdgcn_readfirstlane(p.seq_lens[r]);
  const int from = __builtin_amdgcn_readfirstlane(first_scored(p, r, len));
  const int from_unit = from / kUnitKeys;
  const int units = units_of(len);
  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const uint16_t* kbase = p.k_pool + (size_t)g * tile_elems;
  const uint16_t* vbase = p.v_pool + (size_t)g * tile_elems;
  const bool head_valid = j < p.group;
  const int h = g * p.group + (head_valid ? j : 0);
  const float c = p.scale_log2;
  const float lowest = lowest_reference(c);      // as in decode_ranges_kernel
  bf16x8 qreg[DC];
#pragma unroll
  for (int dc = 0; dc < DC; ++dc) {
    qreg[dc] = bf16x8{};
    if (head_valid)
      qreg[dc] = *reinterpret_cast<const bf16x8*>(p.q + ((size_t)r * p.num_q_heads + h) * D + 32 * dc + 8 * qd);
  }
  f32x4 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{};
  float m_run = -INFINITY, l_run = 0.f;
  const int last_blk = (len - 1) / kBlock;
  int id0 = 0, id1 = 0;
  auto ids_of = [&](int x) {
    id0 = bt[min(x * kUnitBlocks, last_blk)];
    id1 = bt[min(x * kUnitBlocks + 1, last_blk)];
  };
  bf16x8 kreg[2][DC];
  bf16x8 vreg[kVLoads];
  uint16_t* tile = sm.v[wave];
  if (wave < units) {
    ids_of(wave);
    load_chunk_tiles<D, kNonTemporal>(kbase, vbase, id0, id1, slot_elems, lane, kreg, vreg);
    ids_of(wave + kScoreWaves);
  }
  for (int x = wave; x < units; x += kScoreWaves) {
    const int key0 = x * kUnitKeys;
    store_v_tile<D>(vreg, lane, key0, len, tile);
    f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int dc = 0; dc < DC; ++dc)
        s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kreg[mt][dc], qreg[dc], s[mt], 0, 0, 0);
    if (x + kScoreWaves < units) {
      load_chunk_tiles<D, kNonTemporal>(kbase, vbase, id0, id1, slot_elems, lane, kreg, vreg);
      ids_of(x + 2 * kScoreWaves);
    }
    float mloc = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int key = key0 + 16 * mt + 4 * qd + rr;
        s[mt][rr] = key < len ? s[mt][rr] : -INFINITY;
        mloc = fmaxf(mloc, s[mt][rr]);
      }
    const int u = x - from_unit;
    if (u >= 0 && u < p.lds_units) {
      if (head_valid) keep_logits(p, kept_logits + u * kUnitKeys * p.group, lane, s);
    } else if (float* keep = logits_at(p, r, g, x, from_unit); keep != nullptr && head_valid) {
      keep_logits(p, keep, lane, s);
    }
    const float m_unit = fmaxf(quad_max(mloc), lowest);
    const float m_new = fmaxf(m_run, m_unit);
    const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c);
    const float beta = __builtin_amdgcn_exp2f((m_unit - m_new) * c);
    m_run = m_new;
    const float mc = m_unit * c;
    bf16x8 pb;
    float l_unit = 0.f;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][rr], c, -mc));
        pb[4 * mt + rr] = (__bf16)e;
        l_unit += e;
      }
    l_run = __builtin_fmaf(l_run, alpha, l_unit * beta);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_fragment<D>(tile, lane, dt), pb, f32x4{}, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) oacc[dt][e] = __builtin_fmaf(oacc[dt][e], alpha, o[e] * beta);
    }
  }

  // the scores of the first quads, in flight during the merge
  const int first = from / 4 * 4;
  const int last = from < len ? (int)min((long long)len, (long long)(from_unit + p.logit_units) * kUnitKeys) : 0;
  f32x4* at[kScoreQuads];
  f32x4 old[kScoreQuads];
  auto load_scores = [&](int key0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kScoreQuads; ++i) {
      const int key = key0 + 4 * ((int)threadIdx.x + i * kScoreThreads);
      at[i] = reinterpret_cast<f32x4*>(score_at(p, p.block_tables[(size_t)r * p.max_blocks_per_seq + min(key, last - 1) / kBlock],
                                                g, key));
    }
#pragma unroll
    for (int i = 0; i < kScoreQuads; ++i) old[i] = *at[i];
  };
  if (first < last) load_scores(first);
  l_run = quad_sum(l_run);
  __syncthreads();                     // every wave is done with its V tile
  if (qd == 0) {
    sm.merge.m[wave][j] = m_run;
    sm.merge.l[wave][j] = l_run;
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) sm.merge.o[wave][j][16 * dt + 4 * qd + rr] = oacc[dt][rr];
  __syncthreads();
  for (int idx = threadIdx.x; idx < p.group * D; idx += kScoreThreads) {
    const int hj = idx / D;
    const int d = idx % D;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < kScoreWaves; ++w) mx = fmaxf(mx, sm.merge.m[w][hj]);
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < kScoreWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f((sm.merge.m[w][hj] - mx) * c);   // 0 for idle waves
      num += wt * sm.merge.o[w][hj][d];
      den += wt * sm.merge.l[w][hj];
    }
    // a row of an empty sequence (a padded batch) is zero
    p.out[((size_t)r * p.num_q_heads + g * p.group + hj) * D + d] =
        __builtin_bit_cast(uint16_t, (__bf16)(len > 0 ? num / den : 0.f));
    if (d == 0) stat[hj] = make_float2(mx * c, 1.f / den);
  }
  __syncthreads();
  for (int key0 = first; key0 < last; key0 += 4 * kScoreQuads * kScoreThreads) {
    if (key0 != first) load_scores(key0);
#pragma unroll
    for (int i = 0; i < kScoreQuads; ++i) {
      const int key = key0 + 4 * ((int)threadIdx.x + i * kScoreThreads);
      if (key >= last) break;
      const int u = key / kUnitKeys - from_unit;
      const float* logits = u < p.lds_units ? kept_logits + u * kUnitKeys * p.group
                                            : logits_at(p, r, g, key / kUnitKeys, from_unit);
      *at[i] = quad_scores(p, old[i], quad_weights(p, stat, logits + 4 * (key / 4 % 8) * p.group), key, from, len);
    }
  }
}

// One work-group per (sequence, KV head): the final output of cascade decode
// from every partial of the row (shared-prefix chunks, own-key segments).
// The maxima and sums of all partials are gathered into LDS by all threads
// at once, turned into per-partial weights, and every thread then sums its
// output elements over the partials with the loads issued together.
template <int D>
__global__ __launch_bounds__(kThreads) void cascade_merge_kernel(DecParams p) {
  extern __shared__ float wsm[];            // [group][parts]: maxima, then weights
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads;
  const int L = p.seq_lens[r];
  const int shared = shared_len_of(p, r);
  const int n_shared = (shared + p.chunk_keys - 1) / p.chunk_keys;
  const int n_own = (L - shared + kCascadeSegmentKeys - 1) / kCascadeSegmentKeys;
  const int n = n_shared + n_own;
  const int stride = p.chunks + p.segments;     // row length of wsm
  float* m_s = wsm;
  float* l_s = wsm + p.group * stride;
  const float c = p.scale_log2;
  const size_t row0 = (size_t)r * p.num_q_heads + g * p.group;
  auto part_of = [&](int i) { return i < n_shared ? i : p.chunks + (i - n_shared); };
  for (int t = threadIdx.x; t < p.group * n; t += kThreads) {
    const int hj = t / n, i = t % n;
    const float2 ml = *reinterpret_cast<const float2*>(p.ws_ml + 2 * ((size_t)part_of(i) * p.ws_rows + row0 + hj));
    m_s[hj * stride + i] = ml.x;
    l_s[hj * stride + i] = ml.y;
  }
  __syncthreads();
  if ((int)threadIdx.x < p.group) {
    const int hj = threadIdx.x;
    float mx = -INFINITY;
    for (int i = 0; i < n; ++i) mx = fmaxf(mx, m_s[hj * stride + i]);
    float den = 0.f;
    for (int i = 0; i < n; ++i) {
      const float wt = __builtin_amdgcn_exp2f((m_s[hj * stride + i] - mx) * c);
      m_s[hj * stride + i] = wt;              // the maximum becomes the weight
      den += wt * l_s[hj * stride + i];
    }
    const float inv = 1.f / den;
    for (int i = 0; i < n; ++i) m_s[hj * stride + i] *= inv;
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < p.group * D; idx += kThreads) {
    const int hj = idx / D;
    const int d = idx % D;
    const size_t row = row0 + hj;
    float acc = 0.f;
    int i = 0;
    for (; i + 4 <= n; i += 4) {
      float o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = p.ws_o[((size_t)part_of(i + u) * p.ws_rows + row) * D + d];
#pragma unroll
      for (int u = 0; u < 4; ++u) acc += m_s[hj * stride + i + u] * o[u];
    }
    for (; i < n; ++i) acc += m_s[hj * stride + i] * p.ws_o[((size_t)part_of(i) * p.ws_rows + row) * D + d];
    p.out[row * D + d] = __builtin_bit_cast(uint16_t, (__bf16)acc);
  }
}

}  // namespace

// Ranges or one work-group per (sequence, KV head): ranges win from a few
// hundred keys on, at every batch.  us a call back to back, one work-group per pair
// -> ranges with their merge: 32 / 8 heads of 128, 2 sequences of 84-140 keys 11.1 ->
// 8.2, 3 of 2000-6000 49 -> 14, 24 of 500-9000 115 -> 67, 128 of 100-500 67 -> 35, 128 of
// 4200-10800 676 -> 616; 32 / 8 heads of 64, 128 of 2000-6000 210 -> 181.
// At head_dim 64 up to 512 keys, while the pairs fit one round, the merge launch is
// not paid for (8 sequences of 100-500 keys 8.5 -> 8.6).  Past 512 a full round of
// pairs of nearly equal lengths still loses up to 1.3 us to it, ragged ones gain (32
// sequences, 32 / 8 heads: 448-560 keys 10.6 -> 11.4, 112-560 9.9 -> 9.6, 1600-2000
// 23.9 -> 24.8, 400-2000 20.4 -> 19.5).
DecodeGeometry decode_geometry(int batch, int max_seq_len, int num_kv_heads, int head_dim, int cus) {
  DecodeGeometry geo = {};
  if (batch < 1 || batch > kRangeMaxBatch || max_seq_len <= 128) return geo;
  if (head_dim == 64 && max_seq_len <= 512 && (long long)batch * num_kv_heads <= cus) return geo;
  const int groups_per_cu = head_dim == 128 ? kRangeGroupsPerCu128 : kRangeGroupsPerCu64;
  geo.ranges = std::max(1, groups_per_cu * cus / num_kv_heads);
  const int rounds = aligned_rounds(64) * aligned_rounds(128);     // a whole number of waves at both
  const int pieces = rounds * std::max(1, kAlignedPiecesPerCu / rounds * cus / num_kv_heads);
  geo.aligned_ranges = pieces / aligned_rounds(head_dim);
  geo.slots = std::max(geo.ranges, pieces) + batch;
  return geo;
}

namespace {

// LDS of a compute unit, and of decode_scores_pair_kernel without the logits
constexpr int kLdsBytes = 160 * 1024;
constexpr int pair_lds_bytes(int head_dim) {
  return (head_dim == 128 ? (int)sizeof(DecLds<128, kScoreWaves>) : (int)sizeof(DecLds<64, kScoreWaves>)) +
         kMaxGroup * (int)sizeof(float2) + kScoreBatch * (int)sizeof(int) + 256;
}

// work-groups of decode_scores_kernel per (sequence, KV head) that turn logits into weights
long long score_chunks(long long logit_units) { return (logit_units * kUnitKeys + kScoreKeys - 1) / kScoreKeys; }

template <int D, Keys kKeys>
void launch_decode(const DecodeLaunch& a, const DecParams& p, hipStream_t stream) {
  const unsigned rows = (unsigned)((long long)a.batch * a.num_kv_heads);
  if constexpr (kKeys == Keys::kScored) {
    if (a.ranges == 0) {
      DecParams pair = p;
      const int unit_bytes = kUnitKeys * p.group * (int)sizeof(float);
      pair.lds_units = std::min(a.logit_units, (kLdsBytes - pair_lds_bytes(D)) / unit_bytes);
      hipLaunchKernelGGL(decode_scores_pair_kernel<D>, dim3(rows), dim3(kScoreThreads),
                         (size_t)pair.lds_units * unit_bytes, stream, pair);
      return;
    }
  } else if (a.ranges == 0) {
    hipLaunchKernelGGL((paged_decode_attn_kernel<D, kKeys>), dim3(rows), dim3(64 * kDecodeWaves), 0, stream, p);
    return;
  }
  const dim3 grid((unsigned)(std::max(a.ranges, a.aligned_ranges) * a.num_kv_heads)), block(64);
  const size_t staged = kKeys == Keys::kScored ? kStagedUnits * kUnitKeys * p.group * sizeof(float) : 0;
  hipLaunchKernelGGL((decode_ranges_kernel<D, kKeys>), grid, block, staged, stream, p);
  if constexpr (kKeys == Keys::kScored) {
    const unsigned chunks = (unsigned)score_chunks(a.logit_units);
    hipLaunchKernelGGL(decode_scores_kernel<D>, dim3(rows * (1 + chunks)), dim3(kMergeThreads), 0, stream, p);
  } else {
    hipLaunchKernelGGL((decode_ranges_merge_kernel<D, kKeys>), dim3(rows), dim3(kMergeThreads), 0, stream, p);
  }
}

template <int D>
void launch_decode(const DecodeLaunch& a, const DecParams& p, hipStream_t stream) {
  if (a.score_pool != nullptr)
    launch_decode<D, Keys::kScored>(a, p, stream);
  else if (a.win.size > 0)
    launch_decode<D, Keys::kWindow>(a, p, stream);
  else
    launch_decode<D, Keys::kAll>(a, p, stream);
}

}  // namespace

bool decode_fits(const DecodeGeometry& geo, int batch, int num_kv_heads, long long logit_units) {
  const double pairs = (double)batch * num_kv_heads;
  if (geo.ranges == 0) return launch_fits(pairs, logit_units < 0 ? 64 * kDecodeWaves : kScoreThreads);
  return launch_fits((double)std::max(geo.ranges, geo.aligned_ranges) * num_kv_heads, 64) &&
         launch_fits(pairs * (1 + (logit_units < 0 ? 0 : score_chunks(logit_units))), kMergeThreads);
}

hipError_t launch_paged_decode_attn(const DecodeLaunch& a, hipStream_t stream) {
  DecParams p = {};
  p.q = a.q;
  p.k_pool = a.k_pool;
  p.v_pool = a.v_pool;
  p.block_tables = a.block_tables;
  p.seq_lens = a.seq_lens;
  p.out = a.out;
  p.max_blocks_per_seq = a.max_blocks_per_seq;
  p.num_q_heads = a.num_q_heads;
  p.num_kv_heads = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.scale_log2 = a.scale * kLog2e;
  p.batch = a.batch;
  p.window = a.win.size;
  p.sinks = a.win.sinks;
  p.score_from = a.score_from;
  p.score_pool = a.score_pool;
  p.decay = a.decay;
  p.logits = a.logits;
  p.logit_units = a.logit_units;
  if (a.ranges > 0) {
    p.ranges = a.ranges;
    p.aligned_ranges = a.aligned_ranges;
    p.slots = a.slots;
    p.ws_o = static_cast<float*>(a.workspace);
    p.ws_ml = p.ws_o + (size_t)a.slots * a.num_q_heads * a.head_dim;
    p.plan = reinterpret_cast<int2*>(p.ws_ml + (size_t)a.slots * a.num_q_heads * 2);
  }
  if (a.head_dim == 128)
    launch_decode<128>(a, p, stream);
  else
    launch_decode<64>(a, p, stream);
  return hipGetLastError();
}

hipError_t launch_cascade_decode_rest(const CascadeLaunch& a, hipStream_t stream) {
  const CascadeGeometry geo = cascade_geometry(a.num_groups, a.max_group_seqs, a.max_shared_len,
                                               a.max_rest_len, a.num_q_heads, a.num_kv_heads);
  DecParams p = {};
  p.q = a.q;
  p.k_pool = a.k_pool;
  p.v_pool = a.v_pool;
  p.block_tables = a.block_tables;
  p.seq_lens = a.seq_lens;
  p.out = a.out;
  p.max_blocks_per_seq = a.max_blocks_per_seq;
  p.num_q_heads = a.num_q_heads;
  p.num_kv_heads = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.scale_log2 = a.scale * kLog2e;
  p.cu_groups = a.cu_groups;
  p.shared_lens = a.shared_lens;
  p.num_groups = a.num_groups;
  p.batch = a.batch;
  p.chunk_keys = geo.chunk_keys;
  p.chunks = geo.chunks;
  p.segments = geo.segments;
  p.ws_o = a.ws_o;
  p.ws_ml = a.ws_ml;
  p.ws_rows = a.batch * a.num_q_heads;
  const long long rows = (long long)a.batch * a.num_kv_heads;
  if (geo.segments > 0) {
    const dim3 grid((unsigned)(rows * geo.segments)), block(64 * kCascadeWaves);
    if (a.head_dim == 128) {
      hipLaunchKernelGGL((paged_decode_attn_kernel<128, Keys::kCascade>), grid, block, 0, stream, p);
    } else {
      hipLaunchKernelGGL((paged_decode_attn_kernel<64, Keys::kCascade>), grid, block, 0, stream, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const size_t lds = 2 * sizeof(float) * (size_t)p.group * (geo.chunks + geo.segments);
  if (a.head_dim == 128) {
    hipLaunchKernelGGL(cascade_merge_kernel<128>, dim3((unsigned)rows), dim3(kThreads), lds, stream, p);
  } else {
    hipLaunchKernelGGL(cascade_merge_kernel<64>, dim3((unsigned)rows), dim3(kThreads), lds, stream, p);
  }
  return hipGetLastError();
}

}  // namespace cs
