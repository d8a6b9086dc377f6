// Attention weights of a prompt's rows, added up per key, for gfx950.
//
// Eviction by accumulated attention weight keeps the keys that the queries so far gave
// the most weight.  During decode the decode kernels add a token's weights
// (paged_decode_attn.hip); here the last rows of every invocation's suffix add theirs
// after a prefill.  With n observed rows, of G query heads per KV head,
//
//   w[g][j] = sum over the G n rows of softmax_j(scale q . K_j),   j <= the row's position
//
// Two passes over the logits S = K Q^T, each an MFMA product, since a row's weights
// need its maximum and sum over all keys first:
//   * key_stats_kernel: a wave holds 32 rows as the B operand (stacked: token major, the
//     heads of the group fastest, so that 32 rows are a few neighbouring tokens), a
//     work-group of four waves shares the K tiles in LDS, and each lane keeps its row's
//     running maximum and sum; few rows are split over key parts on more work-groups,
//     which key_stats_merge_kernel combines.
//   * key_weights_kernel: a wave holds 32 keys as the A operand, the work-group's waves
//     share the Q tiles in LDS, and each lane adds its rows' weights for 16 keys; one
//     reduction over the lanes at the end gives the sums, which one lane per key adds to
//     the score.  A key belongs to one wave, so there are no atomics and the result is
//     the same from run to run.
#include "direct_lds.h"
#include "internal.h"
#include "wave_ops.h"

#include <float.h>
#include <math.h>

#include <algorithm>

namespace cs {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kBlock = 16;
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 32;                  // rows or keys per wave and MFMA tile
constexpr int kStatRows = kTile * kWaves;  // stacked rows of a statistics work-group
constexpr int kStep = 64;                  // keys per step there
constexpr int kWeightKeys = kTile * kWaves;  // keys of a weights work-group
constexpr int kStageRows = 64;             // stacked rows per step there
constexpr int kFewRows = 512;              // stacked rows whose statistics that merges itself
constexpr int kPartTiles = 32;             // row tiles of a weights work-group, where there is room for more
constexpr float kLog2e = 1.4426950408889634f;

struct ScoreParams {
  const uint16_t* q;
  const uint16_t* k_pool;
  const int32_t* block_tables;
  const int32_t* prefix_lens;
  const int32_t* cu_q_lens;
  const int32_t* score_from;
  float* score_pool;
  float2* stats;              // [parts][batch][num_kv_heads][max_rows * group]: (m c, l), then (m c, 1 / l)
  int batch;
  int max_blocks_per_seq;
  int num_q_heads;
  int num_kv_heads;
  int group;
  // x / group = __umulhi(x, group_magic) + (x & group_one) for x group < 2^32: the magic is
  // ceil(2^32 / group), and 0 for a group of one head, which the mask stands for
  unsigned group_magic, group_one;
  int rows;                   // observed rows per invocation (the last ones)
  int max_rows;               // of any invocation
  int parts;
  int tiles;                  // work-groups per (invocation, KV head)
  int key_tiles;              // of the longest invocation
  float* partials;            // [batch * num_kv_heads][tiles][kWeightKeys], where rows are split
  float scale_log2;
  float decay;
};

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ void pair_swap(float x, float& a, float& b) {
  a = x;
  b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
}

// A value that all lanes hold, in a scalar register (a loaded one would make the branches
// and descriptors that depend on it a loop over the lanes)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Between two steps: the wave's loads into one buffer have landed and its reads of the other are
// done (the products that take them need not be, and the barrier alone does not wait for reads), and
// so are all waves'.
__device__ __forceinline__ void buffers_ready() {
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  __builtin_amdgcn_s_waitcnt(kWaitLgkmcnt0);
  asm volatile("s_barrier" ::: "memory");
}

// An invocation: its observed rows are the stacked rows 0 .. n * group - 1 of a KV head;
// row rho is head rho % group of the token at position pos0 + rho / group.
struct Observed {
  int r, g, q0, n, pos0, len, prefix;
  __device__ __forceinline__ Observed(const ScoreParams& p, int r_, int g_) : r(r_), g(g_) {
    const int first = uniform(p.cu_q_lens[r]);
    const int s = uniform(p.cu_q_lens[r + 1]) - first;
    prefix = uniform(p.prefix_lens[r]);
    len = prefix + s;
    n = min(s, p.rows);
    q0 = first + s - n;
    pos0 = len - n;
  }
  __device__ __forceinline__ const uint16_t* q_row(const ScoreParams& p, int rho, int d) const {
    return p.q + ((size_t)(q0 + rho / p.group) * p.num_q_heads + g * p.group + rho % p.group) * d;
  }
  __device__ __forceinline__ size_t stat(const ScoreParams& p, int part) const {
    return (((size_t)part * p.batch + r) * p.num_kv_heads + g) * ((size_t)p.max_rows * p.group);
  }
};

// The lane's part of staging rows of D elements into LDS (DirectLayout): the row of a
// 1 KB group it fetches from, and the element there.
template <int D>
struct Staging {
  int row, elem;
  __device__ __forceinline__ explicit Staging(int lane)
      : row(lane / (D / 8)), elem(8 * ((lane % (D / 8)) ^ DirectLayout<D>::swz(lane / (D / 8)))) {}
};

// An MFMA operand of 32 staged rows: the lane's row of each 32-row tile, dims 16 ks + 8 half .. +7.
template <int D>
struct Operand {
  static constexpr int kOffs = D == 128 ? 4 : D / 16;
  static constexpr int kGrp = DirectLayout<D>::kGrp;
  int off[kOffs];
  __device__ __forceinline__ Operand(int qi, int half) {
#pragma unroll
    for (int k = 0; k < kOffs; ++k) {
      if constexpr (D == 128)
        off[k] = (qi >> 2) * kGrp + (qi & 3) * D + 8 * half + 32 * (k ^ (qi & 3));
      else
        off[k] = (qi >> 3) * kGrp + (qi & 7) * D + 8 * ((2 * k + half) ^ DirectLayout<D>::swz(qi & 7));
    }
  }
  __device__ __forceinline__ bf16x8 at(const uint16_t* buf, int ks, int tile) const {
    const uint16_t* x;
    if constexpr (D == 128) x = &buf[tile * 8 * kGrp + 16 * (ks & 1) + off[ks >> 1]];
    else x = &buf[tile * 4 * kGrp + off[ks]];
    return as_bf16x8(*reinterpret_cast<const uint4*>(x));
  }
};

template <int D>
__global__ __launch_bounds__(kThreads, 4) void key_stats_kernel(ScoreParams p) {
  using DL = DirectLayout<D>;
  constexpr int KS = D / 16;
  constexpr int kGrp = DL::kGrp;
  constexpr int kLoads = kBlock / DL::kRows;
  constexpr int kGroupElems = DL::kRows * D;
  constexpr int kBuf = (kStep / DL::kRows) * kGrp;
  __shared__ __attribute__((aligned(16))) uint16_t k0[kBuf], k1[kBuf];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qi = lane & 31, half = lane >> 5;
  int rest = blockIdx.x;
  const int g = rest % p.num_kv_heads;
  rest /= p.num_kv_heads;
  // the rows with most keys first; an invocation's together, which share its K
  const int tile = p.tiles - 1 - rest % p.tiles;
  rest /= p.tiles;
  const int part = rest % p.parts;
  const Observed ob(p, rest / p.parts, g);
  const int n_rows = ob.n * p.group;
  if (tile * kStatRows >= n_rows) return;
  const int rho = tile * kStatRows + wave * kTile + qi;
  const bool valid = rho < n_rows;
  const int pos = valid ? ob.pos0 + rho / p.group : ob.len - 1;
  const int last = min(n_rows, (tile + 1) * kStatRows) - 1;
  const int kv_end = ob.pos0 + last / p.group + 1;       // keys the work-group's rows see
  const int wave_first = min(tile * kStatRows + wave * kTile, n_rows - 1);
  const int pos_min = uniform(ob.pos0 + wave_first / p.group);
  const int steps = ceil_div(kv_end, kStep);
  const int s0 = uniform(steps * part / p.parts);        // (at most 32 parts)
  const int s1 = uniform(steps * (part + 1) / p.parts);

  bf16x8 qreg[KS];
  const uint16_t* qrow = ob.q_row(p, valid ? rho : 0, D);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + half * 8));

  // wave w loads pool block 4 step + w; a block past the end loads the last one (its keys are masked)
  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const uint16_t* kbase = p.k_pool + (size_t)g * tile_elems;
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(p.block_tables + (size_t)ob.r * p.max_blocks_per_seq);
  const int last_blk = uniform((ob.len - 1) / kBlock);
  auto block_id = [&](int step) { return uniform(bt[min(step * (kStep / kBlock) + wave, last_blk)]); };
  const Staging<D> lane_at(lane);
  const int dma_off = lane_at.row * D + lane_at.elem;
  auto dma = [&](uint16_t* buf, int id) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(kbase + (size_t)id * slot_elems), (short)0, (int)(tile_elems * sizeof(uint16_t)), kRawBufferWord3);
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rs, (__attribute__((address_space(3))) void*)(buf + (kLoads * wave + u) * kGrp), 16, 2 * dma_off,
          2 * u * kGroupElems, 0, 0);
  };
  const Operand<D> op(qi, half);

  const float c = p.scale_log2;
  // finite, so that keys a row does not see weigh 0 and not NaN
  float m = lowest_reference(c);
  float l[4] = {0.f, 0.f, 0.f, 0.f};
  auto compute = [&](int step, const uint16_t* buf) __attribute__((always_inline)) {
    f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op.at(buf, ks, mt), qreg[ks], s[mt], 0, 0, 0);
    const int kstart = step * kStep;
    if (kstart + kStep - 1 > pos_min) {
      const int lim = pos - kstart - 4 * half;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[mt][rr] = mt * 32 + 8 * (rr >> 2) + (rr & 3) <= lim ? s[mt][rr] : -INFINITY;
    }
    // Each lane half keeps the statistics of its own keys until the end.  The reference m
    // is the maximum of some earlier step: sums of weights relative to it are as exact as to
    // the true maximum, as long as they stay in range, so the maximum of a step is only
    // taken when a sum would not (at the first step always).
    auto sums = [&](float mc, float (&to)[4]) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = l[e];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) to[rr & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][rr], c, -mc));
    };
    float sum[4];
    sums(m * c, sum);
    const bool large = !(fmaxf(fmaxf(sum[0], sum[1]), fmaxf(sum[2], sum[3])) < 0x1p100f);
    if (__builtin_amdgcn_ballot_w64(large) != 0) {
      float mx = s[0][0];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) mx = fmaxf(mx, s[mt][rr]);
      const float m_new = fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f((m - m_new) * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) l[e] *= alpha;
      m = m_new;
      sums(m * c, sum);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) l[e] = sum[e];
  };
  // step j: its K has landed; the loads of step j + 1 go into the other buffer, read last
  // in step j - 1 (rings of three and four buffers, with their loads further ahead, gain
  // nothing: 198 us with two, 200 and 206 with three and four, for work-groups fewer to a CU)
  auto run_step = [&](int j, uint16_t* cur, uint16_t* next, int& id) __attribute__((always_inline)) {
    buffers_ready();
    if (j + 1 < s1) dma(next, id);
    id = block_id(j + 2);
    compute(j, cur);
  };
  if (s0 < s1) {
    dma(k0, block_id(s0));
    int id = block_id(s0 + 1);
    for (int j = s0; j < s1; j += 2) {
      run_step(j, k0, k1, id);
      if (j + 1 < s1) run_step(j + 1, k1, k0, id);
    }
  }
  const float l_half = (l[0] + l[1]) + (l[2] + l[3]);
  float m0, m1, l0, l1;
  pair_swap(m, m0, m1);
  pair_swap(l_half, l0, l1);
  const float m_all = fmaxf(m0, m1);
  const float l_all = l0 * __builtin_amdgcn_exp2f((m0 - m_all) * c) + l1 * __builtin_amdgcn_exp2f((m1 - m_all) * c);
  if (valid && half == 0) p.stats[ob.stat(p, part) + rho] = make_float2(m_all * c, p.parts == 1 ? 1.f / l_all : l_all);
}

// The statistics of a row split over key parts, `stride` apart; their loads in flight together.
__device__ __forceinline__ float2 merged_stats(const ScoreParams& p, const float2* first, size_t stride) {
  constexpr int kAtOnce = 8;
  float m = -FLT_MAX, l = 0.f;
  for (int k0 = 0; k0 < p.parts; k0 += kAtOnce) {
    float2 ml[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      ml[k] = k0 + k < p.parts ? first[(k0 + k) * stride] : make_float2(-FLT_MAX, 0.f);
    float m_new = m;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) m_new = fmaxf(m_new, ml[k].x);
    l *= __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) l += ml[k].y * __builtin_amdgcn_exp2f(ml[k].x - m);
  }
  return make_float2(m, 1.f / l);
}

// All of them, into part 0.
__global__ __launch_bounds__(64) void key_stats_merge_kernel(ScoreParams p) {
  const size_t all = (size_t)p.batch * p.num_kv_heads * p.max_rows * p.group;
  const size_t at = (size_t)blockIdx.x * 64 + threadIdx.x;
  if (at < all) p.stats[at] = merged_stats(p, p.stats + at, all);
}

// The first scored key of an invocation, its length if there is none (score_from may be any
// number from 0 on, and what follows adds to it).
__device__ __forceinline__ int first_scored(const ScoreParams& p, const Observed& ob) {
  return min(max(0, p.score_from[ob.r]), ob.len);
}

// How the scored keys of an invocation are dealt to its p.tiles work-groups: kWeightKeys
// each, and, where work-groups are left (the longest invocation, scored from its first
// key on, has one per key tile), with their rows in parts of at least kPartTiles tiles.
// Work-group w takes part w / key_tiles of key tile w % key_tiles.
struct Dealt {
  int key_tiles, row_tiles, parts;
  __device__ __forceinline__ Dealt(const ScoreParams& p, const Observed& ob, int from) {
    key_tiles = from < ob.len ? ceil_div(ob.len - from / kBlock * kBlock, kWeightKeys) : 0;
    row_tiles = ceil_div(ob.n * p.group, kTile);
    parts = key_tiles == 0 ? 0 : max(1, min(p.tiles / key_tiles, ceil_div(row_tiles, kPartTiles)));
  }
};

// The sum of a key's weights into its score
__device__ __forceinline__ void add_to_score(const ScoreParams& p, const Observed& ob, const int32_t* bt, int key, float w) {
  float* score = p.score_pool + ((size_t)bt[key / kBlock] * p.num_kv_heads + ob.g) * kBlock + key % kBlock;
  *score = key < ob.prefix ? __builtin_fmaf(p.decay, *score, w) : w;
}

// kMerges: the statistics are still in key parts (of at most kFewRows rows), and every
// work-group merges them for itself into LDS while its first loads are on their way, which
// saves a launch (us a call, 64 / 8 heads of 128, the last 32 rows of 4 invocations of 4608 keys
// 26.3 -> 24.5; 32 / 8, 16 rows of one of 8064 18.1 -> 16.4).
template <int D, bool kMerges>
__global__ __launch_bounds__(kThreads, 4) void key_weights_kernel(ScoreParams p) {
  using DL = DirectLayout<D>;
  constexpr int KS = D / 16;
  constexpr int kGrp = DL::kGrp;
  constexpr int kTiles = kStageRows / kTile;
  constexpr int kGroups = kStageRows / DL::kRows;       // 1 KB loads per stage
  constexpr int kLoads = kGroups / kWaves;
  __shared__ __attribute__((aligned(16))) uint16_t q0[kGroups * kGrp], q1[kGroups * kGrp];
  __shared__ float2 few[kMerges ? kFewRows : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int qi = lane & 31, half = lane >> 5;
  int rest = blockIdx.x;
  const int g = rest % p.num_kv_heads;
  rest /= p.num_kv_heads;
  const Observed ob(p, rest / p.tiles, g);
  const int from = uniform(first_scored(p, ob));
  const int n_rows = ob.n * p.group;
  const Dealt dealt(p, ob, from);
  const int wg = rest % p.tiles;
  if (n_rows == 0 || wg >= dealt.parts * dealt.key_tiles) return;
  const int part = uniform(wg / dealt.key_tiles);
  // keys from the first scored block on
  const int key0 = from / kBlock * kBlock + uniform(wg % dealt.key_tiles) * kWeightKeys;
  const int wkey = key0 + wave * kTile;                  // the wave's keys
  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const int32_t* bt = p.block_tables + (size_t)ob.r * p.max_blocks_per_seq;
  const int last_blk = uniform((ob.len - 1) / kBlock);
  bf16x8 kreg[KS];
  {
    const int key = wkey + qi;
    const uint16_t* row = p.k_pool + (size_t)bt[min(key / kBlock, last_blk)] * slot_elems + (size_t)g * tile_elems +
                          (key % kBlock) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(row + ks * 16 + half * 8));
  }
  // row tiles: from `first` on some row sees a key of the work-group, from `seen` on one of
  // the wave; from `whole` on every row sees all of the wave's keys
  const int all_first = max(0, key0 - ob.pos0) * p.group / kTile;
  const int stages = ceil_div(dealt.row_tiles - all_first, kTiles);
  const int first = all_first + uniform(stages * part / dealt.parts) * kTiles;
  const int tiles = min(dealt.row_tiles, all_first + uniform(stages * (part + 1) / dealt.parts) * kTiles);
  const int seen = max(0, wkey - ob.pos0) * p.group / kTile;
  const int whole = ceil_div(max(0, wkey + kTile - 1 - ob.pos0) * p.group, kTile);
  const float2* stats = p.stats + ob.stat(p, 0);
  const Staging<D> lane_at(lane);
  auto token_of = [&](int rho) {
    return (int)(__umulhi((unsigned)rho, p.group_magic) + ((unsigned)rho & p.group_one));
  };
  auto dma = [&](uint16_t* buf, int t) __attribute__((always_inline)) {
    // offsets from the stage's first token
    const int token0 = __builtin_amdgcn_readfirstlane(token_of(min(t * kTile, n_rows - 1)));
    const uint16_t* base = p.q + ((size_t)(ob.q0 + token0) * p.num_q_heads + g * p.group) * D;
    const long long left = (long long)(ob.n - token0) * p.num_q_heads * D * (long long)sizeof(uint16_t);
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)min(left, 0x7fffffffLL), kRawBufferWord3);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int rho = min(t * kTile + (kLoads * wave + u) * DL::kRows + lane_at.row, n_rows - 1);
      const int token = token_of(rho);
      const int off = ((token - token0) * p.num_q_heads + rho - token * p.group) * D + lane_at.elem;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rs, (__attribute__((address_space(3))) void*)(buf + (kLoads * wave + u) * kGrp), 16, 2 * off, 0, 0, 0);
    }
  };
  const Operand<D> op(qi, half);
  const float c = p.scale_log2;
  f32x16 acc = f32x16{};
  const __amdgpu_buffer_rsrc_t stats_rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)stats, (short)0, 8 * n_rows, kRawBufferWord3);
  struct Stats {
    float2 row[kTiles];
  };
  auto load_stats = [&](int t) __attribute__((always_inline)) {
    Stats st;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      const int rho = (t + x) * kTile + qi;
      if constexpr (kMerges)
        st.row[x] = rho < n_rows ? few[rho] : make_float2(0.f, 0.f);
      else
        st.row[x] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(stats_rs, 8 * rho, 0, 0));
    }
    return st;
  };
  // the tiles of a stage together: their products are chains of their own
  auto compute = [&](int t, const uint16_t* buf, Stats st) __attribute__((always_inline)) {
    f32x16 s[kTiles];
#pragma unroll
    for (int x = 0; x < kTiles; ++x) s[x] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kreg[ks], op.at(buf, ks, x), s[x], 0, 0, 0);
    if (t < whole) {
#pragma unroll
      for (int x = 0; x < kTiles; ++x) {
        const int lim = ob.pos0 + token_of((t + x) * kTile + qi) - wkey - 4 * half;
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[x][rr] = 8 * (rr >> 2) + (rr & 3) <= lim ? s[x][rr] : -INFINITY;
      }
    }
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      // a row past the last (its statistics read as 0) weighs 0, and not infinity times 0
      const float mc = (t + x) * kTile + qi < n_rows ? st.row[x].x : FLT_MAX;
#pragma unroll
      for (int rr = 0; rr < 16; ++rr)
        acc[rr] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[x][rr], c, -mc)), st.row[x].y, acc[rr]);
    }
  };
  // stage t: its Q has landed; the loads of the next one go into the other buffer
  auto stage = [&](int t, uint16_t* cur, Stats& st, uint16_t* next, Stats& st_next) __attribute__((always_inline)) {
    buffers_ready();
    if (t + kTiles < tiles) {
      dma(next, t + kTiles);
      st_next = load_stats(t + kTiles);
    }
    if (t + kTiles > seen) compute(t, cur, st);
  };
  if (first < tiles) {
    Stats s0, s1;
    dma(q0, first);
    if constexpr (kMerges) {
      const size_t stride = (size_t)p.batch * p.num_kv_heads * p.max_rows * p.group;
      for (int rho = tid; rho < n_rows; rho += kThreads) few[rho] = merged_stats(p, stats + rho, stride);
      __syncthreads();
    }
    s0 = load_stats(first);
    for (int t = first; t < tiles; t += 2 * kTiles) {
      stage(t, q0, s0, q1, s1);
      if (t + kTiles < tiles) stage(t + kTiles, q1, s1, q0, s0);
    }
  }
  // over the 32 rows in the lanes; lane i of a half then takes the key of register i
  float w = 0.f;
#pragma unroll
  for (int rr = 0; rr < 16; ++rr) {
    float x = acc[rr];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) x += __shfl_xor(x, o);
    w = qi == rr ? x : w;
  }
  const int key = wkey + 8 * (qi >> 2) + 4 * half + (qi & 3);
  if (qi >= 16) return;
  if (dealt.parts > 1)
    p.partials[((size_t)blockIdx.x / p.num_kv_heads / p.tiles * p.num_kv_heads + g) * p.tiles * kWeightKeys +
               (size_t)wg * kWeightKeys + key - key0] = w;
  else if (key >= from && key < ob.len)
    add_to_score(p, ob, bt, key, w);
}

// The scores of invocations whose rows were split: a work-group per key tile adds its parts in order.
__global__ __launch_bounds__(kWeightKeys) void key_weights_merge_kernel(ScoreParams p) {
  int rest = blockIdx.x;
  const int g = rest % p.num_kv_heads;
  rest /= p.num_kv_heads;
  const int tile = rest % p.key_tiles;
  const Observed ob(p, rest / p.key_tiles, g);
  const int from = first_scored(p, ob);
  const Dealt dealt(p, ob, from);
  const int key = from / kBlock * kBlock + tile * kWeightKeys + threadIdx.x;
  if (ob.n == 0 || dealt.parts <= 1 || key < from || key >= ob.len) return;
  const float* part = p.partials + (((size_t)ob.r * p.num_kv_heads + g) * p.tiles + tile) * kWeightKeys + threadIdx.x;
  float w = 0.f;
  for (int i = 0; i < dealt.parts; ++i) w += part[(size_t)i * dealt.key_tiles * kWeightKeys];
  add_to_score(p, ob, p.block_tables + (size_t)ob.r * p.max_blocks_per_seq, key, w);
}

}  // namespace

KeyScoreGeometry key_score_geometry(int batch, int total_q, int max_q_len, int max_kv_len, int rows,
                                    int num_q_heads, int num_kv_heads, int cus) {
  KeyScoreGeometry geo = {};
  geo.max_rows = std::min(rows, max_q_len);
  const long long stacked = (long long)geo.max_rows * (num_q_heads / num_kv_heads);
  geo.row_tiles = (stacked + kStatRows - 1) / kStatRows;
  geo.key_tiles = ((long long)max_kv_len + kWeightKeys - 1) / kWeightKeys;
  // (in one part each; so far this also bounds the products below)
  geo.fits = launch_fits((double)batch * num_kv_heads * std::max(geo.row_tiles, geo.key_tiles), kThreads);
  if (!geo.fits) return geo;
  const long long pairs = (long long)batch * num_kv_heads;
  // room to split the rows of key tiles that have many, in launches that leave CUs idle
  const long long row_parts = std::min((stacked + kTile * kPartTiles - 1) / (kTile * kPartTiles),
                                       16LL * cus / std::max(1LL, pairs * geo.key_tiles));
  geo.weight_groups = geo.key_tiles * std::max(1LL, row_parts);
  const long long steps = ((long long)max_kv_len + kStep - 1) / kStep;
  // work-groups that have rows, in a ragged batch far fewer than its longest invocation's for all
  const long long observed = std::min<long long>(total_q, (long long)batch * geo.max_rows);
  const long long work_groups = std::max(1LL, observed * num_q_heads / kStatRows);
  // Key parts of at least 8 steps: enough to fill the device, and up to 8 (which the merge
  // takes at once) to even out rows that see many keys and few.
  const long long parts = std::max(std::min(12LL * cus / work_groups, 8LL), 2LL * cus / work_groups);
  geo.parts = (int)std::max(1LL, std::min({parts, steps / 8, 32LL}));
  geo.stat_grid = pairs * geo.row_tiles * geo.parts;
  geo.weight_grid = pairs * geo.weight_groups;
  // (the merges have no more threads)
  geo.fits = launch_fits((double)geo.stat_grid, kThreads) && launch_fits((double)geo.weight_grid, kThreads);
  geo.stat_bytes = geo.parts * pairs * stacked * (long long)sizeof(float2);
  // (the partial sums of the split launches: any invocation may have as few scored keys as
  // to be split)
  geo.splits_rows = stacked > kTile * kPartTiles;
  geo.bytes = geo.stat_bytes + (geo.splits_rows ? geo.weight_grid * kWeightKeys * (long long)sizeof(float) : 0);
  return geo;
}

hipError_t launch_key_scores(const KeyScoreLaunch& a, hipStream_t stream) {
  const KeyScoreGeometry& geo = a.geo;
  ScoreParams p;
  p.q = a.q;
  p.k_pool = a.k_pool;
  p.block_tables = a.block_tables;
  p.prefix_lens = a.prefix_lens;
  p.cu_q_lens = a.cu_q_lens;
  p.score_from = a.score_from;
  p.score_pool = a.score_pool;
  p.stats = static_cast<float2*>(a.workspace);
  p.batch = a.batch;
  p.max_blocks_per_seq = a.max_blocks_per_seq;
  p.num_q_heads = a.num_q_heads;
  p.num_kv_heads = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.group_magic = p.group == 1 ? 0 : (unsigned)((0x100000000ULL + p.group - 1) / p.group);
  p.group_one = p.group == 1 ? ~0u : 0;
  p.rows = a.rows;
  p.max_rows = geo.max_rows;
  p.parts = geo.parts;
  p.key_tiles = (int)geo.key_tiles;
  p.partials = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + geo.stat_bytes);
  p.scale_log2 = a.scale * kLog2e;
  p.decay = a.decay;
  const bool few = geo.parts > 1 && (long long)geo.max_rows * p.group <= kFewRows;
  auto launch = [&](auto stats, auto weights, auto weights_of_few) {
    p.tiles = (int)geo.row_tiles;
    hipLaunchKernelGGL(stats, dim3((unsigned)geo.stat_grid), dim3(kThreads), 0, stream, p);
    if (geo.parts > 1 && !few) {
      const long long all = geo.stat_bytes / geo.parts / (long long)sizeof(float2);
      hipLaunchKernelGGL(key_stats_merge_kernel, dim3((unsigned)((all + 63) / 64)), dim3(64), 0, stream, p);
    }
    p.tiles = (int)geo.weight_groups;
    hipLaunchKernelGGL(few ? weights_of_few : weights, dim3((unsigned)geo.weight_grid), dim3(kThreads), 0, stream, p);
    if (geo.splits_rows)
      hipLaunchKernelGGL(key_weights_merge_kernel, dim3((unsigned)(geo.key_tiles * a.batch * a.num_kv_heads)),
                         dim3(kWeightKeys), 0, stream, p);
  };
  if (a.head_dim == 128)
    launch(key_stats_kernel<128>, key_weights_kernel<128, false>, key_weights_kernel<128, true>);
  else
    launch(key_stats_kernel<64>, key_weights_kernel<64, false>, key_weights_kernel<64, true>);
  return hipGetLastError();
}

}  // namespace cs
