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
  int rows;                   // observed rows per invocation (the last ones)
  int max_rows;               // of any invocation
  int parts;
  int tiles;                  // work-groups per (invocation, KV head)
  float scale_log2;
  float decay;
};

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ void pair_swap(float x, float& a, float& b) {
  a = x;
  b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
}

// An invocation: its observed rows are the stacked rows 0 .. n * group - 1 of a KV head;
// row rho is head rho % group of the token at position pos0 + rho / group.
struct Observed {
  int r, g, q0, n, pos0, len, prefix;
  __device__ __forceinline__ Observed(const ScoreParams& p, int r_, int g_) : r(r_), g(g_) {
    const int first = p.cu_q_lens[r];
    const int s = p.cu_q_lens[r + 1] - first;
    prefix = p.prefix_lens[r];
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

template <int D>
__global__ __launch_bounds__(kThreads) void key_stats_kernel(ScoreParams p) {
  constexpr int KS = D / 16;
  constexpr int kStride = D + 8;
  constexpr int kLoads = kStep * D / 8 / kThreads;      // 16-byte vectors per thread and step
  __shared__ uint16_t kbuf[2][kStep * kStride];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int qi = lane & 31, half = lane >> 5;
  int rest = blockIdx.x;
  const int g = rest % p.num_kv_heads;
  rest /= p.num_kv_heads;
  const int tile = p.tiles - 1 - rest % p.tiles;        // the rows with most keys first
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
  const int pos_min = ob.pos0 + wave_first / p.group;
  const int steps = ceil_div(kv_end, kStep);
  const int s0 = (int)((long long)steps * part / p.parts);
  const int s1 = (int)((long long)steps * (part + 1) / p.parts);

  bf16x8 qreg[KS];
  const uint16_t* qrow = ob.q_row(p, valid ? rho : 0, D);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + half * 8));

  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const uint16_t* kbase = p.k_pool + (size_t)g * tile_elems;
  const int32_t* bt = p.block_tables + (size_t)ob.r * p.max_blocks_per_seq;
  const int n_blk = ceil_div(ob.len, kBlock);
  uint4 kreg[kLoads];
  auto load = [&](int step) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int c = tid + kThreads * u;
      const int key = c / (D / 8);
      const int b = min((step * kStep + key) / kBlock, n_blk - 1);   // past the end: masked
      kreg[u] = *reinterpret_cast<const uint4*>(kbase + (size_t)bt[b] * slot_elems + (key % kBlock) * D + (c % (D / 8)) * 8);
    }
  };
  auto store = [&](uint16_t* buf) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int c = tid + kThreads * u;
      *reinterpret_cast<uint4*>(&buf[(c / (D / 8)) * kStride + (c % (D / 8)) * 8]) = kreg[u];
    }
  };

  const float c = p.scale_log2;
  // finite, so that keys a row does not see weigh 0 and not NaN
  float m = -FLT_MAX / fmaxf(c, 1.f), l = 0.f;
  if (s0 < s1) load(s0);
  for (int step = s0; step < s1; ++step) {
    uint16_t* buf = kbuf[step & 1];
    store(buf);
    __syncthreads();
    if (step + 1 < s1) load(step + 1);
    f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const uint4 a = *reinterpret_cast<const uint4*>(&buf[(mt * 32 + qi) * kStride + ks * 16 + half * 8]);
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), qreg[ks], s[mt], 0, 0, 0);
      }
    const int kstart = step * kStep;
    if (kstart + kStep - 1 > pos_min) {
      const int lim = pos - kstart - 4 * half;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[mt][rr] = mt * 32 + 8 * (rr >> 2) + (rr & 3) <= lim ? s[mt][rr] : -INFINITY;
    }
    // each lane half keeps the statistics of its own keys until the end
    float mx = m;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) mx = fmaxf(mx, s[mt][rr]);
    l *= __builtin_amdgcn_exp2f((m - mx) * c);
    m = mx;
    const float mc = m * c;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) l += __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][rr], c, -mc));
  }
  float m0, m1, l0, l1;
  pair_swap(m, m0, m1);
  pair_swap(l, l0, l1);
  m = fmaxf(m0, m1);
  l = l0 * __builtin_amdgcn_exp2f((m0 - m) * c) + l1 * __builtin_amdgcn_exp2f((m1 - m) * c);
  if (valid && half == 0) p.stats[ob.stat(p, part) + rho] = make_float2(m * c, p.parts == 1 ? 1.f / l : l);
}

// The statistics of rows split over key parts, into part 0.
__global__ __launch_bounds__(kThreads) void key_stats_merge_kernel(ScoreParams p) {
  const size_t all = (size_t)p.batch * p.num_kv_heads * p.max_rows * p.group;
  const size_t at = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (at >= all) return;
  float m = -FLT_MAX, l = 0.f;
  for (int k = 0; k < p.parts; ++k) m = fmaxf(m, p.stats[k * all + at].x);
  for (int k = 0; k < p.parts; ++k) {
    const float2 ml = p.stats[k * all + at];
    l += ml.y * __builtin_amdgcn_exp2f(ml.x - m);
  }
  p.stats[at] = make_float2(m, 1.f / l);
}

template <int D>
__global__ __launch_bounds__(kThreads) void key_weights_kernel(ScoreParams p) {
  constexpr int KS = D / 16;
  constexpr int kStride = D + 8;
  constexpr int kLoads = kStageRows * D / 8 / kThreads;
  __shared__ uint16_t qbuf[2][kStageRows * kStride];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int qi = lane & 31, half = lane >> 5;
  int rest = blockIdx.x;
  const int g = rest % p.num_kv_heads;
  rest /= p.num_kv_heads;
  const Observed ob(p, rest / p.tiles, g);
  const int from = max(0, p.score_from[ob.r]);
  // keys from the first scored block on
  const int key0 = from / kBlock * kBlock + rest % p.tiles * kWeightKeys;
  const int n_rows = ob.n * p.group;
  if (key0 >= ob.len || n_rows == 0) return;
  const int wkey = key0 + wave * kTile;                  // the wave's keys
  const size_t tile_elems = (size_t)kBlock * D;
  const size_t slot_elems = (size_t)p.num_kv_heads * tile_elems;
  const int32_t* bt = p.block_tables + (size_t)ob.r * p.max_blocks_per_seq;
  const int n_blk = ceil_div(ob.len, kBlock);
  bf16x8 kreg[KS];
  {
    const int key = wkey + qi;
    const uint16_t* row = p.k_pool + (size_t)bt[min(key / kBlock, n_blk - 1)] * slot_elems + (size_t)g * tile_elems +
                          (key % kBlock) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(row + ks * 16 + half * 8));
  }
  // stacked rows from the first token that sees the work-group's first key on
  const int first = max(0, key0 - ob.pos0) * p.group / kTile;
  const int tiles = ceil_div(n_rows, kTile);
  const float2* stats = p.stats + ob.stat(p, 0);
  uint4 qreg[kLoads];
  auto load = [&](int t) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int c = tid + kThreads * u;
      const int rho = min(t * kTile + c / (D / 8), n_rows - 1);
      qreg[u] = *reinterpret_cast<const uint4*>(ob.q_row(p, rho, D) + (c % (D / 8)) * 8);
    }
  };
  const float c = p.scale_log2;
  f32x16 acc = f32x16{};
  load(first);
  int buf = 0;
  for (int t = first; t < tiles; t += kStageRows / kTile, buf ^= 1) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int cc = tid + kThreads * u;
      *reinterpret_cast<uint4*>(&qbuf[buf][(cc / (D / 8)) * kStride + (cc % (D / 8)) * 8]) = qreg[u];
    }
    float2 st[kStageRows / kTile];
#pragma unroll
    for (int x = 0; x < kStageRows / kTile; ++x) {
      const int rho = (t + x) * kTile + qi;
      st[x] = rho < n_rows ? stats[rho] : make_float2(0.f, 0.f);
    }
    __syncthreads();
    if (t + kStageRows / kTile < tiles) load(t + kStageRows / kTile);
#pragma unroll
    for (int x = 0; x < kStageRows / kTile; ++x) {
      f32x16 s = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint4 b = *reinterpret_cast<const uint4*>(&qbuf[buf][(x * kTile + qi) * kStride + ks * 16 + half * 8]);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kreg[ks], as_bf16x8(b), s, 0, 0, 0);
      }
      const int rho = (t + x) * kTile + qi;
      if (wkey + kTile - 1 > ob.pos0 + min((t + x) * kTile, n_rows - 1) / p.group) {
        const int lim = ob.pos0 + rho / p.group - wkey - 4 * half;
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[rr] = 8 * (rr >> 2) + (rr & 3) <= lim ? s[rr] : -INFINITY;
      }
#pragma unroll
      for (int rr = 0; rr < 16; ++rr)
        acc[rr] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[rr], c, -st[x].x)), st[x].y, acc[rr]);
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
  if (qi >= 16 || key < from || key >= ob.len) return;
  float* score = p.score_pool + ((size_t)bt[key / kBlock] * p.num_kv_heads + g) * kBlock + key % kBlock;
  *score = key < ob.prefix ? __builtin_fmaf(p.decay, *score, w) : w;
}

}  // namespace

KeyScoreGeometry key_score_geometry(int batch, int max_q_len, int max_kv_len, int rows, int num_q_heads,
                                    int num_kv_heads, int cus) {
  KeyScoreGeometry geo;
  geo.max_rows = std::min(rows, max_q_len);
  const long long stacked = (long long)geo.max_rows * (num_q_heads / num_kv_heads);
  geo.row_tiles = (stacked + kStatRows - 1) / kStatRows;
  geo.key_tiles = ((long long)max_kv_len + kWeightKeys - 1) / kWeightKeys;
  const long long pairs = (long long)batch * num_kv_heads;
  const long long steps = ((long long)max_kv_len + kStep - 1) / kStep;
  const long long work_groups = std::max(1LL, pairs * geo.row_tiles);
  geo.parts = (int)std::max(1LL, std::min({2LL * cus / work_groups, steps / 4, 32LL}));
  geo.stat_grid = pairs * geo.row_tiles * geo.parts;
  geo.weight_grid = pairs * geo.key_tiles;
  geo.stat_bytes = geo.parts * pairs * stacked * (long long)sizeof(float2);
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
  p.rows = a.rows;
  p.max_rows = geo.max_rows;
  p.parts = geo.parts;
  p.scale_log2 = a.scale * kLog2e;
  p.decay = a.decay;
  auto launch = [&](auto stats, auto weights) {
    p.tiles = (int)geo.row_tiles;
    hipLaunchKernelGGL(stats, dim3((unsigned)geo.stat_grid), dim3(kThreads), 0, stream, p);
    if (geo.parts > 1) {
      const long long all = geo.stat_bytes / geo.parts / (long long)sizeof(float2);
      hipLaunchKernelGGL(key_stats_merge_kernel, dim3((unsigned)((all + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                         stream, p);
    }
    p.tiles = (int)geo.key_tiles;
    hipLaunchKernelGGL(weights, dim3((unsigned)geo.weight_grid), dim3(kThreads), 0, stream, p);
  };
  if (a.head_dim == 128)
    launch(key_stats_kernel<128>, key_weights_kernel<128>);
  else
    launch(key_stats_kernel<64>, key_weights_kernel<64>);
  return hipGetLastError();
}

}  // namespace cs
