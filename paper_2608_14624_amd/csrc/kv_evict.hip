// Eviction within a sequence by accumulated attention weight, for gfx950: which of its
// keys a sequence keeps, and the copy of what is kept to where it then lies.
//
// A sequence's own keys are those from `keep_from` on (the keys before, a shared anchor
// or the first tokens, stay).  One with more than `trigger` of them keeps `budget`: the
// last `recent`, and of the others the ones with the largest scores, of equal scores
// the first.  The choice is made for every KV head by itself, since the pool holds a
// head's rows apart; all heads keep the same number.
//
//   * evict_select_kernel, a work-group per (sequence, KV head): the value of the least
//     score kept, found digit by digit (a histogram in LDS per 8 bits of the scores' order
//     as integers), then one ordered pass that writes the kept keys in ascending order.
//   * evict_copy_kernel: the kept keys' K, V and scores into other blocks.
//   * evict_compact_kernel: the same within the sequence's own blocks, where the rows
//     written are rows that others are read from.  Kept key i goes to row i or comes from
//     further back (kept[i] >= i), so in ascending order a chunk's rows are free once its
//     own and the earlier chunks' rows are read: a work-group takes one column of 64 bytes
//     of a head's K or V (or its scores), reads a chunk into registers, and writes it
//     behind a barrier, with the next chunk's reads in flight.
#include "internal.h"
#include "wave_ops.h"

#include <algorithm>

namespace cs {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 16;
constexpr int kSelectThreads = 512;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kCopyThreads = 256;
constexpr int kCopyRows = 64;          // rows of a copy work-group
constexpr int kCompactVecs = 4;        // 16-byte vectors of a row per work-group (64 bytes)
constexpr int kCompactUnroll = 8;
// s_waitcnt immediate: no vector memory operation of the wave left in flight
constexpr int kWaitVmcnt0 = 0x0F70;

struct EvictParams {
  const int32_t* block_tables;
  const int32_t* dst_tables;
  const int32_t* seq_lens;
  const int32_t* keep_from;
  int32_t* kept;                 // [batch][num_kv_heads][budget]; a first entry of -1: nothing was evicted
  int32_t* new_lens;
  u32x4* k_pool;
  u32x4* v_pool;
  float* score_pool;
  int batch;
  int max_blocks_per_seq;
  int num_kv_heads;
  int vecs;                      // 16-byte vectors of a row
  int budget;
  int trigger;
  int recent;
};

// A score's place in the order of all scores: larger scores have larger values, the two
// zeros are equal, and NaN comes last.
__device__ __forceinline__ unsigned rank_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x + 0.f);
  if (x != x) return 0;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
  __shared__ unsigned hist[256];
  __shared__ int sums[kSelectWaves];
  __shared__ unsigned found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads;
  const int len = p.seq_lens[r];
  const int from = max(0, p.keep_from[r]);
  int32_t* kept = p.kept + ((size_t)r * p.num_kv_heads + g) * p.budget;
  if (len - from <= p.trigger) {
    if (tid == 0) kept[0] = -1;
    return;
  }
  const int32_t* bt = p.block_tables + (size_t)r * p.max_blocks_per_seq;
  const int end = len - p.recent;                 // the keys from .. end - 1 compete
  auto rank_at = [&](int key) {
    return rank_of(p.score_pool[((size_t)bt[key / kBlock] * p.num_kv_heads + g) * kBlock + key % kBlock]);
  };
  // the `want`-th largest rank
  const int want = p.budget - p.recent;
  unsigned least = 0xffffffffu;
  int need = 0;                                   // how many of the keys at `least` are kept
  if (want > 0) {
    unsigned prefix = 0;
    need = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int key = from + tid; key < end; key += kSelectThreads) {
        const unsigned x = rank_at(key);
        if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(x >> shift) & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {
        // lane i: the digits 255 - 4 i .. 252 - 4 i; counts of all larger digits
        int mine[4], total = 0;
        for (int e = 0; e < 4; ++e) total += mine[e] = (int)hist[255 - 4 * lane - e];
        int before = wave_scan(total) - total;
        for (int e = 0; e < 4; ++e) {
          if (before < need && before + mine[e] >= need) {
            found[0] = prefix | (unsigned)(255 - 4 * lane - e) << shift;
            found[1] = (unsigned)(need - before);
          }
          before += mine[e];
        }
      }
      __syncthreads();
      prefix = found[0];
      need = (int)found[1];
    }
    least = prefix;
  }
  // in ascending order: all keys above `least`, and the first `need` at it
  int above = 0, at = 0;                          // before this chunk
  for (int base = from; base < end && want > 0; base += kSelectThreads) {
    const int key = base + tid;
    const unsigned x = key < end ? rank_at(key) : 0;
    const bool is_above = key < end && x > least, is_at = key < end && x == least;
    const int mine = (is_above ? 1 : 0) | (is_at ? 1 << 16 : 0);
    const int incl = wave_scan(mine);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int before = incl - mine, all = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) before += sums[w];
      all += sums[w];
    }
    const int a = above + (before & 0xffff), e = at + (before >> 16);
    if (is_above || (is_at && e < need)) kept[a + min(e, need)] = key;
    above += all & 0xffff;
    at += all >> 16;
    __syncthreads();
  }
  for (int i = tid; i < p.recent; i += kSelectThreads) kept[want + i] = end + i;
}

__device__ __forceinline__ void store_new_len(const EvictParams& p, int r, bool evicted, int from) {
  p.new_lens[r] = evicted ? from + p.budget : p.seq_lens[r];
}

// Rows i = -lead .. budget - 1 of a sequence and KV head into other blocks, where lead
// keys before keep_from lie in its block and come along.
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(EvictParams p) {
  const int g = blockIdx.x % p.num_kv_heads;
  const int r = blockIdx.x / p.num_kv_heads % p.batch;
  const int chunk = blockIdx.x / p.num_kv_heads / p.batch;
  const int32_t* kept = p.kept + ((size_t)r * p.num_kv_heads + g) * p.budget;
  const int from = max(0, p.keep_from[r]);
  const bool evicted = kept[0] >= 0;
  if (g == 0 && chunk == 0 && threadIdx.x == 0) store_new_len(p, r, evicted, from);
  if (!evicted) return;
  const int lead = from % kBlock;
  const int32_t* bt = p.block_tables + (size_t)r * p.max_blocks_per_seq;
  const int32_t* dt = p.dst_tables + (size_t)r * p.max_blocks_per_seq;
  const int rows = min(kCopyRows, lead + p.budget - chunk * kCopyRows);
  for (int i = threadIdx.x; i < rows * p.vecs; i += kCopyThreads) {
    const int row = chunk * kCopyRows + i / p.vecs - lead;
    const int src = row < 0 ? from + row : kept[row];
    const int dst = from + row;
    const size_t s = ((size_t)bt[src / kBlock] * p.num_kv_heads + g) * kBlock + src % kBlock;
    const size_t d = ((size_t)dt[dst / kBlock] * p.num_kv_heads + g) * kBlock + dst % kBlock;
    const int v = i % p.vecs;
    const u32x4 k = p.k_pool[s * p.vecs + v];
    const u32x4 x = p.v_pool[s * p.vecs + v];
    p.k_pool[d * p.vecs + v] = k;
    p.v_pool[d * p.vecs + v] = x;
    if (v == 0) p.score_pool[d] = p.score_pool[s];
  }
}

// One column of a head's rows, moved within the sequence's blocks.  at(row position):
// index of the column's first element; lanes_per_row threads take a row.
template <typename T>
__device__ __forceinline__ void compact_column(const EvictParams& p, const int32_t* kept, const int32_t* bt, int g, int from,
                                               T* pool, int row_elems, int column, int lanes_per_row) {
  const int sub = threadIdx.x % lanes_per_row;
  const int rows_at_once = kCopyThreads / lanes_per_row;
  const int first = threadIdx.x / lanes_per_row;
  auto at = [&](int pos) {
    return (((size_t)bt[pos / kBlock] * p.num_kv_heads + g) * kBlock + pos % kBlock) * row_elems + column + sub;
  };
  for (int base = 0; base < p.budget; base += rows_at_once * kCompactUnroll) {
    T x[kCompactUnroll];
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u) {
      const int i = base + u * rows_at_once + first;
      if (i < p.budget) x[u] = pool[at(kept[i])];
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();                 // the chunk is read
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u) {
      const int i = base + u * rows_at_once + first;
      if (i < p.budget && kept[i] != from + i) pool[at(from + i)] = x[u];
    }
  }
}

__global__ __launch_bounds__(kCopyThreads) void evict_compact_kernel(EvictParams p) {
  const int columns = p.vecs / kCompactVecs;
  const int g = blockIdx.x % p.num_kv_heads;
  const int rest = blockIdx.x / p.num_kv_heads;
  const int column = rest % (2 * columns + 1);        // K's, V's, the scores
  const int r = rest / (2 * columns + 1);
  const int32_t* kept = p.kept + ((size_t)r * p.num_kv_heads + g) * p.budget;
  const int from = max(0, p.keep_from[r]);
  const bool evicted = kept[0] >= 0;
  if (g == 0 && column == 0 && threadIdx.x == 0) store_new_len(p, r, evicted, from);
  if (!evicted) return;
  const int32_t* bt = p.block_tables + (size_t)r * p.max_blocks_per_seq;
  if (column == 2 * columns) {
    compact_column(p, kept, bt, g, from, p.score_pool, 1, 0, 1);
  } else {
    u32x4* pool = column < columns ? p.k_pool : p.v_pool;
    compact_column(p, kept, bt, g, from, pool, p.vecs, column % columns * kCompactVecs, kCompactVecs);
  }
}

}  // namespace

hipError_t launch_kv_evict(const EvictLaunch& a, hipStream_t stream) {
  EvictParams p;
  p.block_tables = a.block_tables;
  p.dst_tables = a.dst_tables;
  p.seq_lens = a.seq_lens;
  p.keep_from = a.keep_from;
  p.kept = a.kept;
  p.new_lens = a.new_lens;
  p.k_pool = reinterpret_cast<u32x4*>(a.k_pool);
  p.v_pool = reinterpret_cast<u32x4*>(a.v_pool);
  p.score_pool = a.score_pool;
  p.batch = a.batch;
  p.max_blocks_per_seq = a.max_blocks_per_seq;
  p.num_kv_heads = a.num_kv_heads;
  p.vecs = a.head_dim / 8;
  p.budget = a.budget;
  p.trigger = a.trigger;
  p.recent = a.recent;
  const unsigned pairs = (unsigned)((long long)a.batch * a.num_kv_heads);
  hipLaunchKernelGGL(evict_select_kernel, dim3(pairs), dim3(kSelectThreads), 0, stream, p);
  if (a.dst_tables != nullptr) {
    const unsigned chunks = (unsigned)((a.budget + kBlock - 1 + kCopyRows - 1) / kCopyRows);
    hipLaunchKernelGGL(evict_copy_kernel, dim3(pairs * chunks), dim3(kCopyThreads), 0, stream, p);
  } else {
    const unsigned columns = (unsigned)(2 * (p.vecs / kCompactVecs) + 1);
    hipLaunchKernelGGL(evict_compact_kernel, dim3(pairs * columns), dim3(kCopyThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace cs
