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
//     score kept, found digit by digit (a histogram in LDS over 11, 11 and 10 bits of the
//     scores' order as integers), then the kept keys in ascending order by a prefix sum.  A
//     thread holds the scores of one pool block, 64 bytes, in registers throughout, so they
//     are read once (longer sequences are read again for every pass).
//   * evict_copy_kernel: the kept keys' K, V and scores into other blocks.
//   * evict_compact_kernel: the same within the sequence's own blocks, where the rows
//     written are rows that others are read from.  Kept key i goes to row i or comes from
//     further back (kept[i] >= i), so in ascending order a chunk's rows are free once its
//     own and the earlier chunks' rows are read: a work-group takes one column of 64 bytes
//     of a head's K or V (or its scores), reads a chunk into registers, and writes it
//     behind a barrier, with the next chunk's reads in flight.
#include "internal.h"
#include "wave_ops.h"

namespace cs {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 16;
constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2 * kSelectThreads;   // 11 bits
constexpr int kCopyThreads = 256;
constexpr int kCopyRows = 32;          // rows of a copy work-group
constexpr int kCompactVecs = 4;        // 16-byte vectors of a row per work-group (64 bytes)
constexpr int kCompactUnroll = 8;

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
// zeros are equal, and NaN comes last.  0 is no score's rank.
__device__ __forceinline__ unsigned rank_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x + 0.f);
  if (x != x) return 1;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum over the work-group's threads before this one, and over all (three barriers apart
// from the next call).
__device__ __forceinline__ int block_scan(int mine, int lane, int wave, int* sums, int& all) {
  const int incl = wave_scan(mine);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int before = incl - mine;
  all = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) {
    const int x = sums[w];
    before += w < wave ? x : 0;
    all += x;
  }
  return before;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
  __shared__ unsigned hist[kBins];
  __shared__ int sums[2][kSelectWaves];
  __shared__ unsigned found[3];
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
  const int want = p.budget - p.recent;
  for (int i = tid; i < p.recent; i += kSelectThreads) kept[want + i] = end + i;
  if (want == 0) return;
  // thread t holds block first + t of every kSelectThreads blocks: ranks of its keys, 0 for
  // those that do not compete (at least `want` do, so they are never chosen)
  const int first = from / kBlock;
  const int blocks = ceil_div(end, kBlock) - first;
  unsigned rank[kBlock];
  auto load = [&](int chunk) __attribute__((always_inline)) {
    const int b = first + chunk * kSelectThreads + tid;
#pragma unroll
    for (int e = 0; e < kBlock; ++e) rank[e] = 0;
    if (b * kBlock >= end) return;
    const float4* at = reinterpret_cast<const float4*>(p.score_pool + ((size_t)bt[b] * p.num_kv_heads + g) * kBlock);
    float4 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = at[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float four[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = b * kBlock + 4 * e + i;
        rank[4 * e + i] = key >= from && key < end ? rank_of(four[i]) : 0;
      }
    }
  };
  const int chunks = ceil_div(blocks, kSelectThreads);
  load(0);
  hist[tid] = hist[tid + kSelectThreads] = 0;
  __syncthreads();
  // the `want`-th largest rank: digits of 11, 11 and 10 bits
  unsigned prefix = 0;
  int need = want;                                // how many of the keys at it are kept
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int above = pass == 1 ? 21 : 10;        // bits that the passes before have found
    for (int c = 0; c < chunks; ++c) {
      if (chunks > 1) load(c);
#pragma unroll
      for (int e = 0; e < kBlock; ++e)
        if (pass == 0 ? rank[e] != 0 : rank[e] >> above == prefix >> above)
          atomicAdd(&hist[(rank[e] >> shift) & (kBins - 1) & (pass == 2 ? 0x3ffu : ~0u)], 1u);
    }
    __syncthreads();
    // thread t: the digits of its two bins, counted from the largest
    const int d1 = kBins - 1 - 2 * tid, d0 = d1 - 1;
    const int n1 = (int)hist[d1], n0 = (int)hist[d0];
    hist[d1] = hist[d0] = 0;
    int all;
    const int before = block_scan(n1 + n0, lane, wave, sums[pass & 1], all);
    if (before < need && before + n1 + n0 >= need) {
      const bool in_d1 = before + n1 >= need;
      found[0] = prefix | (unsigned)(in_d1 ? d1 : d0) << shift;
      const int left = need - before - (in_d1 ? 0 : n1);
      found[1] = (unsigned)left;
      found[2] = (unsigned)((in_d1 ? n1 : n0) - left);
    }
    __syncthreads();
    prefix = found[0];
    need = (int)found[1];
    const bool rest = found[2] != 0;
    __syncthreads();
    if (!rest) {                                  // all keys of that digit are kept
      prefix -= 1;
      need = 0;
      break;
    }
  }
  // in ascending order: all keys above the rank, and the first `need` at it
  int above = 0, at = 0;                          // before this chunk
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) load(c);
    int n_above = 0, n_at = 0;
#pragma unroll
    for (int e = 0; e < kBlock; ++e) {
      n_above += rank[e] > prefix;
      n_at += rank[e] == prefix;
    }
    int all;
    const int before = block_scan(n_above | n_at << 16, lane, wave, sums[c & 1], all);
    int a = above + (before & 0xffff), t = at + (int)((unsigned)before >> 16);
    const int key = (first + c * kSelectThreads + tid) * kBlock;
#pragma unroll
    for (int e = 0; e < kBlock; ++e) {
      const bool is_above = rank[e] > prefix, is_at = rank[e] == prefix;
      if (is_above || (is_at && t < need)) kept[a + min(t, need)] = key + e;
      a += is_above;
      t += is_at;
    }
    above += all & 0xffff;
    at += (int)((unsigned)all >> 16);
    __syncthreads();
  }
}

__device__ __forceinline__ void store_new_len(const EvictParams& p, int r, bool evicted, int from) {
  p.new_lens[r] = evicted ? from + p.budget : p.seq_lens[r];
}

// Rows i = -lead .. budget - 1 of a sequence and KV head into other blocks, where lead
// keys before keep_from lie in its block and come along.  HBM bound: a third of the rows
// of scattered 4 KiB tiles is read, in 256-byte pieces.  52 sequences to 2048 of 3000-9000
// keys, 8 heads of 128 (870 MB), with the selection: 205.6 us with 64 rows per
// work-group and ordinary stores, 202.0 with 32 rows, 200.6 with 64 and non-temporal
// stores, 197.1 with both (of which 175 are the copy, 5.0 TB/s); non-temporal loads too
// 194.0, but 14.3 us for 3 sequences to 1024 keys instead of 13.7.
template <int D>
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(EvictParams p) {
  constexpr int kVecs = D / 8;                     // 16-byte vectors of a row
  constexpr int kRows = kCopyThreads / kVecs;      // rows at once
  constexpr int kUnroll = kCopyRows / kRows;
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
  // a thread's vector of every row, and its rows: their places first, then all loads
  const int v = threadIdx.x % kVecs;
  const int end = lead + p.budget;
  int src[kUnroll], dst[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int i = min(chunk * kCopyRows + (int)threadIdx.x / kVecs + u * kRows, end - 1) - lead;
    src[u] = i < 0 ? from + i : kept[i];
    dst[u] = from + i;
  }
  size_t s[kUnroll], d[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    s[u] = ((size_t)bt[src[u] / kBlock] * p.num_kv_heads + g) * kBlock + src[u] % kBlock;
    d[u] = ((size_t)dt[dst[u] / kBlock] * p.num_kv_heads + g) * kBlock + dst[u] % kBlock;
  }
  u32x4 k[kUnroll], x[kUnroll];
  float score[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    k[u] = p.k_pool[s[u] * kVecs + v];
    x[u] = p.v_pool[s[u] * kVecs + v];
    score[u] = p.score_pool[s[u]];
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (chunk * kCopyRows + (int)threadIdx.x / kVecs + u * kRows >= end) break;
    __builtin_nontemporal_store(k[u], &p.k_pool[d[u] * kVecs + v]);
    __builtin_nontemporal_store(x[u], &p.v_pool[d[u] * kVecs + v]);
    if (v == 0) p.score_pool[d[u]] = score[u];
  }
}

// One column of a head's rows, moved within the sequence's blocks: kLanes threads take a
// row's elements column .. of row_elems.
template <int kLanes, typename T>
__device__ __forceinline__ void compact_column(const EvictParams& p, const int32_t* kept, const int32_t* bt, int g, int from,
                                               T* pool, int row_elems, int column) {
  constexpr int kRows = kCopyThreads / kLanes;
  constexpr int kChunk = kRows * kCompactUnroll;
  const int sub = threadIdx.x % kLanes;
  const int first = threadIdx.x / kLanes;
  auto at = [&](int pos) {
    return (((size_t)bt[pos / kBlock] * p.num_kv_heads + g) * kBlock + pos % kBlock) * row_elems + column + sub;
  };
  struct Chunk {
    T x[kCompactUnroll];
    bool moves[kCompactUnroll];
  };
  auto read = [&](Chunk& c, int base) __attribute__((always_inline)) {
    int src[kCompactUnroll];
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u) {
      const int i = base + u * kRows + first;
      src[u] = kept[min(i, p.budget - 1)];
      c.moves[u] = i < p.budget && src[u] != from + i;
    }
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u) c.x[u] = pool[at(src[u])];
  };
  auto write = [&](Chunk& c, int base) __attribute__((always_inline)) {
    // the wave's part of the chunk is in registers, then all waves' parts are
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u) asm volatile("" : "+v"(c.x[u]));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kCompactUnroll; ++u)
      if (c.moves[u]) pool[at(from + base + u * kRows + first)] = c.x[u];
  };
  Chunk a, b;
  read(a, 0);
  for (int base = 0; base < p.budget; base += 2 * kChunk) {
    // (the next chunk's rows lie behind all that this one and those before it write)
    if (base + kChunk < p.budget) read(b, base + kChunk);
    write(a, base);
    if (base + kChunk >= p.budget) break;
    if (base + 2 * kChunk < p.budget) read(a, base + 2 * kChunk);
    write(b, base + kChunk);
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
    compact_column<1>(p, kept, bt, g, from, p.score_pool, 1, 0);
  } else {
    u32x4* pool = column < columns ? p.k_pool : p.v_pool;
    compact_column<kCompactVecs>(p, kept, bt, g, from, pool, p.vecs, column % columns * kCompactVecs);
  }
}

unsigned copy_chunks(int budget) { return ((unsigned)budget + kBlock - 1 + kCopyRows - 1) / kCopyRows; }
unsigned compact_columns(int head_dim) { return 2 * (head_dim / 8 / kCompactVecs) + 1; }

}  // namespace

bool evict_fits(int batch, int num_kv_heads, int head_dim, int budget, bool moving) {
  const double pairs = (double)batch * num_kv_heads;
  const double second = moving ? copy_chunks(budget) : compact_columns(head_dim);
  return launch_fits(pairs, kSelectThreads) && launch_fits(pairs * second, kCopyThreads);
}

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
    const unsigned chunks = copy_chunks(a.budget);
    if (a.head_dim == 128)
      hipLaunchKernelGGL(evict_copy_kernel<128>, dim3(pairs * chunks), dim3(kCopyThreads), 0, stream, p);
    else
      hipLaunchKernelGGL(evict_copy_kernel<64>, dim3(pairs * chunks), dim3(kCopyThreads), 0, stream, p);
  } else {
    const unsigned columns = compact_columns(a.head_dim);
    hipLaunchKernelGGL(evict_compact_kernel, dim3(pairs * columns), dim3(kCopyThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace cs
