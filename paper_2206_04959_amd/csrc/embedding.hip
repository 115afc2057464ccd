// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   y[t]  = scale * E[ids[t] - first]           (a row of zeros if that is no row of E)
//   dE[v] (=|+=) scale * sum of dy[t] over the tokens t with ids[t] - first = v
//
// E is one tensor-parallel rank's share of the vocabulary (rows first ..
// first + rows - 1), so ids of other ranks, and padding such as -1, contribute
// nothing: the sum of the ranks' y is the whole lookup.
//
// Both directions move data and compute next to nothing.  The lookup reads the
// tokens' rows and writes y.  The gradient reads dy once and writes dE once: the
// tokens are sorted by row first (tokens of one row in their own order), so each
// row's sum is formed in registers, in one fixed order and without
// floating-point atomics, and rows without a token are written as zeros by the
// same launch.
#include <algorithm>
#include <atomic>

#include "common.h"
#include "kernels.h"

namespace merak {

// Row of the table that `id` names, or `rows` if none.
template <typename I>
__device__ __forceinline__ int table_row(I id, long long first, int rows) {
  const unsigned long long r = (unsigned long long)(long long)id - (unsigned long long)first;
  return r < (unsigned long long)rows ? (int)r : rows;
}

// ---------------------------------------------------------------------------
// Forward: one 16-byte chunk of y per thread and step, consecutive threads on
// consecutive chunks of y; four chunks a thread, so that four ids and then four rows are
// on their way at once.  32768 tokens of 6144 in bf16 (520 MB): 113 us, 4.6 TB/s, the rate
// of a large copy.
// ---------------------------------------------------------------------------
constexpr int kFwdUnroll = 4;

template <typename T, typename I, bool PAST>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(int tokens, int hidden, int rows, long long first,
                                                            float scale, const I* __restrict__ ids,
                                                            const T* __restrict__ table, T* __restrict__ y) {
  constexpr int EPC = 16 / sizeof(T);  // elements per chunk
  const unsigned cpr = hidden / EPC;
  const unsigned long long base = (unsigned long long)blockIdx.x * (256 * kFwdUnroll);
  const unsigned t0 = (unsigned)(base / cpr), c0 = (unsigned)(base % cpr);
  u32x4_t v[kFwdUnroll];
  size_t at[kFwdUnroll];
  bool live[kFwdUnroll];
#pragma unroll
  for (int u = 0; u < kFwdUnroll; ++u) {
    const unsigned local = c0 + threadIdx.x + 256 * u;
    const unsigned dt = local / cpr, c = local - dt * cpr;
    const size_t t = (size_t)t0 + dt;
    live[u] = t < (size_t)tokens;
    at[u] = (t * cpr + c) * EPC;
    v[u] = u32x4_t{0u, 0u, 0u, 0u};
    if (live[u]) {
      const int r = table_row(ids[t], first, rows);
      if (r < rows) v[u] = *reinterpret_cast<const u32x4_t*>(table + ((size_t)r * cpr + c) * EPC);
    }
  }
#pragma unroll
  for (int u = 0; u < kFwdUnroll; ++u) {
    if (!live[u]) continue;
    u32x4_t o;
    if constexpr (sizeof(T) == 2) {
      float f[8];
      unpack8(v[u], f);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(f[2 * e] * scale, f[2 * e + 1] * scale);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(__uint_as_float(v[u][e]) * scale);
    }
    store16<PAST>(y + at[u], o);
  }
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------
// Up to here one launch, without sorting: 2048 tokens of a text of 1024 on 6000 rows 16.6 us,
// sorted 21.0; 1024 tokens 13.4 and 20.1; 257 tokens 8.3 and 16.9.
constexpr int kDirect = 2048;
constexpr int kSortBlock = 2048;  // tokens that are ranked against each other
constexpr int kFillRows = 16;     // most table rows that a workgroup clears
constexpr size_t kFillBytes = 65536;  // that a workgroup clears, about
constexpr int kSlab = 512;        // columns of a wave: 8 a lane
constexpr int kMinChunk = 16, kMaxChunks = 1024;
// A run of up to this many tokens is never split, which leaves embedding_join_kernel the
// frequent tokens only.
constexpr int kWhole = 32;

// Sorted positions per unit of work: at most kMaxChunks units, whole multiples
// of 16 positions.
static inline int chunk_len(int tokens) {
  const int c = (tokens + kMaxChunks - 1) / kMaxChunks;
  return std::max(kMinChunk, (c + 15) / 16 * 16);
}

// Rank of each token within its block of kSortBlock by (row, token): the number of
// tokens of the block that come before it.  A workgroup ranks 64 tokens, each of its
// 16 waves against 128 of the block.  Comparing every pair costs two
// instructions a pair and no dependence between them, in one launch; the keys go
// through LDS as four-key reads that all lanes share.  16384 tokens: 5.3 us.
constexpr int kRankWaves = 16;

template <typename I>
__global__ void __launch_bounds__(64 * kRankWaves) embedding_rank_kernel(int tokens, int rows, long long first,
                                                                         const I* __restrict__ ids,
                                                                         int* __restrict__ skey,
                                                                         int* __restrict__ stok,
                                                                         int* __restrict__ split) {
  if (blockIdx.x == 0 && threadIdx.x == 0) *split = 0;  // for embedding_sum_kernel
  constexpr int NT = 64 * kRankWaves, PER = kSortBlock / NT, Q = kSortBlock / kRankWaves;
  __shared__ __align__(16) unsigned key[kSortBlock];  // past the last token: above every row
  __shared__ int cnt[kRankWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int t0 = blockIdx.x * 64;               // first token of this workgroup
  const int b0 = t0 / kSortBlock * kSortBlock;  // first token of its block
  const int slice = t0 - b0, m = min(kSortBlock, tokens - b0);
  I id[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int j = threadIdx.x + NT * u;
    id[u] = j < m ? ids[b0 + j] : (I)0;
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int j = threadIdx.x + NT * u;
    key[j] = j < m ? (unsigned)table_row(id[u], first, rows) : 0xfffffffeu;
  }
  __syncthreads();
  const unsigned k = key[slice + lane];
  // A token before the slice counts if its row is not larger, one after it if smaller.
  int n = 0;
  auto count = [&](int lo, int hi, unsigned thr) {  // multiples of 64
    for (int j = lo; j < hi; j += 32) {
      u32x4_t v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const u32x4_t*>(key + j + 4 * u);
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) n += v[u][e] < thr;
    }
  };
  const int lo = w * Q, hi = min(lo + Q, (m + 63) & ~63);
  count(lo, min(hi, slice), k + 1);
  count(max(lo, slice + 64), hi, k);
  if (slice >= lo && slice < hi) {
#pragma unroll
    for (int j = 0; j < 64; j += 4) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(key + slice + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) n += v[e] < (j + e < lane ? k + 1 : k);
    }
  }
  cnt[w][lane] = n;
  __syncthreads();
  if (w == 0 && t0 + lane < tokens) {
    int r = 0;
#pragma unroll
    for (int i = 0; i < kRankWaves; ++i) r += cnt[i][lane];
    skey[b0 + r] = (int)k;
    stok[b0 + r] = t0 + lane;
  }
}

// Whole order from the sorted blocks: a token's position is the number of tokens
// before it in each block, found by binary search.  A workgroup places 64 tokens;
// each of its waves (one a block, at most 16) brings a block's keys into LDS and
// searches there: twelve dependent loads from L2 instead took 4 of 5 us.  As every workgroup
// reads all other blocks, the time grows with the square of the tokens: all launches for rows
// of 8 columns take 25 us at 16384 tokens, 34 at 32768, 128 at 131072, 3.3 ms at 2^20 and 48 at
// 2^22, the most that a call takes.
constexpr int kMergeWaves = 16;

__global__ void __launch_bounds__(64 * kMergeWaves) embedding_merge_kernel(int tokens, const int* __restrict__ skey,
                                                                           const int* __restrict__ stok,
                                                                           int* __restrict__ gkey,
                                                                           int* __restrict__ gtok) {
  extern __shared__ __align__(16) int block_keys[];  // [waves][kSortBlock], then the counts [waves][64]
  const int waves = blockDim.x >> 6;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* mine = block_keys + w * kSortBlock;
  int* cnt = block_keys + waves * kSortBlock;
  const int p = blockIdx.x * 64 + lane;
  const int b = blockIdx.x * 64 / kSortBlock, nb = (tokens + kSortBlock - 1) / kSortBlock;
  const int k = p < tokens ? skey[p] : 0;
  const int t = p < tokens ? stok[p] : 0;
  int n = w == b % waves ? p - b * kSortBlock : 0;  // those of its own block
  for (int o = w; o < nb; o += waves) {
    if (o == b) continue;
    const int* kb = skey + (size_t)o * kSortBlock;
    const int m = min(kSortBlock, tokens - o * kSortBlock);
    constexpr int L = kSortBlock / 256;
    u32x4_t v[L];
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int j = 256 * u + lane * 4;  // skey holds whole blocks: keys past m are read and not used
      v[u] = *reinterpret_cast<const u32x4_t*>(kb + j);
    }
#pragma unroll
    for (int u = 0; u < L; ++u) *reinterpret_cast<u32x4_t*>(mine + 256 * u + lane * 4) = v[u];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the keys are this wave's own
    const int thr = o < b ? k + 1 : k;
    int pos = 0;  // tokens known to come before
#pragma unroll
    for (int step = kSortBlock; step > 0; step >>= 1)
      if (pos + step <= m && mine[pos + step - 1] < thr) pos += step;
    n += pos;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  cnt[w * 64 + lane] = n;
  __syncthreads();
  if (w == 0 && p < tokens) {
    int g = 0;
    for (int i = 0; i < waves; ++i) g += cnt[i * 64 + lane];
    gkey[g] = k;
    gtok[g] = t;
  }
}

// First sorted position whose row is not below r, by 16 neighbouring lanes together: they
// probe 16 places at a time, so 2^14 keys take four dependent loads.
__device__ __forceinline__ int lower_bound16(const int* key, int n, int r, int lane) {
  int lo = 0;
  while (n > 0) {  // the same for the 16 lanes
    const int step = (n + 15) >> 4, at = (lane & 15) * step;
    const unsigned long long votes = __ballot(at < n && key[lo + at] < r);
    const int below = __builtin_popcount((unsigned)(votes >> (lane & 48)) & 0xffffu);  // probes below r come first
    if (below == 0) return lo;
    const int from = (below - 1) * step + 1, to = min(below * step, n);
    lo += from;
    n = to - from;
  }
  return lo;
}

// 8 columns of a row of T from their 16-byte pieces.
template <typename T>
__device__ __forceinline__ void unpack_row(const u32x4_t (&v)[sizeof(T) / 2], float f[8]) {
  if constexpr (sizeof(T) == 2) {
    unpack8(v[0], f);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[e >> 2][e & 3]);
  }
}

// 8 columns of a finished row.
__device__ __forceinline__ void write_row(float* out, const float acc[8], float scale, int accumulate) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = acc[e] * scale;
  if (accumulate) {
    float o[8];
    load8(out, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += o[e];
  }
  store8(out, v);
}

template <bool PAST>
__device__ __forceinline__ void clear_row(float* row, int hidden, int lane) {
  for (int c = lane * 4; c < hidden; c += 256) store16<PAST>(row + c, u32x4_t{0u, 0u, 0u, 0u});
}

struct EmbeddingSum {
  int tokens, hidden, rows, chunk, accumulate;
  float scale;
  const int* key;   // [tokens] rows in order, `rows` for tokens without one
  const int* tok;   // [tokens] the tokens in that order
  float* part;      // [chunks][2][hidden]
  int* split;       // split[0]: how many runs are split, then the chunks in which they begin
  float* out;       // [rows][hidden]
  int sum_blocks;   // workgroups that sum; the rest clear fill_rows rows each, from row0 on
  int fill_rows, row0;
  int width;        // columns of a workgroup of embedding_direct_kernel, a multiple of kSlab
};

// Tokens of the run across the border at sorted position p > 0, counted to both sides of
// it and up to kWhole each (0, 0: no run crosses it).  k: the lane's key, at p - 32 + lane.
struct Across {
  int before, after;
  __device__ __forceinline__ bool whole() const { return before + after <= kWhole; }
};

__device__ __forceinline__ int key_at(const EmbeddingSum& a, int p) { return p >= 0 && p < a.tokens ? a.key[p] : -1; }

__device__ __forceinline__ Across run_across(const EmbeddingSum& a, int p, int k) {
  static_assert(kWhole == 32, "a half of the wave looks at each side");
  const int here = __builtin_amdgcn_readlane(k, 32);
  const unsigned long long same = __ballot(k == here && here < a.rows && p > 0 && p < a.tokens);
  const unsigned lo = ~(unsigned)same, hi = ~(unsigned)(same >> 32);
  const int before = lo ? __builtin_clz(lo) : 32;
  if (before == 0) return {0, 0};
  return {before, hi ? __builtin_ctz(hi) : 32};
}

// Sums over runs of equal rows.  A wave takes 512 columns of the runs that begin in
// `chunk` sorted positions, and adds the tokens of a run in order.  A run of up to kWhole
// tokens is finished by the chunk in which it begins, wherever it ends.  Of a longer
// one that crosses chunks each chunk adds its own positions, into part[c][1] if the run
// begins in the chunk, else into part[c][0]; the chunk in which it begins is noted, and
// embedding_join_kernel adds the parts.
// The workgroups after those clear the rows that no token names, so that reading dy and
// writing the table overlap: 16384 tokens of 1920 on 25152 rows (225 MB) 39 us, 5.7 TB/s.
template <typename T, bool PAST>
__global__ void __launch_bounds__(256) embedding_sum_kernel(EmbeddingSum a, const T* __restrict__ dy) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= a.sum_blocks) {
    __shared__ int used[kFillRows];
    const int r0 = a.row0 + (blockIdx.x - a.sum_blocks) * a.fill_rows;
    static_assert(kFillRows * 16 == 256, "16 lanes look for a row");
    const int r = r0 + (threadIdx.x >> 4);
    const int p = (int)threadIdx.x >> 4 < a.fill_rows ? lower_bound16(a.key, a.tokens, r, lane) : 0;
    if ((lane & 15) == 0) used[threadIdx.x >> 4] = p < a.tokens && a.key[p] == r;
    __syncthreads();
    for (int i = w; i < a.fill_rows && r0 + i < a.rows; i += 4)
      if (!used[i]) clear_row<PAST>(a.out + (size_t)(r0 + i) * a.hidden, a.hidden, lane);
    return;
  }
  const int slabs = (a.hidden + kSlab - 1) / kSlab;
  const int unit = blockIdx.x * 4 + w;
  const int c = unit / slabs, slab = unit % slabs, col = slab * kSlab + lane * 8;
  const int lo = c * a.chunk, hi = min(lo + a.chunk, a.tokens);
  if (lo >= a.tokens) return;
  const bool live = col < a.hidden;
  // All keys that the borders and the first 64 positions need, in one step: every load
  // here waits for another kernel's stores.
  const int k_lo = key_at(a, lo - 32 + lane), k_hi = key_at(a, hi - 32 + lane);
  int k_here = key_at(a, lo + lane), t_here = lo + lane < a.tokens ? a.tok[lo + lane] : 0;
  const Across first = run_across(a, lo, k_lo), last = run_across(a, hi, k_hi);
  const int begin = first.whole() ? lo + first.after : lo;
  if (begin >= hi) return;  // all of it belongs to a run that began before
  const int end = last.whole() ? hi + last.after : hi;
  // a split run's row at either end
  const int before = first.before && !first.whole() ? __builtin_amdgcn_readlane(k_lo, 32) : -1;
  const int after = last.before && !last.whole() ? __builtin_amdgcn_readlane(k_hi, 32) : -1;
  int cur = -1;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  float* head = a.part + ((size_t)c * 2) * a.hidden + col;
  for (int base = lo; base < end; base += 64) {
    if (base > lo) {
      k_here = key_at(a, base + lane);
      t_here = base + lane < a.tokens ? a.tok[base + lane] : 0;
    }
    const int m = min(64, end - base);
    constexpr int U = sizeof(T) == 2 ? 16 : 8;  // rows in flight
    constexpr int W = sizeof(T) / 2;            // 16-byte pieces of 8 columns
    for (int i = base == lo ? begin - lo : 0; i < m; i += U) {
      u32x4_t v[U][W];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= m || __builtin_amdgcn_readlane(k_here, (i + u) & 63) >= a.rows) break;  // no more rows
        const T* p = dy + (size_t)__builtin_amdgcn_readlane(t_here, (i + u) & 63) * a.hidden + col;
        if (live) {
#pragma unroll
          for (int e = 0; e < W; ++e) v[u][e] = reinterpret_cast<const u32x4_t*>(p)[e];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= m) break;
        const int k = __builtin_amdgcn_readlane(k_here, (i + u) & 63);
        if (k != cur) {
          if (cur >= 0 && live) {
            if (cur == before) store8(head, acc);
            else write_row(a.out + (size_t)cur * a.hidden + col, acc, a.scale, a.accumulate);
          }
          cur = k < a.rows ? k : -1;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        }
        if (cur < 0) break;  // only tokens without a row from here on
        float f[8];
        unpack_row<T>(v[u], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += f[e];
      }
    }
  }
  if (cur < 0) return;
  if (cur == before) {
    if (live) store8(head, acc);
  } else if (cur == after) {
    if (live) store8(head + a.hidden, acc);
    if (slab == 0 && lane == 0) a.split[1 + atomicAdd(a.split, 1)] = c;
  } else if (live) {
    write_row(a.out + (size_t)cur * a.hidden + col, acc, a.scale, a.accumulate);
  }
}

// Adds the parts of the split runs: a workgroup takes a run and 512 columns at a time, its
// 16 waves every 16th part, and their sums are added in wave order.  (The runs are
// listed in any order; each one's sum has its own.)  The most frequent of 16384 tokens has
// 90 parts: 6 us.
constexpr int kJoinWaves = 16, kJoinBlocks = 128;

__global__ void __launch_bounds__(64 * kJoinWaves) embedding_join_kernel(EmbeddingSum a) {
  static_assert(64 * kJoinWaves >= kMaxChunks, "a thread a chunk");
  __shared__ float red[kJoinWaves - 1][64][9];
  const int slabs = (a.hidden + kSlab - 1) / kSlab;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int items = a.split[0] * slabs;
  for (int item = blockIdx.x; item < items; item += kJoinBlocks) {
    const int c = a.split[1 + item / slabs];
    const int k = a.key[(c + 1) * a.chunk - 1];
    // the chunks after c that begin inside the run (there are at most kMaxChunks)
    const long long at = (long long)(c + 1 + (int)threadIdx.x) * a.chunk;
    const int last = c + __syncthreads_count(at < a.tokens && a.key[at] == k);
    const int col = (item % slabs) * kSlab + lane * 8;
    const bool live = col < a.hidden;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
    if (live) {
#pragma unroll 8
      for (int i = c + w; i <= last; i += kJoinWaves) {
        float v[8];
        load8(a.part + ((size_t)i * 2 + (i == c)) * a.hidden + col, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[e];
      }
    }
    if (w > 0)
#pragma unroll
      for (int e = 0; e < 8; ++e) red[w - 1][lane][e] = acc[e];
    __syncthreads();
    if (w == 0 && live) {
      for (int i = 0; i < kJoinWaves - 1; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += red[i][lane][e];
      write_row(a.out + (size_t)k * a.hidden + col, acc, a.scale, a.accumulate);
    }
    __syncthreads();
  }
}

// Up to kDirect tokens, in one launch without sorting.  Every workgroup brings the tokens'
// rows into LDS.  A wave takes a token and `width` columns; if no earlier token has its
// row, it lists the row's tokens and adds them in order.  Rows of more than kAlone tokens are
// shared by the workgroup's four waves (each lists every fourth 64 tokens'), and the
// waves' sums are added in order.
constexpr int kAlone = 64;

// Appends the tokens of row k among tokens 64 q .. 64 q + 63 to the wave's list.
__device__ __forceinline__ int list_row(const int* key, int k, int q, int lane, unsigned short* list, int n) {
  const bool hit = key[64 * q + lane] == k;
  const unsigned long long m = __ballot(hit);
  if (hit) list[n + __builtin_popcountll(m & ((1ull << lane) - 1))] = (unsigned short)(64 * q + lane);
  return n + __builtin_popcountll(m);
}

// Sum of the listed tokens' 8 columns from col on (which the row has).
template <typename T>
__device__ __forceinline__ void add_listed(const EmbeddingSum& a, const T* dy, int col, const unsigned short* list,
                                           int n, float acc[8]) {
  constexpr int U = sizeof(T) == 2 ? 16 : 8;  // rows in flight
  constexpr int W = sizeof(T) / 2;            // 16-byte pieces of 8 columns
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  for (int i = 0; i < n; i += U) {
    u32x4_t v[U][W];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < W; ++e) v[u][e] = u32x4_t{0u, 0u, 0u, 0u};
      if (i + u < n) {
        const T* p = dy + (size_t)__builtin_amdgcn_readfirstlane(list[i + u]) * a.hidden + col;
#pragma unroll
        for (int e = 0; e < W; ++e) v[u][e] = reinterpret_cast<const u32x4_t*>(p)[e];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[8];
      unpack_row<T>(v[u], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f[e];
    }
  }
}

template <typename T, typename I, bool PAST>
__global__ void __launch_bounds__(256) embedding_direct_kernel(EmbeddingSum a, long long first,
                                                               const I* __restrict__ ids, const T* __restrict__ dy) {
  constexpr int PER = kDirect / 256;
  __shared__ int key[kDirect];
  __shared__ unsigned short lists[4][kDirect];
  __shared__ float red[3][64][9];
  __shared__ int flag[kFillRows];  // rows in use, or the waves' long rows' tokens
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool fill = (int)blockIdx.x >= a.sum_blocks;
  const int r0 = a.row0 + (blockIdx.x - a.sum_blocks) * a.fill_rows;
  if (threadIdx.x < kFillRows) flag[threadIdx.x] = fill ? 0 : -1;
  I id[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int t = 256 * u + threadIdx.x;
    id[u] = t < a.tokens ? ids[t] : (I)0;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int t = 256 * u + threadIdx.x;
    const int k = t < a.tokens ? table_row(id[u], first, a.rows) : a.rows;
    if (!fill) key[t] = k;
    else if (k >= r0 && k < r0 + a.fill_rows && k < a.rows) flag[k - r0] = 1;
  }
  __syncthreads();
  if (fill) {
    for (int i = w; i < a.fill_rows && r0 + i < a.rows; i += 4)
      if (!flag[i]) clear_row<PAST>(a.out + (size_t)(r0 + i) * a.hidden, a.hidden, lane);
    return;
  }
  const int groups = (a.tokens + 63) >> 6, parts = (a.hidden + a.width - 1) / a.width;
  const int t = (blockIdx.x / parts) * 4 + w;
  const int col0 = (blockIdx.x % parts) * a.width, col1 = min(col0 + a.width, a.hidden);  // this workgroup's columns
  const int k = t < a.tokens ? __builtin_amdgcn_readfirstlane(key[t]) : a.rows;
  unsigned short* list = lists[w];
  int n = 0;
  if (k < a.rows) {
    bool earlier = false;
    for (int q = 0; q < t >> 6 && !earlier; ++q) earlier = __ballot(key[64 * q + lane] == k) != 0ull;
    earlier = earlier || (__ballot(key[(t & ~63) + lane] == k) & ((1ull << (t & 63)) - 1)) != 0ull;
    if (!earlier)
      for (int q = t >> 6; q < groups; ++q) n = list_row(key, k, q, lane, list, n);
  }
  if (n > kAlone) {
    if (lane == 0) flag[w] = t;
  } else if (n > 0) {
    for (int col = col0 + lane * 8; col < col1; col += kSlab) {
      float acc[8];
      add_listed(a, dy, col, list, n, acc);
      write_row(a.out + (size_t)k * a.hidden + col, acc, a.scale, a.accumulate);
    }
  }
  __syncthreads();
  for (int i = 0; i < 4; ++i) {
    const int head = flag[i];
    if (head < 0) continue;
    const int row = __builtin_amdgcn_readfirstlane(key[head]);
    n = 0;
    for (int q = w; q < groups; q += 4) n = list_row(key, row, q, lane, list, n);
    for (int c = col0; c < col1; c += kSlab) {
      const int col = c + lane * 8;
      const bool live = col < col1;
      float acc[8];
      if (live) add_listed(a, dy, col, list, n, acc);
      if (w > 0 && live)
#pragma unroll
        for (int e = 0; e < 8; ++e) red[w - 1][lane][e] = acc[e];
      __syncthreads();
      if (w == 0 && live) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += red[j][lane][e];
        write_row(a.out + (size_t)row * a.hidden + col, acc, a.scale, a.accumulate);
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
template <typename T, typename I>
static hipError_t fwd_t(int tokens, int hidden, int rows, long long first, float scale, const void* ids,
                        const void* table, void* y, hipStream_t s) {
  const long long chunks = (long long)tokens * (hidden / (16 / (int)sizeof(T)));
  const long long wg = (chunks + 256 * kFwdUnroll - 1) / (256 * kFwdUnroll);
  if (wg > max_groups(256)) return hipErrorInvalidConfiguration;
  const bool past = (size_t)tokens * hidden * sizeof(T) >= kStreamBytes;
  hipLaunchKernelGGL((past ? embedding_fwd_kernel<T, I, true> : embedding_fwd_kernel<T, I, false>), dim3((unsigned)wg),
                     dim3(256), 0, s, tokens, hidden, rows, first, scale, (const I*)ids, (const T*)table, (T*)y);
  return hipGetLastError();
}

hipError_t launch_embedding_fwd(int dtype, int id_type, int tokens, int hidden, int rows, long long first, float scale,
                                const void* ids, const void* table, void* y, hipStream_t s) {
  if (dtype == DT_BF16)
    return id_type == ID_I32 ? fwd_t<bf16_t, int>(tokens, hidden, rows, first, scale, ids, table, y, s)
                             : fwd_t<bf16_t, long long>(tokens, hidden, rows, first, scale, ids, table, y, s);
  return id_type == ID_I32 ? fwd_t<float, int>(tokens, hidden, rows, first, scale, ids, table, y, s)
                           : fwd_t<float, long long>(tokens, hidden, rows, first, scale, ids, table, y, s);
}

// Scratch: the sorted blocks' rows and tokens, the whole order's rows and tokens, the
// list of split runs, and their parts.
// (The orders are held in whole blocks: embedding_merge_kernel reads them so.)
static size_t order_bytes(int tokens) { return ((size_t)tokens + kSortBlock - 1) / kSortBlock * kSortBlock * 4; }

size_t embedding_scratch_bytes(int tokens, int hidden) {
  if (tokens <= kDirect) return 0;
  const int len = chunk_len(tokens);
  const size_t chunks = ((size_t)tokens + len - 1) / len;
  return 4 * order_bytes(tokens) + order_bytes(1 + kMaxChunks) + chunks * 2 * hidden * sizeof(float);
}

// Launch of a kernel whose workgroups sum and clear.  What one launch cannot clear (from 2^28
// rows of few columns on) further ones do, which sum nothing.
template <typename... P, typename... A>
static hipError_t launch_sum_and_clear(void (*kernel)(EmbeddingSum, P...), EmbeddingSum a, hipStream_t s, A... args) {
  long long left = a.accumulate ? 0 : ((long long)a.rows + a.fill_rows - 1) / a.fill_rows;
  do {
    const long long fill = std::min(left, max_groups(256) - a.sum_blocks);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.sum_blocks + fill)), dim3(256), 0, s, a, args...);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.row0 += (int)fill * a.fill_rows;
    a.sum_blocks = 0;
    left -= fill;
  } while (left > 0);
  return hipSuccess;
}

template <typename T, typename I>
static hipError_t bwd_t(EmbeddingSum a, long long first, const void* ids, const void* dy, char* scratch,
                        hipStream_t s) {
  const long long slabs = (a.hidden + kSlab - 1) / kSlab;
  const bool past = (size_t)a.rows * a.hidden * sizeof(float) >= kStreamBytes;
  // four rows or more, at most 16, of about kFillBytes together
  a.fill_rows = std::min(kFillRows, std::max(4, (int)(kFillBytes / (a.hidden * sizeof(float)))));
  if (a.tokens <= kDirect) {
    // 512 columns a workgroup, more where that makes over 2048 workgroups, each of which reads
    // all ids.
    const long long quads = (a.tokens + 3) / 4, per = (quads * slabs + 2047) / 2048;
    a.width = (int)(per * kSlab);
    a.sum_blocks = (int)(quads * ((slabs + per - 1) / per));
    return launch_sum_and_clear((past ? embedding_direct_kernel<T, I, true> : embedding_direct_kernel<T, I, false>), a,
                                s, first, (const I*)ids, (const T*)dy);
  }
  const size_t ob = order_bytes(a.tokens);
  int* gkey = (int*)scratch;
  int* gtok = (int*)(scratch + ob);
  int* skey = (int*)(scratch + 2 * ob);
  int* stok = (int*)(scratch + 3 * ob);
  a.split = (int*)(scratch + 4 * ob);
  const unsigned wg = (unsigned)((a.tokens + 63) / 64);
  hipLaunchKernelGGL((embedding_rank_kernel<I>), dim3(wg), dim3(64 * kRankWaves), 0, s, a.tokens, a.rows, first,
                     (const I*)ids, skey, stok, a.split);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int waves = std::min(kMergeWaves, (a.tokens + kSortBlock - 1) / kSortBlock);
  const size_t lds = (size_t)waves * (kSortBlock + 64) * sizeof(int);
  static std::atomic<uint64_t> lds_set{0};
  e = allow_dynamic_lds(reinterpret_cast<const void*>(embedding_merge_kernel),
                        (size_t)kMergeWaves * (kSortBlock + 64) * sizeof(int), lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embedding_merge_kernel, dim3(wg), dim3(64 * waves), lds, s, a.tokens, skey, stok, gkey, gtok);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.chunk = chunk_len(a.tokens);
  a.key = gkey;
  a.tok = gtok;
  a.part = (float*)(scratch + 4 * ob + order_bytes(1 + kMaxChunks));
  const long long units = (((long long)a.tokens + a.chunk - 1) / a.chunk) * slabs;
  a.sum_blocks = (int)((units + 3) / 4);
  e = launch_sum_and_clear((past ? embedding_sum_kernel<T, true> : embedding_sum_kernel<T, false>), a, s,
                           (const T*)dy);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embedding_join_kernel, dim3(kJoinBlocks), dim3(64 * kJoinWaves), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_embedding_bwd(int dtype, int id_type, int tokens, int hidden, int rows, long long first, float scale,
                                const void* ids, const void* dy, float* dtable, int accumulate, void* scratch,
                                hipStream_t s) {
  EmbeddingSum a{};
  a.tokens = tokens;
  a.hidden = hidden;
  a.rows = rows;
  a.accumulate = accumulate;
  a.scale = scale;
  a.out = dtable;
  char* sc = (char*)scratch;
  if (dtype == DT_BF16)
    return id_type == ID_I32 ? bwd_t<bf16_t, int>(a, first, ids, dy, sc, s)
                             : bwd_t<bf16_t, long long>(a, first, ids, dy, sc, s);
  return id_type == ID_I32 ? bwd_t<float, int>(a, first, ids, dy, sc, s)
                           : bwd_t<float, long long>(a, first, ids, dy, sc, s);
}

}  // namespace merak
