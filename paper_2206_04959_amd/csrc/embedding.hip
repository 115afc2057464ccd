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
// consecutive chunks of y.
// ---------------------------------------------------------------------------
constexpr int kFwdUnroll = 4;

template <typename T, typename I>
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
    if constexpr (sizeof(T) == 2) {
      float f[8];
      unpack8(v[u], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= scale;
      store8(y + at[u], f);
    } else {
      const f32x4_t f = __builtin_bit_cast(f32x4_t, v[u]);
      const float o[4] = {f[0] * scale, f[1] * scale, f[2] * scale, f[3] * scale};
      store4(y + at[u], o);
    }
  }
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------
constexpr int kDirect = 256;      // up to here one launch, without sorting
constexpr int kSortBlock = 2048;  // tokens that are ranked against each other
constexpr int kFillRows = 16;     // table rows that a workgroup clears
constexpr int kSlab = 512;        // columns of a wave: 8 a lane
constexpr int kMinChunk = 16, kMaxChunks = 1024;

// Sorted positions per unit of work: at most kMaxChunks units, whole multiples
// of 16 positions.
static inline int chunk_len(int tokens) {
  const int c = (tokens + kMaxChunks - 1) / kMaxChunks;
  return std::max(kMinChunk, (c + 15) / 16 * 16);
}

// Rank of each token within its block of kSortBlock by (row, token): the number of
// tokens of the block that come before it.  A workgroup ranks 64 tokens, each of its
// eight waves against an eighth of the block.  Comparing every pair costs two
// instructions a pair and no dependence between them, in one launch; the keys go
// through LDS as four-key reads that all lanes share.
constexpr int kRankWaves = 8;

template <typename I>
__global__ void __launch_bounds__(64 * kRankWaves) embedding_rank_kernel(int tokens, int rows, long long first,
                                                                         const I* __restrict__ ids,
                                                                         int* __restrict__ skey,
                                                                         int* __restrict__ stok) {
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
    for (int j = lo; j < hi; j += 16) {
      u32x4_t v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const u32x4_t*>(key + j + 4 * u);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) n += v[u][e] < thr;
    }
  };
  const int lo = w * Q, hi = min(lo + Q, (m + 63) & ~63);
  count(lo, min(hi, slice), k + 1);
  count(max(lo, slice + 64), hi, k);
  if (slice >= lo && slice < hi) {
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
// before it in each block, found by binary search.  A workgroup places 64 tokens,
// its 16 waves search every 16th block: a search is a chain of 12 loads, so they are
// spread wide.
constexpr int kMergeWaves = 16;

__global__ void __launch_bounds__(64 * kMergeWaves) embedding_merge_kernel(int tokens, const int* __restrict__ skey,
                                                                           const int* __restrict__ stok,
                                                                           int* __restrict__ gkey,
                                                                           int* __restrict__ gtok) {
  __shared__ int cnt[kMergeWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int p = blockIdx.x * 64 + lane;
  const int b = blockIdx.x * 64 / kSortBlock, nb = (tokens + kSortBlock - 1) / kSortBlock;
  const int k = p < tokens ? skey[p] : 0;
  const int t = p < tokens ? stok[p] : 0;
  int n = w == b % kMergeWaves ? p - b * kSortBlock : 0;  // those of its own block
  for (int o = w; o < nb; o += kMergeWaves) {
    if (o == b) continue;
    const int* kb = skey + (size_t)o * kSortBlock;
    const int m = min(kSortBlock, tokens - o * kSortBlock);
    const int thr = o < b ? k + 1 : k;
    int pos = 0;  // tokens known to come before
#pragma unroll
    for (int step = kSortBlock; step > 0; step >>= 1)
      if (pos + step <= m && kb[pos + step - 1] < thr) pos += step;
    n += pos;
  }
  cnt[w][lane] = n;
  __syncthreads();
  if (w == 0 && p < tokens) {
    int g = 0;
#pragma unroll
    for (int i = 0; i < kMergeWaves; ++i) g += cnt[i][lane];
    gkey[g] = k;
    gtok[g] = t;
  }
}

// First sorted position whose row is not below r.
__device__ __forceinline__ int lower_bound(const int* key, int n, int r) {
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1;
    if (key[lo + half] < r) {
      lo += half + 1;
      n -= half + 1;
    } else {
      n = half;
    }
  }
  return lo;
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

__device__ __forceinline__ void clear_row(float* row, int hidden, int lane) {
  for (int c = lane * 4; c < hidden; c += 256) *reinterpret_cast<f32x4_t*>(row + c) = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
}

struct EmbeddingSum {
  int tokens, hidden, rows, chunk, accumulate;
  float scale;
  const int* key;   // [tokens] rows in order, `rows` for tokens without one
  const int* tok;   // [tokens] the tokens in that order
  float* part;      // [chunks][2][hidden]
  float* out;       // [rows][hidden]
  int sum_blocks;   // workgroups that sum; the rest clear rows
};

// Sums over runs of equal rows.  A wave takes `chunk` sorted positions and 512
// columns and adds the tokens of a run in order.  A run within the chunk is
// finished here.  Of a run that other chunks share, the chunk's part goes to
// part[c][1] if the run begins in the chunk, else to part[c][0];
// embedding_join_kernel adds them up.
// The workgroups after those clear the rows that no token names.
template <typename T>
__global__ void __launch_bounds__(256) embedding_sum_kernel(EmbeddingSum a, const T* __restrict__ dy) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= a.sum_blocks) {
    __shared__ int used[kFillRows];
    const int r0 = (blockIdx.x - a.sum_blocks) * kFillRows;
    if (threadIdx.x < kFillRows) {
      const int r = r0 + threadIdx.x;
      const int p = lower_bound(a.key, a.tokens, r);
      used[threadIdx.x] = p < a.tokens && a.key[p] == r;
    }
    __syncthreads();
    for (int i = w; i < kFillRows && r0 + i < a.rows; i += 4)
      if (!used[i]) clear_row(a.out + (size_t)(r0 + i) * a.hidden, a.hidden, lane);
    return;
  }
  const int slabs = (a.hidden + kSlab - 1) / kSlab;
  const int unit = blockIdx.x * 4 + w;
  const int c = unit / slabs, col = (unit % slabs) * kSlab + lane * 8;
  const int lo = c * a.chunk, hi = min(lo + a.chunk, a.tokens);
  if (lo >= a.tokens) return;
  const bool live = col < a.hidden;
  const int before = lo > 0 ? a.key[lo - 1] : -1;
  const int after = hi < a.tokens ? a.key[hi] : -1;
  int cur = -1;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  float* head = a.part + ((size_t)c * 2) * a.hidden + col;
  for (int base = lo; base < hi; base += 64) {
    const int m = min(64, hi - base);
    const int kk = lane < m ? a.key[base + lane] : a.rows;
    const int tt = lane < m ? a.tok[base + lane] : 0;
    constexpr int U = 4;
    for (int i = 0; i < m; i += U) {
      float v[U][8];
      int k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        k[u] = __builtin_amdgcn_readlane(kk, i + u);  // i + u < 64; lanes past m hold `rows`
        const size_t t = (size_t)__builtin_amdgcn_readlane(tt, i + u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
        if (live && k[u] < a.rows) load8(dy + t * a.hidden + col, v[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k[u] != cur) {
          if (cur >= 0 && live) {
            if (cur == before) store8(head, acc);
            else write_row(a.out + (size_t)cur * a.hidden + col, acc, a.scale, a.accumulate);
          }
          cur = k[u] < a.rows ? k[u] : -1;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[u][e];
      }
      if (k[U - 1] >= a.rows) break;  // only tokens without a row from here on
    }
  }
  if (cur >= 0 && live) {
    if (cur == before) store8(head, acc);
    else if (cur == after) store8(head + a.hidden, acc);
    else write_row(a.out + (size_t)cur * a.hidden + col, acc, a.scale, a.accumulate);
  }
}

// Adds the parts of a run that spans chunks, for the chunk in which it begins:
// eight waves take every eighth part, and their sums are added in wave order.
constexpr int kJoinWaves = 8;

__global__ void __launch_bounds__(64 * kJoinWaves) embedding_join_kernel(EmbeddingSum a) {
  __shared__ float red[kJoinWaves - 1][64][9];
  const int slabs = (a.hidden + kSlab - 1) / kSlab;
  const int c = blockIdx.x / slabs;
  const int lo = c * a.chunk, hi = min(lo + a.chunk, a.tokens);
  if (hi >= a.tokens) return;
  const int k = a.key[hi - 1];
  if (k >= a.rows || a.key[hi] != k || (lo > 0 && a.key[lo - 1] == k)) return;
  const int end = lower_bound(a.key, a.tokens, k + 1) - 1;  // last position of the run
  const int last = end / a.chunk;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = (blockIdx.x % slabs) * kSlab + lane * 8;
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
#pragma unroll
    for (int i = 0; i < kJoinWaves - 1; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += red[i][lane][e];
    write_row(a.out + (size_t)k * a.hidden + col, acc, a.scale, a.accumulate);
  }
}

// Up to kDirect tokens: every wave holds all rows in its lanes, four a lane.  A wave per
// token and 512 columns; the first token of a row adds the row's tokens in order.
template <typename T, typename I>
__global__ void __launch_bounds__(256) embedding_direct_kernel(EmbeddingSum a, long long first,
                                                               const I* __restrict__ ids, const T* __restrict__ dy) {
  constexpr int KG = kDirect / 64;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int key[KG];
#pragma unroll
  for (int g = 0; g < KG; ++g) {
    const int t = 64 * g + lane;
    key[g] = t < a.tokens ? table_row(ids[t], first, a.rows) : a.rows;
  }
  if ((int)blockIdx.x >= a.sum_blocks) {
    const int r0 = (blockIdx.x - a.sum_blocks) * kFillRows;
    for (int i = w; i < kFillRows && r0 + i < a.rows; i += 4) {
      bool used = false;
#pragma unroll
      for (int g = 0; g < KG; ++g) used |= key[g] == r0 + i;
      if (__ballot(used) == 0ull) clear_row(a.out + (size_t)(r0 + i) * a.hidden, a.hidden, lane);
    }
    return;
  }
  const int slabs = (a.hidden + kSlab - 1) / kSlab;
  const int unit = blockIdx.x * 4 + w;
  const int t = unit / slabs, col = (unit % slabs) * kSlab + lane * 8;
  if (t >= a.tokens) return;
  int k = a.rows;
#pragma unroll
  for (int g = 0; g < KG; ++g)
    if (t >> 6 == g) k = __builtin_amdgcn_readlane(key[g], t & 63);
  if (k >= a.rows) return;
  unsigned long long run[KG];
  int head = -1;  // the row's first token
#pragma unroll
  for (int g = KG - 1; g >= 0; --g) {
    run[g] = __ballot(key[g] == k);
    if (run[g]) head = 64 * g + __builtin_ctzll(run[g]);
  }
  if (head != t) return;
  const bool live = col < a.hidden;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int g = 0; g < KG; ++g) {
    unsigned long long r = run[g];
    while (r) {
      constexpr int U = 8;  // rows in flight
      float v[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
        if (r) {
          if (live) load8(dy + (size_t)(64 * g + __builtin_ctzll(r)) * a.hidden + col, v[u]);
          r &= r - 1;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[u][e];
    }
  }
  if (live) write_row(a.out + (size_t)k * a.hidden + col, acc, a.scale, a.accumulate);
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
template <typename T, typename I>
static hipError_t fwd_t(int tokens, int hidden, int rows, long long first, float scale, const void* ids,
                        const void* table, void* y, hipStream_t s) {
  const long long chunks = (long long)tokens * (hidden / (16 / (int)sizeof(T)));
  const long long wg = (chunks + 256 * kFwdUnroll - 1) / (256 * kFwdUnroll);
  if (wg > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((embedding_fwd_kernel<T, I>), dim3((unsigned)wg), dim3(256), 0, s, tokens, hidden, rows, first,
                     scale, (const I*)ids, (const T*)table, (T*)y);
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

// Scratch: the sorted blocks' rows and tokens, the whole order's rows and
// tokens, and the parts of runs that span chunks.
static size_t order_bytes(int tokens) { return ((size_t)tokens * 4 + 255) / 256 * 256; }

size_t embedding_scratch_bytes(int tokens, int hidden) {
  if (tokens <= kDirect) return 0;
  const int len = chunk_len(tokens);
  const size_t chunks = ((size_t)tokens + len - 1) / len;
  return 4 * order_bytes(tokens) + chunks * 2 * hidden * sizeof(float);
}

template <typename T, typename I>
static hipError_t bwd_t(EmbeddingSum a, long long first, const void* ids, const void* dy, char* scratch,
                        hipStream_t s) {
  const long long slabs = (a.hidden + kSlab - 1) / kSlab;
  const long long fill = a.accumulate ? 0 : ((long long)a.rows + kFillRows - 1) / kFillRows;
  if (a.tokens <= kDirect) {
    a.sum_blocks = (int)((a.tokens * slabs + 3) / 4);
    hipLaunchKernelGGL((embedding_direct_kernel<T, I>), dim3((unsigned)(a.sum_blocks + fill)), dim3(256), 0, s, a,
                       first, (const I*)ids, (const T*)dy);
    return hipGetLastError();
  }
  const size_t ob = order_bytes(a.tokens);
  int* gkey = (int*)scratch;
  int* gtok = (int*)(scratch + ob);
  int* skey = (int*)(scratch + 2 * ob);
  int* stok = (int*)(scratch + 3 * ob);
  const bool one = a.tokens <= kSortBlock;  // one block: its order is the whole order
  const unsigned wg = (unsigned)(((long long)a.tokens + 63) / 64);
  hipLaunchKernelGGL((embedding_rank_kernel<I>), dim3(wg), dim3(64 * kRankWaves), 0, s, a.tokens, a.rows, first, (const I*)ids,
                     one ? gkey : skey, one ? gtok : stok);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!one) {
    hipLaunchKernelGGL(embedding_merge_kernel, dim3(wg), dim3(64 * kMergeWaves), 0, s, a.tokens, skey, stok, gkey, gtok);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  a.chunk = chunk_len(a.tokens);
  a.key = gkey;
  a.tok = gtok;
  a.part = (float*)(scratch + 4 * ob);
  const long long units = (((long long)a.tokens + a.chunk - 1) / a.chunk) * slabs;
  a.sum_blocks = (int)((units + 3) / 4);
  hipLaunchKernelGGL(embedding_sum_kernel<T>, dim3((unsigned)(a.sum_blocks + fill)), dim3(256), 0, s, a,
                     (const T*)dy);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embedding_join_kernel, dim3((unsigned)units), dim3(64 * kJoinWaves), 0, s, a);
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
