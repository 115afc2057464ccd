// RMS norm of each head's queries and keys with the position rotation in the same
// pass, and its gradient.
//
// A token's row holds q_heads + kv_heads + kv_heads heads of d features, [q | k | v].
// For every query and key head x with gain g (one for queries, one for keys):
//   n = x * rstd,  rstd = 1 / sqrt(mean(x^2) + eps),  z = n * g,
//   (a, b) -> (a c - b s, b c + a s)   for each rotated pair (a, b) of z, with
//   c, s the cosine and sine of the pair's angle at the token's position.
// Pairs are (z[i], z[i + r/2]) or, interleaved, (z[2i], z[2i + 1]), i < r/2; the
// features from r on are not rotated.
// Backward, with dz the upstream gradient rotated back:
//   dg = sum over tokens and heads of dz * n,
//   dx = rstd * (dz g - n * mean(dz g n)).
// rstd and n are rebuilt from x, which the gradient needs anyway, so nothing but
// the raw rows is kept for it.  Statistics and sums are fp32, outputs are rounded
// once.
//
// Bound by memory.  G lanes own a head, CH chunks of 8 features each; a workgroup holds
// 256 / G heads of one kind (queries or keys, so one gain) at a time, and others copy
// the values.  How the chunks lie on the lanes, so that loads cover whole segments and
// the two members of a pair meet cheaply:
//   64, 128, 256 features: two chunks a lane, half a head apart; pairs of a fully
//     rotated head lie in one lane;
//   96: three neighbouring chunks on each of four lanes, pairs in lanes that differ in
//     one bit;
//   any other head, or any other number of rotated features: one chunk a lane, pairs
//     anywhere in the group.
// In bf16, values copied: 32768 tokens of 20 + 20 heads of 96 163 us (4.6 TB/s; a large copy
// has 4.8 to 5.1), 16384 tokens of 12 + 12 of 128 64 (4.7), of 256 121 (5.0), of 80 67 (2.8:
// 6 of 16 lanes idle); in fp32 of 128 119 (5.1); gradients of 16384 tokens: 25 + 25 heads of 64
// 87 us (4.8), 12 + 12 of 128 84 (4.8), of 256 161 (5.0), of 96 72 (4.2: three waves a SIMD), of
// 80 77 (3.3); in fp32 of 128 162 (5.0).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "kernels.h"

namespace merak {

// cos and sin of a position's angles: [positions][rope_dim / 2][2].
__global__ void __launch_bounds__(256) rope_table_kernel(int positions, int half, double log_theta,
                                                         float* __restrict__ table) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)positions * half) return;
  const long long p = i / half;
  const int j = (int)(i - p * half);
  // in 64 bits: at position 2^17 a 32-bit angle is off by up to 2^-8
  const double a = (double)p * exp(-log_theta * (double)j / (double)half);
  double s, c;
  sincos(a, &s, &c);
  *reinterpret_cast<f32x2_t*>(table + 2 * i) = f32x2_t{(float)c, (float)s};
}

struct QkArgs {
  int tokens, q_heads, kv_heads, d;
  int rope;         // rotated features of a head
  int table_rows;
  int seq_len;      // without positions: token t of the call is at t % seq_len
  int first;        // the call's tokens before this launch's
  float eps;
  const int* positions;  // this launch's
  const float* table;
};

// The value of the lane whose number differs in bit(s) X.
template <int X>
__device__ __forceinline__ float xor_lane(float v) {
  const int i = __float_as_int(v);
  int r;
  if constexpr (X == 1) r = __builtin_amdgcn_update_dpp(0, i, 0xB1, 0xf, 0xf, true);        // quad_perm [1,0,3,2]
  else if constexpr (X == 2) r = __builtin_amdgcn_update_dpp(0, i, 0x4E, 0xf, 0xf, true);   // quad_perm [2,3,0,1]
  else if constexpr (X == 8) r = __builtin_amdgcn_update_dpp(0, i, 0x128, 0xf, 0xf, true);  // row_ror:8
  else r = __builtin_amdgcn_ds_swizzle(i, 0x1f | (X << 10));  // 4, 16: exclusive or within 32 lanes
  return __int_as_float(r);
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (G > 1) v += xor_lane<1>(v);
  if constexpr (G > 2) v += xor_lane<2>(v);
  if constexpr (G > 4) v += xor_lane<4>(v);
  if constexpr (G > 8) v += xor_lane<8>(v);
  if constexpr (G > 16) v += xor_lane<16>(v);
  return v;
}

// How the two members of a pair meet: neighbours (interleaved), in a lane's two chunks, in
// lanes that differ in one bit, or anywhere in the group.
enum { INTERLEAVED = 0, IN_LANE = -2, ANYWHERE = -1 };  // else the bit

// Chunk i of lane j.
template <int G, int CH>
__device__ __forceinline__ int chunk_of(int j, int i) {
  return CH == 2 ? j + G * i : j * CH + i;
}

// Rotation of a lane's features by its token's angles, forward (dir = 1) or back
// (dir = -1).  The lane is the group's j-th, `base` its first lane.  A position outside
// the table rotates by NaN.
template <int G, int CH, int MODE>
__device__ __forceinline__ void rotate(const QkArgs& a, int pos, int j, int base, float dir, float (&z)[CH][8]) {
  const bool in = pos >= 0 && pos < a.table_rows;
  const float* row = a.table + (size_t)(in ? pos : 0) * a.rope;  // rope / 2 pairs of floats
  if constexpr (MODE == INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = chunk_of<G, CH>(j, i);
      if (c * 8 >= a.rope) continue;
      float t[8];
      load8(row + c * 8, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float co = in ? t[2 * e] : NAN, si = (in ? t[2 * e + 1] : NAN) * dir;
        const float x = z[i][2 * e], y = z[i][2 * e + 1];
        z[i][2 * e] = x * co - y * si;
        z[i][2 * e + 1] = y * co + x * si;
      }
    }
  } else if constexpr (MODE == IN_LANE) {
    static_assert(CH == 2, "the lane's chunks are half a head apart");
    float t[16];
    load8(row + j * 16, t);
    load8(row + j * 16 + 8, t + 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float co = in ? t[2 * e] : NAN, si = (in ? t[2 * e + 1] : NAN) * dir;
      const float x = z[0][e], y = z[1][e];
      z[0][e] = x * co - y * si;
      z[1][e] = y * co + x * si;
    }
  } else {
    constexpr int ROT = CH == 2 ? 1 : CH;    // chunks of a lane that are rotated (CH = 2: the lower half of a head)
    const int lanes = (a.rope >> 4) / ROT;   // lanes that hold the pairs' first members
    const bool low = j < lanes, rot = j < 2 * lanes;
    const float sign = low ? -dir : dir;
    const float* cs = row + (low ? j : j - lanes) * ROT * 16;
#pragma unroll
    for (int i = 0; i < ROT; ++i) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (MODE > 0) p[e] = xor_lane<(MODE > 0 ? MODE : 1)>(z[i][e]);
        else p[e] = __shfl(z[i][e], rot ? base + (low ? j + lanes : j - lanes) : base, 64);
      }
      if (!rot) continue;
      float t[16];
      load8(cs + i * 16, t);
      load8(cs + i * 16 + 8, t + 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float co = in ? t[2 * e] : NAN, si = (in ? t[2 * e + 1] : NAN) * sign;
        z[i][e] = z[i][e] * co + p[e] * si;
      }
    }
  }
}

__device__ __forceinline__ int position_of(const QkArgs& a, unsigned t) {
  return a.positions ? a.positions[t] : (int)((a.first + t) % (unsigned)a.seq_len);
}

// Workgroups of a launch: for queries, for keys, for copying values.
struct QkGrid {
  int q, k, v;
};

constexpr int kCopyUnroll = 4;  // 16-byte chunks of the values a thread moves

// Copy of the value heads by workgroup b.
template <typename T>
__device__ __forceinline__ void copy_values(const QkArgs& a, unsigned b, const T* in, T* out) {
  constexpr unsigned EPC = 16 / sizeof(T);
  const unsigned per = a.kv_heads * a.d / EPC;  // chunks of a row's values
  const size_t row = (size_t)(a.q_heads + 2 * a.kv_heads) * a.d, skip = (size_t)(a.q_heads + a.kv_heads) * a.d;
  const unsigned long long first = (unsigned long long)b * (256 * kCopyUnroll);
  const unsigned t0 = (unsigned)(first / per), c0 = (unsigned)(first % per);
  u32x4_t v[kCopyUnroll];
  size_t at[kCopyUnroll];
  bool live[kCopyUnroll];
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u) {
    const unsigned local = c0 + threadIdx.x + 256 * u, dt = local / per;
    live[u] = (unsigned long long)t0 + dt < (unsigned)a.tokens;
    at[u] = ((size_t)t0 + dt) * row + skip + (size_t)(local - dt * per) * EPC;
    if (live[u]) v[u] = *reinterpret_cast<const u32x4_t*>(in + at[u]);
  }
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u)
    if (live[u]) *reinterpret_cast<u32x4_t*>(out + at[u]) = v[u];
}

// The heads of one kind, numbered through all tokens: token and head of number
// first + i, first a workgroup's first.
struct HeadRange {
  int heads, head0;
  unsigned t0, h0;
  __device__ __forceinline__ HeadRange(int heads, int head0, unsigned long long first)
      : heads(heads), head0(head0), t0((unsigned)(first / heads)), h0((unsigned)(first % heads)) {}
  // Element of the head in a row-major [tokens][row heads][d]; *t is its token.
  __device__ __forceinline__ size_t at(unsigned i, const QkArgs& a, unsigned* t) const {
    const unsigned local = h0 + i, dt = local / (unsigned)heads;
    *t = t0 + dt;
    return ((size_t)*t * (a.q_heads + 2 * a.kv_heads) + head0 + (local - dt * heads)) * a.d;
  }
};

// Lane j's chunks of a head at p.
template <int G, int CH, typename T>
__device__ __forceinline__ void load_chunks(const T* p, int j, int d, float (&v)[CH][8]) {
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = chunk_of<G, CH>(j, i) * 8;
    if (CH > 1 || c < d) {  // (a head fills its lanes where they hold more than one chunk)
      load8(p + c, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
    }
  }
}

template <int G, int CH, typename T>
__device__ __forceinline__ void store_chunks(T* p, int j, int d, const float (&v)[CH][8]) {
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = chunk_of<G, CH>(j, i) * 8;
    if (CH > 1 || c < d) store8(p + c, v[i]);
  }
}

template <typename T, int G, int CH, int MODE>
__global__ void __launch_bounds__(256) qk_fwd_kernel(QkArgs a, QkGrid grid, const T* in, const T* __restrict__ gq,
                                                     const T* __restrict__ gk, T* out) {
  if ((int)blockIdx.x >= grid.q + grid.k) {
    copy_values(a, blockIdx.x - grid.q - grid.k, in, out);
    return;
  }
  const bool keys = (int)blockIdx.x >= grid.q;
  const unsigned b = blockIdx.x - (keys ? grid.q : 0);
  const HeadRange range(keys ? a.kv_heads : a.q_heads, keys ? a.q_heads : 0, (unsigned long long)b * (256 / G));
  const int lane = threadIdx.x & 63, j = lane & (G - 1), base = lane - j;
  unsigned t;
  const size_t at = range.at(threadIdx.x / G, a, &t);
  if (t >= (unsigned)a.tokens) return;  // whole groups leave: the exchanges stay within a group
  float x[CH][8], g[CH][8];
  load_chunks<G, CH>(in + at, j, a.d, x);
  const int pos = a.rope ? position_of(a, t) : 0;
  load_chunks<G, CH>(keys ? gk : gq, j, a.d, g);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[i][e] * x[i][e];
  const float rstd = 1.0f / sqrtf(group_sum<G>(s) / (float)a.d + a.eps);
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * rstd * g[i][e];
  if (a.rope) rotate<G, CH, MODE>(a, pos, j, base, 1.0f, x);
  store_chunks<G, CH>(out + at, j, a.d, x);
}

// Gradient: the workgroups of a kind step through its heads, each lane keeping the sums
// of its gain columns; a workgroup's sums go to part[workgroup][d], queries' first, and
// qk_gain_kernel adds those in order.  Without part each kind has one workgroup, whose
// sums are the gains' gradients.
template <typename T, int G, int CH, int MODE>
__global__ void __launch_bounds__(256) qk_bwd_kernel(QkArgs a, QkGrid grid, const T* dout, const T* __restrict__ in,
                                                     const T* __restrict__ gq, const T* __restrict__ gk, T* dx,
                                                     float* __restrict__ part, float* __restrict__ dgq,
                                                     float* __restrict__ dgk, int accumulate) {
  if ((int)blockIdx.x >= grid.q + grid.k) {
    copy_values(a, blockIdx.x - grid.q - grid.k, dout, dx);
    return;
  }
  __shared__ float red[4][G * CH * 8];
  const bool keys = (int)blockIdx.x >= grid.q;
  const unsigned b = blockIdx.x - (keys ? grid.q : 0), blocks = keys ? grid.k : grid.q;
  const int heads = keys ? a.kv_heads : a.q_heads;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, j = lane & (G - 1), base = lane - j;
  float g[CH][8], sum[CH][8];
  load_chunks<G, CH>(keys ? gk : gq, j, a.d, g);
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[i][e] = 0.0f;
  const unsigned long long total = (unsigned long long)a.tokens * heads;
  for (unsigned long long first = (unsigned long long)b * (256 / G); first < total;
       first += (unsigned long long)blocks * (256 / G)) {
    const HeadRange range(heads, keys ? a.q_heads : 0, first);
    unsigned t;
    const size_t at = range.at(threadIdx.x / G, a, &t);
    if (t >= (unsigned)a.tokens) continue;
    float dz[CH][8], x[CH][8];
    load_chunks<G, CH>(dout + at, j, a.d, dz);
    load_chunks<G, CH>(in + at, j, a.d, x);
    if (a.rope) rotate<G, CH, MODE>(a, position_of(a, t), j, base, -1.0f, dz);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[i][e] * x[i][e];
    const float rstd = 1.0f / sqrtf(group_sum<G>(s) / (float)a.d + a.eps);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] *= rstd;
        sum[i][e] += dz[i][e] * x[i][e];
        dz[i][e] *= g[i][e];
        m += dz[i][e] * x[i][e];
      }
    m = group_sum<G>(m) / (float)a.d;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) dz[i][e] = rstd * (dz[i][e] - x[i][e] * m);
    store_chunks<G, CH>(dx + at, j, a.d, dz);
  }
  // the wave's groups, then the four waves, as trees
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int off = G; off < 64; off <<= 1) sum[i][e] += __shfl_xor(sum[i][e], off, 64);
      if (lane < G) red[w][chunk_of<G, CH>(j, i) * 8 + e] = sum[i][e];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < a.d; i += 256) {
    const float v = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
    if (part) {
      part[(size_t)blockIdx.x * a.d + i] = v;
    } else {
      float* o = (keys ? dgk : dgq) + i;
      *o = accumulate ? *o + v : v;
    }
  }
}

// Gain gradients from the workgroups' sums, 16 columns of one gain a workgroup: 64
// threads a column take every 64th sum (16 in flight), and are added as a tree: in a chain
// the last additions' roundings were most of the result's (1023 tokens of 24 heads of 128 in
// fp32: off by 1.8e-7, 1.3e-7 so).  (One column a lane with 16 waves, the way the other
// column sums end, took 17 us for 1024 sums.)
__global__ void __launch_bounds__(1024) qk_gain_kernel(int d, QkGrid grid, const float* __restrict__ part,
                                                       float* __restrict__ dgq, float* __restrict__ dgk,
                                                       int accumulate) {
  __shared__ float red[64][17];
  const int per = (d + 15) / 16;  // workgroups of a gain
  const bool keys = (int)blockIdx.x >= per;
  const int col = (blockIdx.x - (keys ? per : 0)) * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
  const int n = keys ? grid.k : grid.q;
  const float* p = part + (size_t)(keys ? grid.q : 0) * d;
  float s = 0.0f;
  if (col < d) {
    constexpr int U = 16;
    for (int i = slice; i < n; i += 64 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = i + 64 * u < n ? p[(size_t)(i + 64 * u) * d + col] : 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
  }
  red[slice][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x < 16 && col < d) {
    float v[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = red[i][threadIdx.x];
#pragma unroll
    for (int n = 32; n > 0; n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) v[i] += v[i + n];
    float* o = (keys ? dgk : dgq) + col;
    *o = accumulate ? *o + v[0] : v[0];
  }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
// Lanes of a head, chunks of a lane and how its pairs meet (see the top).
struct QkLanes {
  int G, CH, mode;
};

static QkLanes lanes_of(const QkShape& q) {
  const int n = q.head_dim / 8;  // chunks
  const bool one = q.interleaved || q.rope_dim == 0;
  const bool full = q.rope_dim == q.head_dim, half = 2 * q.rope_dim == q.head_dim;
  if (one || full || half) {
    if (n == 8 || n == 16 || n == 32) return {n / 2, 2, one ? INTERLEAVED : full ? IN_LANE : n / 4};
    if (n == 12) return {4, 3, one ? INTERLEAVED : full ? 2 : 1};
  }
  return {n <= 8 ? 8 : n <= 16 ? 16 : 32, 1, one ? INTERLEAVED : ANYWHERE};
}

static long long heads_blocks(long long tokens, int heads, int G) { return (tokens * heads + 256 / G - 1) / (256 / G); }

static long long copy_blocks(long long tokens, const QkShape& q, size_t esz) {
  const long long chunks = tokens * q.kv_heads * q.head_dim * (long long)esz / 16;
  return (chunks + 256 * kCopyUnroll - 1) / (256 * kCopyUnroll);
}

// Workgroups of the gradient's two kinds: as many as the chip holds at once (four a CU;
// three with three chunks a lane, by their registers, and so for all heads of 96, as the
// scratch size does not depend on the rotation) shared out by the kinds' heads, or one for
// each 32 heads if that is fewer.
static void bwd_blocks(int tokens, int q_heads, int kv_heads, int d, int* bq, int* bk) {
  const long long all = d == 96 ? 768 : 1024;
  const long long share = std::max(1LL, all * q_heads / (q_heads + kv_heads));
  *bq = (int)std::min(heads_blocks(tokens, q_heads, 8), share);
  *bk = (int)std::min(heads_blocks(tokens, kv_heads, 8), std::max(1LL, all - share));
}

size_t qk_norm_rope_scratch_elems(int tokens, int q_heads, int kv_heads, int d) {
  int bq, bk;
  bwd_blocks(tokens, q_heads, kv_heads, d, &bq, &bk);
  return (size_t)(bq + bk) * d;
}

hipError_t launch_rope_table(int positions, int rope_dim, double theta, float* table, hipStream_t s) {
  const long long wg = ((long long)positions * (rope_dim / 2) + 255) / 256;
  if (wg > max_groups(256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)wg), dim3(256), 0, s, positions, rope_dim / 2, std::log(theta),
                     table);
  return hipGetLastError();
}

static QkArgs qk_args(const QkShape& q) {
  return QkArgs{q.tokens, q.q_heads, q.kv_heads, q.head_dim, q.rope_dim, q.table_rows, q.seq_len > 0 ? q.seq_len : 1,
                0, q.eps, q.positions, q.table};
}

struct QkCall {
  const QkShape& q;
  const void *dout, *in, *gq, *gk;  // dout: gradient only
  void* out;
  hipStream_t s;
  float *dgq, *dgk, *part;  // gradient only
  int accumulate;
};

struct Fwd {
  template <typename T, int G, int CH, int MODE>
  static hipError_t run(const QkCall& c) {
    const QkShape& q = c.q;
    QkArgs a = qk_args(q);
    // Tokens that one launch can hold; a call of more goes in several.
    constexpr long long heads = 256 / G, chunks = 256 * kCopyUnroll;  // of a workgroup
    const long long per = (long long)(q.q_heads + q.kv_heads) * chunks +
                          (c.in != c.out ? (long long)q.kv_heads * q.head_dim * sizeof(T) / 16 * heads : 0);
    const long long most = (max_groups(256) - 3) * (heads * chunks) / per;
    const size_t row = (size_t)(q.q_heads + 2 * q.kv_heads) * q.head_dim;
    for (long long t = 0; t < q.tokens; t += a.tokens) {
      a.first = (int)t;
      a.tokens = (int)std::min(most, q.tokens - t);
      a.positions = q.positions ? q.positions + t : nullptr;
      const long long bq = heads_blocks(a.tokens, q.q_heads, G), bk = heads_blocks(a.tokens, q.kv_heads, G);
      const long long bv = c.in != c.out ? copy_blocks(a.tokens, q, sizeof(T)) : 0;
      hipLaunchKernelGGL((qk_fwd_kernel<T, G, CH, MODE>), dim3((unsigned)(bq + bk + bv)), dim3(256), 0, c.s, a,
                         QkGrid{(int)bq, (int)bk, (int)bv}, (const T*)c.in + t * row, (const T*)c.gq, (const T*)c.gk,
                         (T*)c.out + t * row);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
};

struct Bwd {
  template <typename T, int G, int CH, int MODE>
  static hipError_t run(const QkCall& c) {
    const QkShape& q = c.q;
    int bq = 1, bk = 1;
    // Up to four steps of one workgroup a kind take less than the launch that would add the
    // sums of several: 8 or 20 tokens of 6 + 6 heads of 128 (2 or 4 steps) 9.4 us a call, with it
    // 12.4.  (In a replayed graph, where a launch costs less: 5.5 or 7.6, with it 7.0.)
    const bool one = heads_blocks(q.tokens, std::max(q.q_heads, q.kv_heads), G) <= 4;
    if (!one) {
      bwd_blocks(q.tokens, q.q_heads, q.kv_heads, q.head_dim, &bq, &bk);
      bq = (int)std::min<long long>(bq, heads_blocks(q.tokens, q.q_heads, G));  // with 64 heads a workgroup
      bk = (int)std::min<long long>(bk, heads_blocks(q.tokens, q.kv_heads, G));
    }
    const long long bv = c.dout != c.out ? copy_blocks(q.tokens, q, sizeof(T)) : 0;
    if (bq + bk + bv > max_groups(256)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((qk_bwd_kernel<T, G, CH, MODE>), dim3((unsigned)(bq + bk + bv)), dim3(256), 0, c.s, qk_args(q),
                       QkGrid{bq, bk, (int)bv}, (const T*)c.dout, (const T*)c.in, (const T*)c.gq, (const T*)c.gk,
                       (T*)c.out, one ? nullptr : c.part, c.dgq, c.dgk, c.accumulate);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || one) return e;
    hipLaunchKernelGGL(qk_gain_kernel, dim3(2 * ((q.head_dim + 15) / 16)), dim3(1024), 0, c.s, q.head_dim,
                       QkGrid{bq, bk, 0}, c.part, c.dgq, c.dgk, c.accumulate);
    return hipGetLastError();
  }
};

template <typename P, typename T, int G, int CH>
static hipError_t run_mode(const QkCall& c, int mode) {
  if (mode == INTERLEAVED) return P::template run<T, G, CH, INTERLEAVED>(c);
  if constexpr (CH == 1) {
    return P::template run<T, G, CH, ANYWHERE>(c);
  } else if constexpr (CH == 2) {
    if (mode == IN_LANE) return P::template run<T, G, CH, IN_LANE>(c);
    return P::template run<T, G, CH, G / 2>(c);
  } else {
    if (mode == 2) return P::template run<T, G, CH, 2>(c);
    return P::template run<T, G, CH, 1>(c);
  }
}

template <typename P, typename T>
static hipError_t run_lanes(const QkCall& c) {
  const QkLanes l = lanes_of(c.q);
  if (l.CH == 2) return l.G == 4 ? run_mode<P, T, 4, 2>(c, l.mode) : l.G == 8 ? run_mode<P, T, 8, 2>(c, l.mode)
                                                                             : run_mode<P, T, 16, 2>(c, l.mode);
  if (l.CH == 3) return run_mode<P, T, 4, 3>(c, l.mode);
  return l.G == 8 ? run_mode<P, T, 8, 1>(c, l.mode) : l.G == 16 ? run_mode<P, T, 16, 1>(c, l.mode)
                                                                : run_mode<P, T, 32, 1>(c, l.mode);
}

hipError_t launch_qk_norm_rope_fwd(int dtype, const QkShape& q, const void* in, const void* gq, const void* gk,
                                   void* out, hipStream_t s) {
  const QkCall c{q, nullptr, in, gq, gk, out, s, nullptr, nullptr, nullptr, 0};
  return dtype == DT_BF16 ? run_lanes<Fwd, bf16_t>(c) : run_lanes<Fwd, float>(c);
}

hipError_t launch_qk_norm_rope_bwd(int dtype, const QkShape& q, const void* dout, const void* in, const void* gq,
                                   const void* gk, void* dx, float* dgq, float* dgk, int accumulate, float* part,
                                   hipStream_t s) {
  const QkCall c{q, dout, in, gq, gk, dx, s, dgq, dgk, part, accumulate};
  return dtype == DT_BF16 ? run_lanes<Bwd, bf16_t>(c) : run_lanes<Bwd, float>(c);
}

}  // namespace merak
