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
// Bound by memory.  A group of 8, 16 or 32 lanes owns a head, 8 features a lane,
// so a wave moves 8, 4 or 2 neighbouring heads at a time; the two halves of a pair
// meet by a lane exchange.
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
  int seq_len;      // without positions: token t is at t % seq_len
  float eps;
  const int* positions;
  const float* table;
};

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int off = G / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Rotation of the 8 features of chunk c by the token's angles, forward (dir = 1)
// or back (dir = -1).  `base` is the group's first lane.  A position outside the
// table rotates by NaN.
template <bool INTER>
__device__ __forceinline__ void rotate8(const QkArgs& a, int pos, int c, int base, float dir, float z[8]) {
  const int pc = a.rope >> 4;  // chunks of half the rotated features
  const bool in = pos >= 0 && pos < a.table_rows;
  const bool rot = c < 2 * pc;
  if constexpr (INTER) {
    if (!rot) return;
    const float* cs = a.table + ((size_t)(in ? pos : 0) * (a.rope >> 1) + c * 4) * 2;
    float t[8];
    load8(cs, t);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float co = in ? t[2 * e] : NAN, si = (in ? t[2 * e + 1] : NAN) * dir;
      const float x = z[2 * e], y = z[2 * e + 1];
      z[2 * e] = x * co - y * si;
      z[2 * e + 1] = y * co + x * si;
    }
  } else {
    const bool low = c < pc;
    const int other = rot ? base + (low ? c + pc : c - pc) : base;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = __shfl(z[e], other, 64);
    if (!rot) return;
    const float* cs = a.table + ((size_t)(in ? pos : 0) * (a.rope >> 1) + (low ? c : c - pc) * 8) * 2;
    float t[16];
    load8(cs, t);
    load8(cs + 8, t + 8);
    const float sign = low ? -dir : dir;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float co = in ? t[2 * e] : NAN, si = (in ? t[2 * e + 1] : NAN) * sign;
      z[e] = z[e] * co + p[e] * si;
    }
  }
}

__device__ __forceinline__ int position_of(const QkArgs& a, int t) {
  return a.positions ? a.positions[t] : t % a.seq_len;
}

// One head per group of G lanes and step.  `copy`: also move the value heads
// (out is not in).
template <typename T, int G, bool INTER>
__global__ void __launch_bounds__(256) qk_fwd_kernel(QkArgs a, int copy, const T* in, const T* __restrict__ gq,
                                                     const T* __restrict__ gk, T* out) {
  const int lane = threadIdx.x & 63, j = lane & (G - 1), base = lane - j;
  const int row_heads = a.q_heads + 2 * a.kv_heads, qk = a.q_heads + a.kv_heads;
  const int heads = copy ? row_heads : qk;
  const long long slot = ((long long)blockIdx.x * 256 + threadIdx.x) / G;
  const long long t = slot / heads;
  if (t >= a.tokens) return;  // whole groups leave: the exchanges below stay within a group
  const int h = (int)(slot - t * heads);
  const bool live = j * 8 < a.d;
  const size_t at = ((size_t)t * row_heads + h) * a.d + j * 8;
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 0.0f;
  if (live) load8(in + at, x);
  if (h >= qk) {
    if (live) store8(out + at, x);
    return;
  }
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += x[e] * x[e];
  const float rstd = 1.0f / sqrtf(group_sum<G>(s) / (float)a.d + a.eps);
  float g[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = 0.0f;
  if (live) load8((h < a.q_heads ? gq : gk) + j * 8, g);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * g[e];
  if (a.rope) rotate8<INTER>(a, position_of(a, (int)t), j, base, 1.0f, x);
  if (live) store8(out + at, x);
}

// Gradient: workgroups step through the heads, each lane keeping the sums of its
// 8 gain columns for queries and for keys; the workgroup's sums go to
// part[query or key][workgroup][d], and launch_reduce_partials adds those in order.
template <typename T, int G, bool INTER>
__global__ void __launch_bounds__(256) qk_bwd_kernel(QkArgs a, int copy, const T* dout, const T* __restrict__ in,
                                                     const T* __restrict__ gq, const T* __restrict__ gk, T* dx,
                                                     float* __restrict__ part) {
  __shared__ float red[2][4][G * 8];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, j = lane & (G - 1), base = lane - j;
  const int row_heads = a.q_heads + 2 * a.kv_heads, qk = a.q_heads + a.kv_heads;
  const int heads = copy ? row_heads : qk;
  const bool live = j * 8 < a.d;
  const long long slots = (long long)a.tokens * heads, stride = (long long)gridDim.x * (256 / G);
  float sq[8], sk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sq[e] = sk[e] = 0.0f;
  for (long long slot = ((long long)blockIdx.x * 256 + threadIdx.x) / G; slot < slots; slot += stride) {
    const long long t = slot / heads;
    const int h = (int)(slot - t * heads);
    const size_t at = ((size_t)t * row_heads + h) * a.d + j * 8;
    float dz[8], x[8], g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dz[e] = x[e] = g[e] = 0.0f;
    if (live) load8(dout + at, dz);
    if (h >= qk) {
      if (live) store8(dx + at, dz);
      continue;
    }
    if (live) {
      load8(in + at, x);
      load8((h < a.q_heads ? gq : gk) + j * 8, g);
    }
    if (a.rope) rotate8<INTER>(a, position_of(a, (int)t), j, base, -1.0f, dz);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[e] * x[e];
    const float rstd = 1.0f / sqrtf(group_sum<G>(s) / (float)a.d + a.eps);
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] *= rstd;
      const float c = dz[e] * x[e];
      if (h < a.q_heads) sq[e] += c;
      else sk[e] += c;
      dz[e] *= g[e];
      m += dz[e] * x[e];
    }
    m = group_sum<G>(m) / (float)a.d;
#pragma unroll
    for (int e = 0; e < 8; ++e) dz[e] = rstd * (dz[e] - x[e] * m);
    if (live) store8(dx + at, dz);
  }
  // the wave's groups, then the four waves in order
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int off = G; off < 64; off <<= 1) {
      sq[e] += __shfl_xor(sq[e], off, 64);
      sk[e] += __shfl_xor(sk[e], off, 64);
    }
    if (lane < G) {
      red[0][w][j * 8 + e] = sq[e];
      red[1][w][j * 8 + e] = sk[e];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
    const int which = i >= a.d, c = i - which * a.d;
    const float v = red[which][0][c] + red[which][1][c] + red[which][2][c] + red[which][3][c];
    part[((size_t)which * gridDim.x + blockIdx.x) * a.d + c] = v;
  }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
constexpr int kBwdBlocks = 1024;

static inline int group_lanes(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Workgroups of the gradient: the same for a size whether the values are copied or not.
static inline int bwd_blocks(int tokens, int q_heads, int kv_heads, int d) {
  const long long per = 256 / group_lanes(d);
  const long long need = ((long long)tokens * (q_heads + kv_heads) + per - 1) / per;
  return (int)std::min<long long>(need, kBwdBlocks);
}

size_t qk_norm_rope_scratch_elems(int tokens, int q_heads, int kv_heads, int d) {
  return (size_t)2 * bwd_blocks(tokens, q_heads, kv_heads, d) * d;
}

hipError_t launch_rope_table(int positions, int rope_dim, double theta, float* table, hipStream_t s) {
  const long long wg = ((long long)positions * (rope_dim / 2) + 255) / 256;
  if (wg > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)wg), dim3(256), 0, s, positions, rope_dim / 2, std::log(theta),
                     table);
  return hipGetLastError();
}

static QkArgs qk_args(const QkShape& q) {
  return QkArgs{q.tokens, q.q_heads, q.kv_heads, q.head_dim, q.rope_dim, q.table_rows, q.seq_len > 0 ? q.seq_len : 1,
                q.eps, q.positions, q.table};
}

template <typename T, int G>
static hipError_t fwd_t(const QkShape& q, const void* in, const void* gq, const void* gk, void* out, hipStream_t s) {
  const int copy = in != out;
  const int heads = q.q_heads + q.kv_heads + (copy ? q.kv_heads : 0);
  const long long wg = ((long long)q.tokens * heads * G + 255) / 256;
  if (wg > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wg);
  if (q.interleaved)
    hipLaunchKernelGGL((qk_fwd_kernel<T, G, true>), grid, dim3(256), 0, s, qk_args(q), copy, (const T*)in,
                       (const T*)gq, (const T*)gk, (T*)out);
  else
    hipLaunchKernelGGL((qk_fwd_kernel<T, G, false>), grid, dim3(256), 0, s, qk_args(q), copy, (const T*)in,
                       (const T*)gq, (const T*)gk, (T*)out);
  return hipGetLastError();
}

template <typename T>
static hipError_t fwd_dispatch(const QkShape& q, const void* in, const void* gq, const void* gk, void* out,
                               hipStream_t s) {
  switch (group_lanes(q.head_dim)) {
    case 8: return fwd_t<T, 8>(q, in, gq, gk, out, s);
    case 16: return fwd_t<T, 16>(q, in, gq, gk, out, s);
    default: return fwd_t<T, 32>(q, in, gq, gk, out, s);
  }
}

hipError_t launch_qk_norm_rope_fwd(int dtype, const QkShape& q, const void* in, const void* gq, const void* gk,
                                   void* out, hipStream_t s) {
  return dtype == DT_BF16 ? fwd_dispatch<bf16_t>(q, in, gq, gk, out, s) : fwd_dispatch<float>(q, in, gq, gk, out, s);
}

template <typename T, int G>
static hipError_t bwd_t(const QkShape& q, const void* dout, const void* in, const void* gq, const void* gk, void* dx,
                        float* part, hipStream_t s) {
  const int copy = dout != dx;
  const dim3 grid(bwd_blocks(q.tokens, q.q_heads, q.kv_heads, q.head_dim));
  if (q.interleaved)
    hipLaunchKernelGGL((qk_bwd_kernel<T, G, true>), grid, dim3(256), 0, s, qk_args(q), copy, (const T*)dout,
                       (const T*)in, (const T*)gq, (const T*)gk, (T*)dx, part);
  else
    hipLaunchKernelGGL((qk_bwd_kernel<T, G, false>), grid, dim3(256), 0, s, qk_args(q), copy, (const T*)dout,
                       (const T*)in, (const T*)gq, (const T*)gk, (T*)dx, part);
  return hipGetLastError();
}

template <typename T>
static hipError_t bwd_dispatch(const QkShape& q, const void* dout, const void* in, const void* gq, const void* gk,
                               void* dx, float* part, hipStream_t s) {
  switch (group_lanes(q.head_dim)) {
    case 8: return bwd_t<T, 8>(q, dout, in, gq, gk, dx, part, s);
    case 16: return bwd_t<T, 16>(q, dout, in, gq, gk, dx, part, s);
    default: return bwd_t<T, 32>(q, dout, in, gq, gk, dx, part, s);
  }
}

hipError_t launch_qk_norm_rope_bwd(int dtype, const QkShape& q, const void* dout, const void* in, const void* gq,
                                   const void* gk, void* dx, float* dgq, float* dgk, int accumulate, float* part,
                                   hipStream_t s) {
  hipError_t e = dtype == DT_BF16 ? bwd_dispatch<bf16_t>(q, dout, in, gq, gk, dx, part, s)
                                  : bwd_dispatch<float>(q, dout, in, gq, gk, dx, part, s);
  if (e != hipSuccess) return e;
  const int n = bwd_blocks(q.tokens, q.q_heads, q.kv_heads, q.head_dim);
  const ReduceJob jobs[2] = {{n, q.head_dim, part, dgq, accumulate},
                             {n, q.head_dim, part + (size_t)n * q.head_dim, dgk, accumulate}};
  return launch_reduce_partials_batch(jobs, 2, s);
}

}  // namespace merak
