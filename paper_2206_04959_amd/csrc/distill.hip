// Loss of a student that learns from a teacher's largest logits and from labels, and the
// gradient of the student's logits, on the whole vocabulary or one rank's share of it.
//
// A token has the student's logits z over the vocabulary, the teacher's entries (id_k, t_k),
// k < K, and a label c.  With the temperature T and the weight a:
//   p = softmax(t / T) over the entries that are there
//   loss = a T^2 sum_k p_k (log p_k - log softmax(z / T)[id_k]) - (1 - a) log softmax(z)[c]
//   dz_v = w (a T (P softmax(z / T)_v - sum_{k: id_k = v} p_k) + (1 - a) L (softmax(z)_v - [v = c])),
// w the gradient that reaches the loss; P = sum p_k is 1, or 0 without entries, L is 1, or 0
// without a label.  With m = max z, S_T = sum exp((z - m) / T) and S_1 = sum exp(z - m),
//   loss = a T^2 P log S_T + (1 - a) L log S_1 - lin,
//   lin = sum_k (a T p_k (z_k - m) - a T^2 p_k log p_k) + (1 - a) L (z_c - m).
// Everything in z is a difference from m, so a common offset of the logits costs nothing.  A
// rank has its columns' m and sums, the part of lin, P and L that its columns hold, and the
// teacher's own maximum and sum (which all ranks form from all entries): the token's row of
// statistics.  Ranks' rows join by moving to the largest m.
//
// Bound by memory: the logits are read once (maximum and sums in one pass, the sums rescaled
// when the maximum grows), the gradient is written once.  Its columns with entries or the label
// are then written once more, each by one thread that adds all that lies on it in the entries'
// order, so nothing depends on timing and each value is rounded once.  Sums are fp32.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace merak {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A launch's tokens; what it needs of the call.
struct DistillArgs {
  int tokens, vocab, ld, top;
  long long first, total;
  float alpha, tau;
  float rate_t, rate_1;          // log2(e) / T, log2(e); with one sum (TWO = false) rate_t is its rate
  bool want_t, want_1;           // sums that the loss needs
  bool id64, label64, teacher_bf16;
  const void* ids;               // [tokens][top], null without entries
  const void* teacher;
  const void* labels;            // null without labels
};

__device__ __forceinline__ long long id_at(const void* p, bool wide, size_t i) {
  return wide ? static_cast<const long long*>(p)[i] : static_cast<const int*>(p)[i];
}

// The token's own columns of the vocabulary, -1 for an id that is another rank's or none's.
__device__ __forceinline__ int column_of(const DistillArgs& a, long long id) {
  const long long c = id - a.first;
  return id >= 0 && id < a.total && c >= 0 && c < a.vocab ? (int)c : -1;
}

// The teacher's logit k of a token; -infinity for an entry that is not there.
__device__ __forceinline__ float teacher_at(const DistillArgs& a, size_t i, long long id) {
  const float t = a.teacher_bf16 ? bf2f(static_cast<const bf16_t*>(a.teacher)[i])
                                 : static_cast<const float*>(a.teacher)[i];
  return id >= 0 && id < a.total ? t : -INFINITY;
}

// A token's entries and its label (entry `top`) in LDS.
struct Entries {
  int* col;    // own column, or -1
  float* t;    // teacher's logit; then weight in the gradient
  float* z;    // student's logit at the column
};
__device__ __forceinline__ Entries entries_in(char* lds, int top) {
  const int n = (top + 4) & ~3;  // whole groups of four
  return Entries{reinterpret_cast<int*>(lds), reinterpret_cast<float*>(lds) + n, reinterpret_cast<float*>(lds) + 2 * n};
}
static size_t entries_bytes(int top) { return (size_t)((top + 4) & ~3) * 12; }

// 16 bytes of logits as floats.
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(u32x4_t r, float (&v)[8]) { unpack8(r, v); }
  static __device__ __forceinline__ u32x4_t put(const float (&v)[8]) {
    return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(u32x4_t r, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(r[e]);
  }
  static __device__ __forceinline__ u32x4_t put(const float (&v)[4]) {
    return u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};

// What a maximum's differences are formed from: 0 where nothing was above -infinity.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// By how much sums relative to the maximum m move to those relative to `base` (sums that are 0
// stay 0: the difference from a base far below 0 would have no finite exponential).
__device__ __forceinline__ float moved(float m, float base) { return m == -INFINITY ? 0.0f : m - base; }

template <int NT, int N>
__device__ __forceinline__ void block_max(float (&v)[N], float* red) {
  constexpr int W = NT / 64;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_max(v[n]);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) red[(threadIdx.x >> 6) * N + n] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    v[n] = red[n];
#pragma unroll
    for (int w = 1; w < W; ++w) v[n] = fmaxf(v[n], red[w * N + n]);
  }
}

template <int NT, int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* red) {
  constexpr int W = NT / 64;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) red[(threadIdx.x >> 6) * N + n] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    v[n] = red[n];
#pragma unroll
    for (int w = 1; w < W; ++w) v[n] += red[w * N + n];
  }
}

struct Stats {
  float m, s1, st, lin, mass, label, tm, ts;
};

__device__ __forceinline__ float loss_of(const Stats& s, float alpha, float tau) {
  float l = -s.lin;
  if (s.mass != 0.0f) l += alpha * tau * tau * s.mass * logf(s.st);
  if (s.label != 0.0f) l += (1.0f - alpha) * s.label * logf(s.s1);
  return l;
}

__device__ __forceinline__ void store_stats(float* p, const Stats& s) {
  reinterpret_cast<f32x4_t*>(p)[0] = f32x4_t{s.m, s.s1, s.st, s.lin};
  reinterpret_cast<f32x4_t*>(p)[1] = f32x4_t{s.mass, s.label, s.tm, s.ts};
}
__device__ __forceinline__ Stats load_stats(const float* p) {
  const f32x4_t a = reinterpret_cast<const f32x4_t*>(p)[0], b = reinterpret_cast<const f32x4_t*>(p)[1];
  return Stats{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// The gradient's factors of exp((z - m) / T) and exp(z - m); with one sum (TWO = false) the first
// is the factor of both.
template <bool TWO>
__device__ __forceinline__ void factors(const DistillArgs& a, const Stats& s, float w, float* ft, float* f1) {
  *ft = s.mass != 0.0f ? w * a.alpha * a.tau * s.mass / s.st : 0.0f;
  *f1 = s.label != 0.0f ? w * (1.0f - a.alpha) * s.label / s.s1 : 0.0f;
  if (!TWO) *ft += *f1;
}

template <bool TWO>
__device__ __forceinline__ float slope(const DistillArgs& a, float z, float m, float ft, float f1) {
  const float d = z - m;
  float g = ft * exp2_fast(d * a.rate_t);
  if (TWO) g += f1 * exp2_fast(d * a.rate_1);
  return g;
}

// Columns [lo, hi) of a row: dz from z (the same memory, or another row's).
template <typename T, int NT, bool TWO>
__device__ __forceinline__ void write_slopes(const DistillArgs& a, const T* z, T* dz, int lo, int hi, float m, float ft,
                                             float f1) {
  constexpr int N = Vec<T>::N;
  for (int c = lo + (int)threadIdx.x * N; c < hi; c += NT * N) {
    float v[N];
    Vec<T>::get(*reinterpret_cast<const u32x4_t*>(z + c), v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = c + e < a.vocab ? slope<TWO>(a, v[e], m, ft, f1) : 0.0f;
    *reinterpret_cast<u32x4_t*>(dz + c) = Vec<T>::put(v);
  }
}

template <typename T, int NT>
__device__ __forceinline__ void write_zeros(T* dz, int lo, int hi) {
  for (int c = lo + (int)threadIdx.x * Vec<T>::N; c < hi; c += NT * Vec<T>::N)
    *reinterpret_cast<u32x4_t*>(dz + c) = u32x4_t{0, 0, 0, 0};
}

// The columns that have entries: each is written by its first entry's thread.
template <typename T, int NT, bool TWO>
__device__ __forceinline__ void write_entries(const DistillArgs& a, const Entries& en, T* dz, float m, float ft,
                                              float f1) {
  for (int e = threadIdx.x; e <= a.top; e += NT) {
    const int c = en.col[e];
    if (c < 0) continue;
    float total = 0.0f;
    bool first = true;
    for (int k = 0; k <= a.top; ++k)
      if (en.col[k] == c) {
        first = first && k >= e;
        total += en.t[k];
      }
    if (first) dz[c] = Elem<T>::from_f(slope<TWO>(a, en.z[e], m, ft, f1) - total);
  }
}

// One workgroup a token: statistics, loss and, with GRAD, the gradient (a second look at the
// row).
template <typename T, int NT, bool TWO, bool GRAD>
__global__ void __launch_bounds__(NT) distill_kernel(DistillArgs a, const T* z, float* __restrict__ stats,
                                                     float* __restrict__ loss, const float* __restrict__ dloss, T* dz) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2][NT / 64 * 6];
  const Entries en = entries_in(smem, a.top);
  const size_t row = blockIdx.x;
  const T* zr = z + row * a.ld;

  // entries and label
  float mx[2] = {-INFINITY, -INFINITY};  // of the student's logits, of the teacher's
  for (int k = threadIdx.x; k < a.top; k += NT) {
    const size_t i = row * a.top + k;
    const long long id = id_at(a.ids, a.id64, i);
    const int c = column_of(a, id);
    const float t = teacher_at(a, i, id);
    en.col[k] = c;
    en.t[k] = t;
    en.z[k] = c >= 0 ? Elem<T>::to_f(zr[c]) : 0.0f;
    mx[1] = fmaxf(mx[1], t != t ? INFINITY : t);  // NaN: no probabilities
  }
  const long long label = a.labels ? id_at(a.labels, a.label64, row) : -1;
  const bool labelled = label >= 0 && label < a.total;
  if (threadIdx.x == 0) {
    const int c = column_of(a, label);
    en.col[a.top] = c;
    en.z[a.top] = c >= 0 ? Elem<T>::to_f(zr[c]) : 0.0f;
  }

  // maximum and sums of the logits
  constexpr int N = Vec<T>::N;
  float st = 0.0f, s1 = 0.0f;
  for (int c = (int)threadIdx.x * N; c < a.vocab; c += NT * N) {
    float v[N];
    Vec<T>::get(*reinterpret_cast<const u32x4_t*>(zr + c), v);
    float m = mx[0];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (c + e >= a.vocab) v[e] = -INFINITY;
      m = fmaxf(m, v[e]);
    }
    const float base = base_of(m), old = moved(mx[0], base);
    st *= exp2_fast(old * a.rate_t);
    if (TWO) s1 *= exp2_fast(old * a.rate_1);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      st += exp2_fast((v[e] - base) * a.rate_t);
      if (TWO) s1 += exp2_fast((v[e] - base) * a.rate_1);
    }
    mx[0] = m;
  }
  const float own = mx[0];
  block_max<NT>(mx, red[0]);
  const float base = base_of(mx[0]), tm = base_of(mx[1]);
  // S_T, S_1, teacher's sum, mass here, sum p (z - m), sum p t
  const float d0 = moved(own, base);
  float s[6] = {st * exp2_fast(d0 * a.rate_t), TWO ? s1 * exp2_fast(d0 * a.rate_1) : 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = threadIdx.x; k < a.top; k += NT) {
    const float d = en.t[k] - tm, p = exp2_fast(d * a.rate_t);
    en.t[k] = p;
    if (p == 0.0f) {
      en.col[k] = -1;
      continue;
    }
    s[2] += p;
    if (en.col[k] >= 0) {
      s[3] += p;
      s[4] += p * (en.z[k] - base);
      s[5] += p * d;
    }
  }
  block_sum<NT>(s, red[1]);
  Stats r;
  r.m = mx[0];
  r.st = a.want_t ? s[0] : 0.0f;
  r.s1 = a.want_1 ? (TWO ? s[1] : s[0]) : 0.0f;
  r.tm = tm;
  r.ts = s[2];
  const int lc = en.col[a.top];
  const float inv = s[2] != 0.0f ? 1.0f / s[2] : 0.0f;
  r.mass = s[3] * inv;
  r.label = labelled && lc >= 0 ? 1.0f : 0.0f;
  r.lin = 0.0f;
  if (s[2] != 0.0f)
    r.lin = a.alpha * a.tau * inv * s[4] - a.alpha * a.tau * (inv * s[5] - a.tau * r.mass * logf(s[2]));
  if (r.label != 0.0f) r.lin += (1.0f - a.alpha) * (en.z[a.top] - base);
  const bool idle = s[2] == 0.0f && !labelled;  // nothing to learn here
  if (threadIdx.x == 0) {
    if (stats) store_stats(stats + row * kDistillStats, r);
    if (loss) loss[row] = idle ? 0.0f : loss_of(r, a.alpha, a.tau);
  }
  if constexpr (GRAD) {
    T* dr = dz + row * a.ld;
    const float w = dloss[row];
    if (idle || w == 0.0f) {
      write_zeros<T, NT>(dr, 0, a.ld);
      return;
    }
    float ft, f1;
    factors<TWO>(a, r, w, &ft, &f1);
    for (int k = threadIdx.x; k <= a.top; k += NT)
      en.t[k] = k < a.top ? w * a.alpha * a.tau * inv * en.t[k] : w * (1.0f - a.alpha);
    write_slopes<T, NT, TWO>(a, zr, dr, 0, a.ld, base, ft, f1);
    __syncthreads();
    write_entries<T, NT, TWO>(a, en, dr, base, ft, f1);
  }
}

// The gradient from a token's (joined) statistics: a workgroup a piece of `piece` columns of a
// row.
template <typename T, int NT, bool TWO>
__global__ void __launch_bounds__(NT) distill_bwd_kernel(DistillArgs a, int pieces, int piece, const T* z,
                                                         const float* __restrict__ stats,
                                                         const float* __restrict__ dloss, T* dz) {
  extern __shared__ __align__(16) char smem[];
  const Entries en = entries_in(smem, a.top);
  const size_t row = blockIdx.x / pieces;
  const int lo = (int)(blockIdx.x % pieces) * piece, hi = min(lo + piece, a.ld);
  const T* zr = z + row * a.ld;
  T* dr = dz + row * a.ld;
  const Stats s = load_stats(stats + row * kDistillStats);
  const float w = dloss[row];
  if ((s.mass == 0.0f && s.label == 0.0f) || w == 0.0f) {
    write_zeros<T, NT>(dr, lo, hi);
    return;
  }
  const float base = base_of(s.m);
  const float inv = s.ts != 0.0f ? w * a.alpha * a.tau / s.ts : 0.0f;
  for (int k = threadIdx.x; k <= a.top; k += NT) {
    int c;
    float t;
    if (k < a.top) {
      const size_t i = row * a.top + k;
      const long long id = id_at(a.ids, a.id64, i);
      c = column_of(a, id);
      const float p = exp2_fast((teacher_at(a, i, id) - s.tm) * a.rate_t);
      t = inv * p;
      if (p == 0.0f) c = -1;
    } else {
      c = a.labels ? column_of(a, id_at(a.labels, a.label64, row)) : -1;
      t = w * (1.0f - a.alpha);
    }
    if (c < lo || c >= hi) c = -1;
    en.col[k] = c;
    en.t[k] = t;
    en.z[k] = c >= 0 ? Elem<T>::to_f(zr[c]) : 0.0f;
  }
  __syncthreads();
  float ft, f1;
  factors<TWO>(a, s, w, &ft, &f1);
  write_slopes<T, NT, TWO>(a, zr, dr, lo, hi, base, ft, f1);
  __syncthreads();
  write_entries<T, NT, TWO>(a, en, dr, base, ft, f1);
}

// Ranks' statistics [ranks][tokens] to the whole vocabulary's, in the ranks' order.
__global__ void __launch_bounds__(256) distill_join_kernel(int tokens, int ranks, float alpha, float tau, float rate_t,
                                                           const float* __restrict__ parts, float* __restrict__ stats,
                                                           float* __restrict__ loss) {
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (t >= tokens) return;
  float m = -INFINITY;
  for (int r = 0; r < ranks; ++r) m = fmaxf(m, parts[((size_t)r * tokens + t) * kDistillStats]);
  const float base = base_of(m);
  Stats s{m, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int r = 0; r < ranks; ++r) {
    const Stats p = load_stats(parts + ((size_t)r * tokens + t) * kDistillStats);
    const float d = moved(p.m, base);
    s.s1 += p.s1 * exp2_fast(d * kLog2e);
    s.st += p.st * exp2_fast(d * rate_t);
    s.lin += p.lin;
    if (p.mass != 0.0f) s.lin += alpha * tau * p.mass * d;
    if (p.label != 0.0f) s.lin += (1.0f - alpha) * p.label * d;
    s.mass += p.mass;
    s.label += p.label;
    s.tm = p.tm;
    s.ts = p.ts;
  }
  store_stats(stats + t * kDistillStats, s);
  loss[t] = loss_of(s, alpha, tau);
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
static DistillArgs distill_args(const DistillShape& q) {
  DistillArgs a{};
  a.vocab = q.vocab, a.ld = q.ld;
  a.first = q.first, a.total = q.total;
  a.alpha = q.alpha, a.tau = q.tau;
  a.want_t = q.top > 0 && q.alpha > 0.0f;
  a.want_1 = q.labels && q.alpha < 1.0f;
  a.top = a.want_t ? q.top : 0;
  a.rate_1 = kLog2e;
  a.rate_t = a.want_t ? kLog2e / q.tau : kLog2e;
  a.id64 = q.id_type == ID_I64, a.label64 = q.label_type == ID_I64, a.teacher_bf16 = q.teacher_type == DT_BF16;
  a.ids = q.ids, a.teacher = q.teacher, a.labels = a.want_1 ? q.labels : nullptr;
  return a;
}

// Moves a launch's arguments to the tokens [t, t + n).
static DistillArgs at_tokens(const DistillShape& q, DistillArgs a, long long t, int n) {
  a.tokens = n;
  if (a.top) {
    a.ids = (const char*)a.ids + (size_t)t * a.top * (a.id64 ? 8 : 4);
    a.teacher = (const char*)a.teacher + (size_t)t * a.top * (a.teacher_bf16 ? 2 : 4);
  }
  if (a.labels) a.labels = (const char*)a.labels + (size_t)t * (a.label64 ? 8 : 4);
  return a;
}

template <typename T, int NT, bool TWO, bool GRAD>
static hipError_t run_rows(const DistillShape& q, const void* z, float* stats, float* loss, const float* dloss, void* dz,
                           hipStream_t s) {
  const DistillArgs all = distill_args(q);
  const long long most = max_groups(NT);
  for (long long t = 0; t < q.tokens; t += most) {
    const int n = (int)std::min(most, q.tokens - t);
    const DistillArgs a = at_tokens(q, all, t, n);
    hipLaunchKernelGGL((distill_kernel<T, NT, TWO, GRAD>), dim3(n), dim3(NT), entries_bytes(a.top), s, a,
                       (const T*)z + t * q.ld, stats ? stats + t * kDistillStats : nullptr, loss ? loss + t : nullptr,
                       dloss ? dloss + t : nullptr, dz ? (T*)dz + t * q.ld : nullptr);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

static bool two_sums(const DistillShape& q) {
  const DistillArgs a = distill_args(q);
  return a.want_t && a.want_1 && q.tau != 1.0f;
}

template <typename T>
static hipError_t run_forward(const DistillShape& q, const void* z, float* stats, float* loss, const float* dloss,
                              void* dz, hipStream_t s) {
  if (two_sums(q)) return dz ? run_rows<T, 256, true, true>(q, z, stats, loss, dloss, dz, s)
                             : run_rows<T, 256, true, false>(q, z, stats, loss, dloss, dz, s);
  return dz ? run_rows<T, 256, false, true>(q, z, stats, loss, dloss, dz, s)
            : run_rows<T, 256, false, false>(q, z, stats, loss, dloss, dz, s);
}

hipError_t launch_distill(int dtype, const DistillShape& q, const void* z, float* stats, float* loss,
                          const float* dloss, void* dz, hipStream_t s) {
  return dtype == DT_BF16 ? run_forward<bf16_t>(q, z, stats, loss, dloss, dz, s)
                          : run_forward<float>(q, z, stats, loss, dloss, dz, s);
}

hipError_t launch_distill_join(int tokens, int ranks, float alpha, float tau, const float* parts, float* stats,
                               float* loss, hipStream_t s) {
  hipLaunchKernelGGL(distill_join_kernel, dim3((unsigned)(((long long)tokens + 255) / 256)), dim3(256), 0, s, tokens,
                     ranks, alpha, tau, kLog2e / tau, parts, stats, loss);
  return hipGetLastError();
}

template <typename T, bool TWO>
static hipError_t run_backward(const DistillShape& q, const void* z, const float* stats, const float* dloss, void* dz,
                               hipStream_t s) {
  constexpr int NT = 256, piece = NT * Vec<T>::N * 4;
  const DistillArgs all = distill_args(q);
  const int pieces = (q.ld + piece - 1) / piece;
  const long long most = max_groups(NT) / pieces;
  for (long long t = 0; t < q.tokens; t += most) {
    const int n = (int)std::min(most, q.tokens - t);
    const DistillArgs a = at_tokens(q, all, t, n);
    hipLaunchKernelGGL((distill_bwd_kernel<T, NT, TWO>), dim3((unsigned)(n * pieces)), dim3(NT), entries_bytes(a.top), s,
                       a, pieces, piece, (const T*)z + t * q.ld, stats + t * kDistillStats, dloss + t,
                       (T*)dz + t * q.ld);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_distill_bwd(int dtype, const DistillShape& q, const void* z, const float* stats, const float* dloss,
                              void* dz, hipStream_t s) {
  if (dtype == DT_BF16)
    return two_sums(q) ? run_backward<bf16_t, true>(q, z, stats, dloss, dz, s)
                       : run_backward<bf16_t, false>(q, z, stats, dloss, dz, s);
  return two_sums(q) ? run_backward<float, true>(q, z, stats, dloss, dz, s)
                     : run_backward<float, false>(q, z, stats, dloss, dz, s);
}

}  // namespace merak
