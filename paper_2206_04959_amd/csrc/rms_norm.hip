// The residual's addition with the root-mean-square norm of the sum, its output in the
// type, in 8 bits or in both, and its gradient.
//
//   h = x + r, rounded to the type (what the next layers read); without r, h = x
//   n = h * rstd,  rstd = 1 / sqrt(mean(h^2) + eps),  y = n * g
// y in 8 bits (act8.hip says how) is taken from the unrounded y: rounded once.
// Backward, with ds the gradient that reaches h from elsewhere (the residual's way):
//   dg = sum over rows of dy * n,
//   dh = ds + rstd * (dy g - n * mean(dy g n)),
// the gradient of x and of r alike.  rstd is rebuilt from h, whose square sum comes with the
// sum that the gradient needs anyway, so nothing but h is kept.  Statistics and sums are
// fp32, outputs are rounded once.
//
// Bound by memory.  A row stays in the registers of its NT threads, CH chunks of 8 features
// each: chunk i of thread j holds the features from (j + NT i) * 8 on.
#include <algorithm>

#include "act8_codes.h"
#include "common.h"
#include "kernels.h"
#include "wave.h"

namespace merak {

constexpr int threads_of(int nt) { return nt < 256 ? 256 : nt; }  // of a workgroup: four rows of 64 threads, or one

// v rounded to T (what a store would keep).
template <typename T>
__device__ __forceinline__ void round8(float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = Elem<T>::to_f(Elem<T>::from_f(v[e]));
}

struct NormFwd {
  int rows, cols;
  float eps;
};

// sum may be x or r.
template <typename T, int NT, int CH, bool Q8>
__global__ void __launch_bounds__(threads_of(NT)) rms_fwd_kernel(NormFwd a, const T* x, const T* r,
                                                                 const T* __restrict__ g, T* sum,
                                                                 T* __restrict__ y, uint8_t* __restrict__ q,
                                                                 uint8_t* __restrict__ scales) {
  __shared__ float red[NT > 64 ? NT / 64 : 1];
  constexpr int R = threads_of(NT) / NT;
  const int j = threadIdx.x % NT;
  const int row = blockIdx.x * R + threadIdx.x / NT;
  if (row >= a.rows) return;  // whole waves (NT = 64), else none
  const size_t at = (size_t)row * a.cols;
  float h[CH][8];
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (j + NT * i) * 8;
    if (c < a.cols) {
      load8(x + at + c, h[i]);
      if (r) {
        float v[8];
        load8(r + at + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] += v[e];
        round8<T>(h[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += h[i][e] * h[i][e];
    }
  }
  block_reduce<AddOp, NT>(s, red);
  const float rstd = 1.0f / sqrtf(s[0] / (float)a.cols + a.eps);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (j + NT * i) * 8;
    if (c >= a.cols) continue;
    if (sum) store8(sum + at + c, h[i]);
    float w[8], o[8];
    load8(g + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = h[i][e] * rstd * w[e];
    if (y) store8(y + at + c, o);
    if constexpr (Q8) {
      // a block of 32 features lies on four neighbouring lanes, all in the row or none
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, finite_mag(o[e]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 1, 64));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2, 64));
      const int b = scale_byte(m);
      const float inv = __uint_as_float((uint32_t)(254 - b) << 23);
      *reinterpret_cast<u32x2_t*>(q + at + c) = u32x2_t{encode4(o, inv), encode4(o + 4, inv)};
      if ((j & 3) == 0) scales[(at + c) / kScaleBlock] = (uint8_t)b;
    }
  }
}

// The workgroups step through the rows; each thread keeps its columns' sums of dy * n, and a
// workgroup's go to part[workgroup][cols].  dx may be dy or ds.
template <typename T, int NT, int CH>
__global__ void __launch_bounds__(threads_of(NT)) rms_bwd_kernel(int rows, int cols, float eps, const T* dy,
                                                                 const T* ds, const T* __restrict__ h,
                                                                 const T* __restrict__ g, T* dx,
                                                                 float* __restrict__ part) {
  constexpr int R = threads_of(NT) / NT;
  __shared__ float red[NT > 64 ? 2 * 2 * (NT / 64) : R * CH * 512];
  const int j = threadIdx.x % NT;
  float sum[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[i][e] = 0.0f;
  int buf = 0;
  for (long long row = (long long)blockIdx.x * R + threadIdx.x / NT; row < rows; row += (long long)gridDim.x * R) {
    const size_t at = (size_t)row * cols;
    float d[CH][8], v[CH][8];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      load8(dy + at + c, d[i]);
      load8(h + at + c, v[i]);
      float w[8];
      load8(g + c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[0] += v[i][e] * v[i][e];
        s[1] += d[i][e] * w[e] * v[i][e];
      }
    }
    block_reduce<AddOp, NT>(s, red + buf);
    buf ^= 2 * (NT / 64);  // two areas in turn: one barrier a row is enough
    const float rstd = 1.0f / sqrtf(s[0] / (float)cols + eps);
    const float m = s[1] * rstd / (float)cols;  // mean(dy g n)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      float w[8], o[8];
      load8(g + c, w);
      if (ds) {
        load8(ds + at + c, o);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = v[i][e] * rstd;
        sum[i][e] += d[i][e] * n;
        o[e] += rstd * (d[i][e] * w[e] - n * m);
      }
      store8(dx + at + c, o);
    }
  }
  if constexpr (NT > 64) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c < cols) store8(part + (size_t)blockIdx.x * cols + c, sum[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) red[(threadIdx.x / NT) * CH * 512 + (j + NT * i) * 8 + e] = sum[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 256)
      part[(size_t)blockIdx.x * cols + c] =
          (red[c] + red[CH * 512 + c]) + (red[2 * CH * 512 + c] + red[3 * CH * 512 + c]);
  }
}

// The gain's gradient from the workgroups' sums, 16 columns a workgroup: 64 threads a column
// take every 64th sum, and are added as a tree.
__global__ void __launch_bounds__(1024) rms_gain_kernel(int cols, int n, const float* __restrict__ part,
                                                        float* __restrict__ dg, int accumulate) {
  __shared__ float red[64][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
  float s = 0.0f;
  if (col < cols) {
    constexpr int U = 16;
    for (int i = slice; i < n; i += 64 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = i + 64 * u < n ? part[(size_t)(i + 64 * u) * cols + col] : 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
  }
  red[slice][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x < 16 && col < cols) {
    float v[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = red[i][threadIdx.x];
#pragma unroll
    for (int k = 32; k > 0; k >>= 1)
#pragma unroll
      for (int i = 0; i < k; ++i) v[i] += v[i + k];
    dg[col] = accumulate ? dg[col] + v[0] : v[0];
  }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
struct NormCall {
  int rows, cols;
  float eps;
  hipStream_t s;
  // forward
  const void *x, *r, *g;
  void *sum, *y;
  uint8_t *q, *scales;
  // backward
  const void *dy, *ds, *h;
  void* dx;
  float *dg, *part;
  int accumulate;
};

struct NormForward {
  template <typename T, int NT, int CH>
  static hipError_t run(const NormCall& c) {
    constexpr int threads = threads_of(NT), R = threads / NT;
    const long long most = max_groups(threads) * R;  // rows of a launch; a call of more goes in several
    for (long long at = 0; at < c.rows; at += most) {
      const NormFwd a{(int)std::min(most, c.rows - at), c.cols, c.eps};
      const dim3 grid((unsigned)((a.rows + R - 1) / R));
      const size_t off = (size_t)at * c.cols;
      auto past = [off](const void* p) { return p ? (T*)p + off : nullptr; };
      if (c.q)
        hipLaunchKernelGGL((rms_fwd_kernel<T, NT, CH, true>), grid, dim3(threads), 0, c.s, a, past(c.x), past(c.r),
                           (const T*)c.g, past(c.sum), past(c.y), c.q + off, c.scales + off / kScaleBlock);
      else
        hipLaunchKernelGGL((rms_fwd_kernel<T, NT, CH, false>), grid, dim3(threads), 0, c.s, a, past(c.x), past(c.r),
                           (const T*)c.g, past(c.sum), past(c.y), nullptr, nullptr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
};

// Workgroups of the gradient, from the threads of a row.
static int bwd_groups(int rows, int nt) {
  const int per = threads_of(nt) / nt;
  return std::min((rows + per - 1) / per, 1024 * 256 / threads_of(nt));
}

struct NormBackward {
  template <typename T, int NT, int CH>
  static hipError_t run(const NormCall& c) {
    const int wg = bwd_groups(c.rows, NT);
    hipLaunchKernelGGL((rms_bwd_kernel<T, NT, CH>), dim3(wg), dim3(threads_of(NT)), 0, c.s, c.rows, c.cols, c.eps,
                       (const T*)c.dy, (const T*)c.ds, (const T*)c.h, (const T*)c.g, (T*)c.dx, c.part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(rms_gain_kernel, dim3((c.cols + 15) / 16), dim3(1024), 0, c.s, c.cols, wg, c.part, c.dg,
                       c.accumulate);
    return hipGetLastError();
  }
};

template <typename T>
static hipError_t forward_lanes(const NormCall& c) {
  const int n = (c.cols + 511) / 512;
  if (n <= 1) return NormForward::run<T, 64, 1>(c);
  if (n <= 2) return NormForward::run<T, 64, 2>(c);
  if (n <= 3) return NormForward::run<T, 64, 3>(c);
  if (n <= 4) return NormForward::run<T, 64, 4>(c);
  if (n <= 8) return NormForward::run<T, 256, 2>(c);
  if (n <= 12) return NormForward::run<T, 256, 3>(c);
  if (n <= 16) return NormForward::run<T, 256, 4>(c);
  if (n <= 32) return NormForward::run<T, 1024, 2>(c);
  return NormForward::run<T, 1024, 4>(c);
}

static int bwd_threads(int cols) { return cols <= 1024 ? 64 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024; }

template <typename T>
static hipError_t backward_lanes(const NormCall& c) {
  const int n = (c.cols + 511) / 512;
  if (n <= 1) return NormBackward::run<T, 64, 1>(c);
  if (n <= 2) return NormBackward::run<T, 64, 2>(c);
  if (n <= 4) return NormBackward::run<T, 256, 1>(c);
  if (n <= 8) return NormBackward::run<T, 256, 2>(c);
  if (n <= 16) return NormBackward::run<T, 512, 2>(c);
  if (n <= 32) return NormBackward::run<T, 1024, 2>(c);
  return NormBackward::run<T, 1024, 4>(c);
}

hipError_t launch_add_rms_norm_fwd(int dtype, int rows, int cols, float eps, const void* x, const void* r,
                                   const void* g, void* sum, void* y, uint8_t* q, uint8_t* scales, hipStream_t s) {
  NormCall c{};
  c.rows = rows, c.cols = cols, c.eps = eps, c.s = s;
  c.x = x, c.r = r, c.g = g, c.sum = sum, c.y = y, c.q = q, c.scales = scales;
  return dtype == DT_BF16 ? forward_lanes<bf16_t>(c) : forward_lanes<float>(c);
}

size_t add_rms_norm_scratch_elems(int rows, int cols) { return (size_t)bwd_groups(rows, bwd_threads(cols)) * cols; }

hipError_t launch_add_rms_norm_bwd(int dtype, int rows, int cols, float eps, const void* dy, const void* ds,
                                   const void* h, const void* g, void* dx, float* dg, int accumulate, float* part,
                                   hipStream_t s) {
  NormCall c{};
  c.rows = rows, c.cols = cols, c.eps = eps, c.s = s;
  c.dy = dy, c.ds = ds, c.h = h, c.g = g, c.dx = dx, c.dg = dg, c.part = part, c.accumulate = accumulate;
  return dtype == DT_BF16 ? backward_lanes<bf16_t>(c) : backward_lanes<float>(c);
}

}  // namespace merak
