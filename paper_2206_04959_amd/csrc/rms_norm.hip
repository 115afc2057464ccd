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
// each: chunk i of thread j holds the features from (j + NT i) * 8 on.  In bf16 with a residual:
// 32768 x 6144 262 us (6.1 TB/s; a large copy has 5.1), 16384 x 1920 with y and its 8 bits 54
// (5.3); gradients of 16384 x 6144 139 (5.8), of 4097 x 1600 13.6 and 4 for the gain (3.9).
#include <algorithm>

#include "act8_codes.h"
#include "common.h"
#include "kernels.h"
#include "wave.h"

namespace merak {

constexpr int threads_of(int nt) { return nt == 64 ? 256 : nt; }  // of a workgroup: four rows of 64 threads, or one row

// v rounded to T (what a store would keep).
template <typename T>
__device__ __forceinline__ void round8(float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = Elem<T>::to_f(Elem<T>::from_f(v[e]));
}

// Eight values as they lie in memory.
template <typename T>
struct Eight {
  u32x4_t r[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = reinterpret_cast<const u32x4_t*>(p)[i];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (sizeof(T) == 2) {
      unpack8(r[0], v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r[e / 4][e % 4]);
    }
  }
};

// Eight values to memory, past the caches if PAST.
template <bool PAST>
__device__ __forceinline__ void put8(bf16_t* p, const float v[8]) {
  store16<PAST>(p, u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                           pack_bf16x2(v[6], v[7])});
}
template <bool PAST>
__device__ __forceinline__ void put8(float* p, const float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 4)
    store16<PAST>(p + i, u32x4_t{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]),
                                 __float_as_uint(v[i + 3])});
}

// Where a row's squares leave fp32 (a sum of 2^128: a row of 16384 features of 2^57) the sums are taken
// again of 2^-80 h, whose squares stay below 2^110; rstd is 2^-80 times that of the scaled row,
// down to 2^-128 (22 bits).  The branch is the whole row's, taken by no ordinary one.
constexpr float kUnit = 0x1p-80f;
__device__ __forceinline__ float scaled_rstd(float squares, int cols, float eps) {
  return 1.0f / sqrtf(squares / (float)cols + eps * kUnit * kUnit);
}

struct NormFwd {
  int rows, cols;
  float eps;
};

// sum may be x or r.
template <typename T, int NT, int CH, bool Q8, bool PAST>
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
  float rstd = 1.0f / sqrtf(s[0] / (float)a.cols + a.eps);
  if (s[0] == INFINITY) {
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if ((j + NT * i) * 8 >= a.cols) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += (h[i][e] * kUnit) * (h[i][e] * kUnit);
    }
    if constexpr (NT > 64) __syncthreads();  // the first sums are read
    block_reduce<AddOp, NT>(s, red);
    rstd = scaled_rstd(s[0], a.cols, a.eps) * kUnit;
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (j + NT * i) * 8;
    if (c >= a.cols) continue;
    if (sum) put8<PAST>(sum + at + c, h[i]);
    float w[8], o[8];
    load8(g + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = h[i][e] * rstd * w[e];
    if (y) put8<PAST>(y + at + c, o);
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

constexpr int kRun = 256;  // rows that a thread of the gradient adds up one after the other

// The workgroups step through the rows; each thread keeps its columns' sums of dy * n, and a
// workgroup's go to part[workgroup][cols] (without part there is one workgroup, whose sums are
// the gain's gradient).  With one chunk a thread a row's loads are issued while the row before
// it is reduced and written: 16384 x 1920 in bf16 57 -> 51 us, x 6144 156 -> 144; with more the
// registers would not hold both.  dx may be dy or ds: a row is loaded whole before it is written.
// A thread's sum of kRun rows goes into memory (into LDS with 64 threads a row) and the next one starts
// at 0, so a column's longest chain of additions is kRun + rows / (rows at a time) / kRun and a tree.
template <typename T, int NT, int CH, bool PAST>
__global__ void __launch_bounds__(threads_of(NT)) rms_bwd_kernel(int rows, int cols, float eps, const T* dy,
                                                                 const T* ds, const T* __restrict__ h,
                                                                 const T* __restrict__ g, T* dx,
                                                                 float* __restrict__ part, float* __restrict__ dg,
                                                                 int accumulate) {
  constexpr int R = threads_of(NT) / NT;
  constexpr bool AHEAD = CH == 1;
  __shared__ __align__(16) float red[NT > 64 ? 2 * 2 * (NT / 64) : R * CH * 512];
  const int j = threadIdx.x % NT;
  const long long step = (long long)gridDim.x * R;
  float sum[CH][8];
  Eight<T> w[CH], d[CH], v[CH], s[CH];  // the gain; the row's dy, h and ds
  auto load_row = [&](long long r) {
    const size_t at = (size_t)r * cols;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      d[i].load(dy + at + c);
      v[i].load(h + at + c);
      if (AHEAD && ds) s[i].load(ds + at + c);
    }
  };
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (j + NT * i) * 8;
    if (AHEAD && c < cols) w[i].load(g + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[i][e] = 0.0f;
  }
  const long long first = (long long)blockIdx.x * R + threadIdx.x / NT;
  if (AHEAD && first < rows) load_row(first);
  int buf = 0;
  float* const out = part ? part + (size_t)blockIdx.x * cols : dg;
  // The thread's sums to its place, on top of what is there if `add`.
  auto give = [&](bool add) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      float* const to = NT > 64 ? out + c : red + (threadIdx.x / NT) * CH * 512 + c;
      if (add) {
        float before[8];
        load8(to, before);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[i][e] += before[e];
      }
      store8(to, sum[i]);
    }
  };
  bool given = false;
  int run = 0;
  for (long long row = first; row < rows; row += step) {
    const size_t at = (size_t)row * cols;
    if (!AHEAD) load_row(row);
    float t[2] = {0.0f, 0.0f};
    float dv[CH][8], hv[CH][8], o[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      float g8[8];
      if (!AHEAD) w[i].load(g + c);
      w[i].get(g8);
      d[i].get(dv[i]);
      v[i].get(hv[i]);
      if (AHEAD && ds) s[i].get(o[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[0] += hv[i][e] * hv[i][e];
        t[1] += dv[i][e] * g8[e] * hv[i][e];
      }
    }
    if (AHEAD && row + step < rows) load_row(row + step);
    block_reduce<AddOp, NT>(t, red + buf);
    buf ^= 2 * (NT / 64);  // two areas in turn: one barrier a row is enough
    float rstd = 1.0f / sqrtf(t[0] / (float)cols + eps);
    float m = t[1] * rstd / (float)cols;  // mean(dy g n)
    if (t[0] == INFINITY) {
      t[0] = t[1] = 0.0f;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = (j + NT * i) * 8;
        if (c >= cols) continue;
        float g8[8];
        if (!AHEAD) w[i].load(g + c);
        w[i].get(g8);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = hv[i][e] * kUnit;
          t[0] += u * u;
          t[1] += dv[i][e] * g8[e] * u;
        }
      }
      block_reduce<AddOp, NT>(t, red + buf);
      buf ^= 2 * (NT / 64);
      rstd = scaled_rstd(t[0], cols, eps);
      m = t[1] * rstd / (float)cols;
      rstd *= kUnit;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (j + NT * i) * 8;
      if (c >= cols) continue;
      float g8[8];
      if (!AHEAD) {
        w[i].load(g + c);
        if (ds) {
          s[i].load(ds + at + c);
          s[i].get(o[i]);
        }
      }
      w[i].get(g8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = hv[i][e] * rstd, x = rstd * (dv[i][e] * g8[e] - n * m);
        sum[i][e] += dv[i][e] * n;
        o[i][e] = ds ? o[i][e] + x : x;
      }
      put8<PAST>(dx + at + c, o[i]);
    }
    if (++run == kRun) {  // (one workgroup without part has four rows)
      give(given);
      given = true;
      run = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[i][e] = 0.0f;
    }
  }
  const bool add = !part && accumulate;
  if constexpr (NT > 64) {
    give(given || add);
  } else {
    give(given);
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 256) {
      const float v = (red[c] + red[CH * 512 + c]) + (red[2 * CH * 512 + c] + red[3 * CH * 512 + c]);
      out[c] = add ? out[c] + v : v;
    }
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

template <typename T>
static size_t out_bytes(const NormCall& c) { return (size_t)c.rows * c.cols * sizeof(T); }

struct NormForward {
  template <typename T, int NT, int CH, bool Q8, bool PAST>
  static hipError_t launch(const NormCall& c) {
    constexpr int threads = threads_of(NT), R = threads / NT;
    const long long most = max_groups(threads) * R;  // rows of a launch; a call of more goes in several
    for (long long at = 0; at < c.rows; at += most) {
      const NormFwd a{(int)std::min(most, c.rows - at), c.cols, c.eps};
      const size_t off = (size_t)at * c.cols;
      auto past = [off](const void* p) { return p ? (T*)p + off : nullptr; };
      hipLaunchKernelGGL((rms_fwd_kernel<T, NT, CH, Q8, PAST>), dim3((unsigned)((a.rows + R - 1) / R)), dim3(threads), 0,
                         c.s, a, past(c.x), past(c.r), (const T*)c.g, past(c.sum), past(c.y), Q8 ? c.q + off : nullptr,
                         Q8 ? c.scales + off / kScaleBlock : nullptr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  template <typename T, int NT, int CH>
  static hipError_t run(const NormCall& c) {
    if (out_bytes<T>(c) >= kStreamBytes) return c.q ? launch<T, NT, CH, true, true>(c) : launch<T, NT, CH, false, true>(c);
    return c.q ? launch<T, NT, CH, true, false>(c) : launch<T, NT, CH, false, false>(c);
  }
};

// Threads of a row in the gradient: one chunk a thread up to 8192 columns.
static int bwd_threads(int cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }

// Workgroups of the gradient: few, as a row is loaded ahead and each one's sums are written and
// read again, but at least two rows each.  16384 rows in bf16 with 256 / 512 / 1024 (of 1024,
// 512, 256 threads): x 8192 (256 or 512 of 1024) 103 / 107 us, x 4096 (512) 97 / 104, x 1920 (256)
// 67 / 51 / 54, x 1000 (128) - / 29 / 32; 300 x 6144 with 128 / 256 / 300 11.7 / 12.5 / 14.1.
static int bwd_groups(int rows, int cols) {
  const int nt = bwd_threads(cols), per = threads_of(nt) / nt;
  const int most = nt >= 512 ? 256 : nt == 128 ? 1024 : 512;
  return std::max(1, std::min((rows + 2 * per - 1) / (2 * per), most));
}

// Up to four steps of one workgroup take less than the launch that would add the sums of several.
static bool bwd_alone(int rows, int cols) {
  const int nt = bwd_threads(cols);
  return rows <= 4 * (threads_of(nt) / nt);
}

struct NormBackward {
  template <typename T, int NT, int CH, bool PAST>
  static hipError_t launch(const NormCall& c) {
    const bool alone = bwd_alone(c.rows, c.cols);
    const int wg = alone ? 1 : bwd_groups(c.rows, c.cols);
    hipLaunchKernelGGL((rms_bwd_kernel<T, NT, CH, PAST>), dim3(wg), dim3(threads_of(NT)), 0, c.s, c.rows, c.cols, c.eps,
                       (const T*)c.dy, (const T*)c.ds, (const T*)c.h, (const T*)c.g, (T*)c.dx,
                       alone ? nullptr : c.part, c.dg, c.accumulate);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || alone) return e;
    hipLaunchKernelGGL(rms_gain_kernel, dim3((c.cols + 15) / 16), dim3(1024), 0, c.s, c.cols, wg, c.part, c.dg,
                       c.accumulate);
    return hipGetLastError();
  }
  template <typename T, int NT, int CH>
  static hipError_t run(const NormCall& c) {
    return out_bytes<T>(c) >= kStreamBytes ? launch<T, NT, CH, true>(c) : launch<T, NT, CH, false>(c);
  }
};

// One chunk a thread up to 4096 columns, two up to 8192: 16384 x 1920 with a residual in bf16
// 44 us (four chunks on 64 threads 55), 32768 x 6144 265 with two on 512 (three on 256 274, one on
// 1024 271).
template <typename T>
static hipError_t forward_lanes(const NormCall& c) {
  if (c.cols <= 512) return NormForward::run<T, 64, 1>(c);
  if (c.cols <= 1024) return NormForward::run<T, 128, 1>(c);
  if (c.cols <= 2048) return NormForward::run<T, 256, 1>(c);
  if (c.cols <= 4096) return NormForward::run<T, 512, 1>(c);
  if (c.cols <= 8192) return NormForward::run<T, 512, 2>(c);
  return NormForward::run<T, 1024, 2>(c);
}

template <typename T>
static hipError_t backward_lanes(const NormCall& c) {
  switch (bwd_threads(c.cols)) {
    case 64: return NormBackward::run<T, 64, 1>(c);
    case 128: return NormBackward::run<T, 128, 1>(c);
    case 256: return NormBackward::run<T, 256, 1>(c);
    case 512: return NormBackward::run<T, 512, 1>(c);
  }
  return c.cols <= 8192 ? NormBackward::run<T, 1024, 1>(c) : NormBackward::run<T, 1024, 2>(c);
}

hipError_t launch_add_rms_norm_fwd(int dtype, int rows, int cols, float eps, const void* x, const void* r,
                                   const void* g, void* sum, void* y, uint8_t* q, uint8_t* scales, hipStream_t s) {
  NormCall c{};
  c.rows = rows, c.cols = cols, c.eps = eps, c.s = s;
  c.x = x, c.r = r, c.g = g, c.sum = sum, c.y = y, c.q = q, c.scales = scales;
  return dtype == DT_BF16 ? forward_lanes<bf16_t>(c) : forward_lanes<float>(c);
}

size_t add_rms_norm_scratch_elems(int rows, int cols) {
  return bwd_alone(rows, cols) ? 0 : (size_t)bwd_groups(rows, cols) * cols;
}

hipError_t launch_add_rms_norm_bwd(int dtype, int rows, int cols, float eps, const void* dy, const void* ds,
                                   const void* h, const void* g, void* dx, float* dg, int accumulate, float* part,
                                   hipStream_t s) {
  NormCall c{};
  c.rows = rows, c.cols = cols, c.eps = eps, c.s = s;
  c.dy = dy, c.ds = ds, c.h = h, c.g = g, c.dx = dx, c.dg = dg, c.part = part, c.accumulate = accumulate;
  return dtype == DT_BF16 ? backward_lanes<bf16_t>(c) : backward_lanes<float>(c);
}

}  // namespace merak
