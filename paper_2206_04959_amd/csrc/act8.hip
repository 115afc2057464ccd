// Activation checkpoints in 8 bits, and the gradients taken straight from them.
//
// x [rows, cols] is kept as e4m3 codes [rows, cols] and one scale byte for each 32
// consecutive features of a row, [rows, cols / 32].  A scale is a power of two,
// 2^(byte - 127): the smallest that brings the block's largest finite magnitude to
// 448, e4m3's largest value, or below, but at least 2^-117 (the smallest restored
// value, 2^-126, is then still a normal number).  Values are rounded to nearest,
// ties to even: off by at most 2^-4 of the value, or, below 2^-6 of the scale, by
// 2^-10 of the scale.  Magnitudes above 240 * 2^120 are taken as that: the next
// value would restore to infinity.  NaN and infinities are kept as NaN and leave
// their neighbours as they are.
// With power-of-two scales saving divides without rounding, and a restored value
// has 4 significant bits, so it is exact in bf16 too: the bf16 matrix instruction
// takes it as it is.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "gemm_operands.h"
#include "kernels.h"

namespace merak {

constexpr int kScaleBlock = 32;
constexpr int kMinScale = 127 - 117;  // smallest scale byte
constexpr float kLargest = 0x1.ep127f;  // 240 * 2^120

// Scale byte for a block whose largest finite |x| has the bits `m`: exponent - 8,
// plus one where the significand is above 1.75 = 448 / 256.
__device__ __forceinline__ int scale_byte(uint32_t m) {
  const int b = (int)(m >> 23) - 8 + ((m & 0x7fffffu) > 0x600000u);
  return max(b, kMinScale);
}

// Bits of |x| for the block's maximum: 0 for NaN and infinities.
__device__ __forceinline__ uint32_t finite_mag(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}

// Four codes; inv = 1 / scale.
__device__ __forceinline__ uint32_t encode4(const float v[4], float inv) {
  float s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float c = fminf(fmaxf(v[e], -kLargest), kLargest);
    s[e] = finite_mag(v[e]) == (__float_as_uint(v[e]) & 0x7fffffffu) ? c * inv : NAN;
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], r, true);
  return (uint32_t)r;
}

__device__ __forceinline__ void decode4(uint32_t q, float scale, float v[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = lo[0] * scale;
  v[1] = lo[1] * scale;
  v[2] = hi[0] * scale;
  v[3] = hi[1] * scale;
}

// Scale from its byte (10 .. 247 in a saved checkpoint).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// ---------------------------------------------------------------------------
// Save and restore: four lanes to a block, 8 features a lane.
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) act8_save_kernel(long long chunks, const T* __restrict__ x,
                                                        uint8_t* __restrict__ q, uint8_t* __restrict__ scales) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;  // chunk of 8 features
  if (i >= chunks) return;  // chunks is a multiple of 4: whole blocks leave
  float v[8];
  load8(x + i * 8, v);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, finite_mag(v[e]));
  m = max(m, (uint32_t)__shfl_xor((int)m, 1, 64));
  m = max(m, (uint32_t)__shfl_xor((int)m, 2, 64));
  const int b = scale_byte(m);
  const float inv = __uint_as_float((uint32_t)(254 - b) << 23);
  *reinterpret_cast<u32x2_t*>(q + i * 8) = u32x2_t{encode4(v, inv), encode4(v + 4, inv)};
  if ((i & 3) == 0) scales[i >> 2] = (uint8_t)b;
}

template <typename T>
__global__ void __launch_bounds__(256) act8_restore_kernel(long long chunks, const uint8_t* __restrict__ q,
                                                           const uint8_t* __restrict__ scales, T* __restrict__ x) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const u32x2_t c = *reinterpret_cast<const u32x2_t*>(q + i * 8);
  const float s = scale_of(scales[i >> 2]);
  float v[8];
  decode4(c[0], s, v);
  decode4(c[1], s, v + 4);
  store8(x + i * 8, v);
}

// GeLU (tanh form) and its derivative with s = sigmoid(w), w = 2 sqrt(2/pi) (u +
// 0.044715 u^3): gelu = u s, gelu' = s + u s (1 - s) w'(u).  e = exp(-|w|) <= 1 gives
// the larger of s and 1 - s as 1 / (1 + e) and the smaller as e / (1 + e), so
// neither is a difference of nearly equal numbers, in fp32 as in bf16.  From |u| = 64
// on s is 0 or 1; w is formed from the clamped u, so it stays finite.
__device__ __forceinline__ void gelu_both(float u, float* gelu, float* slope) {
  const float uc = fminf(fmaxf(u, -64.0f), 64.0f), u2 = uc * uc;
  const float w = 2.0f * kGeluC * (uc + kGeluA * u2 * uc);
  const float e = __expf(-fabsf(w));
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  const float s = w >= 0.0f ? big : small;
  *gelu = u * s;
  *slope = s + u * (big * small) * (2.0f * kGeluC * (1.0f + 3.0f * kGeluA * u2));
}

// du = dg * gelu'(u) and, unless g is NULL, g = gelu(u), with u in 8 bits.
template <typename T>
__global__ void __launch_bounds__(256) act8_gelu_bwd_kernel(long long chunks, const T* dg, const uint8_t* __restrict__ q,
                                                            const uint8_t* __restrict__ scales, T* du,
                                                            T* __restrict__ g) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const u32x2_t c = *reinterpret_cast<const u32x2_t*>(q + i * 8);
  const float s = scale_of(scales[i >> 2]);
  float u[8], d[8];
  decode4(c[0], s, u);
  decode4(c[1], s, u + 4);
  load8(dg + i * 8, d);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float slope;
    gelu_both(u[e], &u[e], &slope);
    d[e] *= slope;
  }
  store8(du + i * 8, d);
  if (g) store8(g + i * 8, u);
}

// ---------------------------------------------------------------------------
// Weight gradient dW[n, m] (=|+=) sum over tokens t of dY[t, n] X[t, m], X in 8 bits.
//
// bf16: both operands are staged in LDS as they lie in memory, tokens by features,
// and read by the transposing LDS read, as in the weight-gradient GEMM of gemm.hip;
// X's codes become bf16 on the way into LDS.
// ---------------------------------------------------------------------------
constexpr int kDwTile = 128;

// 16 codes of one scale block as 16 bf16 values (exact).
__device__ __forceinline__ void decode16(u32x4_t c, float scale, u32x4_t out[2]) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    decode4(c[i], scale, v);
    out[i >> 1][2 * (i & 1)] = pack_bf16x2(v[0], v[1]);
    out[i >> 1][2 * (i & 1) + 1] = pack_bf16x2(v[2], v[3]);
  }
}

__global__ void __launch_bounds__(256) act8_dw_bf16_kernel(int tokens, int n_out, int n_in,
                                                           const bf16_t* __restrict__ dy,
                                                           const uint8_t* __restrict__ q,
                                                           const uint8_t* __restrict__ scales, float* __restrict__ dw,
                                                           int accumulate) {
  constexpr int R = kDwTile, CPR = R / 8;
  __shared__ __align__(16) char smem[2 * R * 128];
  char* sa = smem;            // dY [64 tokens][128 outputs] bf16
  char* sb = smem + R * 128;  // X  [64 tokens][128 inputs] bf16
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int tiles_n = (n_in + R - 1) / R;
  const int m0 = (blockIdx.x / tiles_n) * R, n0 = (blockIdx.x % tiles_n) * R;
  FragReader<true, R> fr;
  fr.init(lane);
  f32x16_t acc[2][2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.0f;
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  for (int k0 = 0; k0 < tokens; k0 += kBK) {
    __syncthreads();  // the stage before has been read
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // dY: 64 x 16 chunks of 8 outputs
      const int i = threadIdx.x + 256 * u, kr = i / CPR, ch = i % CPR;
      const int t = k0 + kr, m = m0 + ch * 8;
      const u32x4_t v = t < tokens && m < n_out
                            ? *reinterpret_cast<const u32x4_t*>(dy + (size_t)t * n_out + m) : zero;
      *reinterpret_cast<u32x4_t*>(sa + kr * 2 * R + ((ch + 4 * (kr & 3)) % CPR) * 16) = v;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // X: 64 x 8 runs of 16 codes
      const int i = threadIdx.x + 256 * u, kr = i / (R / 16), run = i % (R / 16);
      const int t = k0 + kr, n = n0 + run * 16;
      u32x4_t v[2] = {zero, zero};
      if (t < tokens && n < n_in) {
        const u32x4_t c = *reinterpret_cast<const u32x4_t*>(q + (size_t)t * n_in + n);
        decode16(c, scale_of(scales[(size_t)t * (n_in / kScaleBlock) + n / kScaleBlock]), v);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<u32x4_t*>(sb + kr * 2 * R + ((run * 2 + e + 4 * (kr & 3)) % CPR) * 16) = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < kBK / 16; ++ks) {
      bf16x8_t a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = fr.read(sa, wm * 64 + i * 32, ks);
        b[i] = fr.read(sb, wn * 64 + i * 32, ks);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[i], acc[j][i], 0, 0, 0);
    }
  }
  // acc[j][i][r]: output lane % 32, input (r / 4) * 8 + (lane / 32) * 4 + r % 4
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int m = m0 + wm * 64 + i * 32 + (lane & 31);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = n0 + wn * 64 + j * 32 + g * 8 + (lane >> 5) * 4;
        if (m >= n_out || n >= n_in) continue;
        float v[4] = {acc[j][i][4 * g], acc[j][i][4 * g + 1], acc[j][i][4 * g + 2], acc[j][i][4 * g + 3]};
        float* out = dw + (size_t)m * n_in + n;
        if (accumulate) {
          float o[4];
          load4(out, o);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += o[e];
        }
        store4(out, v);
      }
    }
}

// fp32 check mode, on the fp32 matrix instruction (32 x 32 x 2): 64 x 64 tiles, four
// waves of 32 x 32, 32 tokens a stage.
__global__ void __launch_bounds__(256) act8_dw_f32_kernel(int tokens, int n_out, int n_in, const float* __restrict__ dy,
                                                          const uint8_t* __restrict__ q,
                                                          const uint8_t* __restrict__ scales, float* __restrict__ dw,
                                                          int accumulate) {
  constexpr int R = 64, KB = 32;
  __shared__ __align__(16) float sa[KB][R];
  __shared__ __align__(16) float sb[KB][R];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, hf = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  const int tiles_n = (n_in + R - 1) / R;
  const int m0 = (blockIdx.x / tiles_n) * R, n0 = (blockIdx.x % tiles_n) * R;
  f32x16_t acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
  for (int k0 = 0; k0 < tokens; k0 += KB) {
    __syncthreads();
    const int kr = threadIdx.x >> 3, c8 = (threadIdx.x & 7) * 8;
    const int t = k0 + kr;
    float a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.0f;
    if (t < tokens && m0 + c8 < n_out) load8(dy + (size_t)t * n_out + m0 + c8, a);
    if (t < tokens && n0 + c8 < n_in) {
      const u32x2_t c = *reinterpret_cast<const u32x2_t*>(q + (size_t)t * n_in + n0 + c8);
      const float s = scale_of(scales[(size_t)t * (n_in / kScaleBlock) + (n0 + c8) / kScaleBlock]);
      decode4(c[0], s, b);
      decode4(c[1], s, b + 4);
    }
    store8(&sa[kr][c8], a);
    store8(&sb[kr][c8], b);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KB; k += 2)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(sa[k + hf][wm * 32 + l32], sb[k + hf][wn * 32 + l32], acc, 0, 0, 0);
  }
  // acc[r]: output (r / 4) * 8 + 4 * hf + r % 4, input l32
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int m = m0 + wm * 32 + (r >> 2) * 8 + hf * 4 + (r & 3), n = n0 + wn * 32 + l32;
    if (m >= n_out || n >= n_in) continue;
    float* out = dw + (size_t)m * n_in + n;
    *out = accumulate ? *out + acc[r] : acc[r];
  }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
static bool chunk_grid(int rows, int cols, long long* chunks, dim3* grid) {
  *chunks = (long long)rows * (cols / 8);
  const long long wg = (*chunks + 255) / 256;
  if (wg > 0x7fffffffLL) return false;
  *grid = dim3((unsigned)wg);
  return true;
}

hipError_t launch_act8_save(int dtype, int rows, int cols, const void* x, uint8_t* q, uint8_t* scales, hipStream_t s) {
  long long n;
  dim3 grid;
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidValue;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(act8_save_kernel<bf16_t>, grid, dim3(256), 0, s, n, (const bf16_t*)x, q, scales);
  else
    hipLaunchKernelGGL(act8_save_kernel<float>, grid, dim3(256), 0, s, n, (const float*)x, q, scales);
  return hipGetLastError();
}

hipError_t launch_act8_restore(int dtype, int rows, int cols, const uint8_t* q, const uint8_t* scales, void* x,
                               hipStream_t s) {
  long long n;
  dim3 grid;
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidValue;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(act8_restore_kernel<bf16_t>, grid, dim3(256), 0, s, n, q, scales, (bf16_t*)x);
  else
    hipLaunchKernelGGL(act8_restore_kernel<float>, grid, dim3(256), 0, s, n, q, scales, (float*)x);
  return hipGetLastError();
}

hipError_t launch_act8_gelu_bwd(int dtype, int rows, int cols, const void* dg, const uint8_t* q, const uint8_t* scales,
                                void* du, void* g, hipStream_t s) {
  long long n;
  dim3 grid;
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidValue;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(act8_gelu_bwd_kernel<bf16_t>, grid, dim3(256), 0, s, n, (const bf16_t*)dg, q, scales,
                       (bf16_t*)du, (bf16_t*)g);
  else
    hipLaunchKernelGGL(act8_gelu_bwd_kernel<float>, grid, dim3(256), 0, s, n, (const float*)dg, q, scales, (float*)du,
                       (float*)g);
  return hipGetLastError();
}

size_t act8_gemm_dw_scratch_bytes(int dtype, int tokens, int n_out, int n_in) {
  (void)dtype; (void)tokens; (void)n_out; (void)n_in;
  return 0;
}

hipError_t launch_act8_gemm_dw(int dtype, int tokens, int n_out, int n_in, const void* dy, const uint8_t* q,
                               const uint8_t* scales, float* dw, int accumulate, void* scratch, hipStream_t s) {
  (void)scratch;
  const long long tile = dtype == DT_BF16 ? kDwTile : 64;
  const long long wg = ((n_out + tile - 1) / tile) * ((n_in + tile - 1) / tile);
  if (wg > 0x7fffffffLL) return hipErrorInvalidValue;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(act8_dw_bf16_kernel, dim3((unsigned)wg), dim3(256), 0, s, tokens, n_out, n_in,
                       (const bf16_t*)dy, q, scales, dw, accumulate);
  else
    hipLaunchKernelGGL(act8_dw_f32_kernel, dim3((unsigned)wg), dim3(256), 0, s, tokens, n_out, n_in, (const float*)dy,
                       q, scales, dw, accumulate);
  return hipGetLastError();
}

}  // namespace merak
