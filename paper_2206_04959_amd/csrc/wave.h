// Sums and maxima over the lanes of a wave and the waves of a workgroup without LDS traffic
// between lanes: exchanges within 16 lanes by DPP, beyond by gfx950's row swaps.  Every lane gets
// the result, the sums of the same pairs as in a butterfly (xor 1, 2, 4, 8, 16, 32).
#pragma once

#include "common.h"

namespace merak {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

struct AddOp {
  static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct MaxOp {
  static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

// Over groups of LANES neighbouring lanes (a power of two).
template <typename Op, int LANES>
__device__ __forceinline__ float lanes_reduce(float v) {
  if constexpr (LANES > 1) v = Op::of(v, dpp<0xB1>(v));   // quad_perm [1,0,3,2]
  if constexpr (LANES > 2) v = Op::of(v, dpp<0x4E>(v));   // quad_perm [2,3,0,1]
  if constexpr (LANES > 4) v = Op::of(v, dpp<0x141>(v));  // row_half_mirror: the other four of eight
  if constexpr (LANES > 8) v = Op::of(v, dpp<0x140>(v));  // row_mirror: the other eight of sixteen
  if constexpr (LANES > 16) {  // rows 0, 0, 2, 2 and 1, 1, 3, 3
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = Op::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (LANES > 32) {  // both halves twice
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = Op::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}

// N values over the NT threads of a workgroup (NT a multiple of 64).  red: NT / 64 * N floats of
// LDS; one barrier, so an area may be used again only behind another one.
template <typename Op, int NT, int N>
__device__ __forceinline__ void block_reduce(float (&v)[N], float* red) {
  constexpr int W = NT / 64;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lanes_reduce<Op, 64>(v[n]);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) red[n * W + (threadIdx.x >> 6)] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_reduce<Op, W>(red[n * W + (threadIdx.x & (W - 1))]);
  }
}

}  // namespace merak
