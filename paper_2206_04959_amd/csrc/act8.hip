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
#include <atomic>
#include <cmath>

#include "act8_codes.h"
#include "common.h"
#include "gemm_operands.h"
#include "kernels.h"

namespace merak {

__device__ __forceinline__ void decode4(uint32_t q, float scale, float v[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = lo[0] * scale;
  v[1] = lo[1] * scale;
  v[2] = hi[0] * scale;
  v[3] = hi[1] * scale;
}

// Two codes of a word as bf16 (exact).
template <bool HI>
__device__ __forceinline__ uint32_t decode2_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

__device__ __forceinline__ u32x4_t decode8_bf16(uint32_t lo, uint32_t hi, float scale) {
  return u32x4_t{decode2_bf16<false>(lo, scale), decode2_bf16<true>(lo, scale), decode2_bf16<false>(hi, scale),
                 decode2_bf16<true>(hi, scale)};
}

// Scale from its byte (10 .. 247 in a saved checkpoint).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// ---------------------------------------------------------------------------
// Save and restore: four lanes to a block, 8 features a lane.  Bound by memory: 16384 x
// 6144 in bf16 (305 MB each) 54 and 49 us, one behind the other 98 (the codes are then
// still in the last-level cache); in fp32 (506 MB) 87 and 132.
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

template <typename T, bool PAST>
__global__ void __launch_bounds__(256) act8_restore_kernel(long long chunks, const uint8_t* __restrict__ q,
                                                           const uint8_t* __restrict__ scales, T* __restrict__ x) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const u32x2_t c = *reinterpret_cast<const u32x2_t*>(q + i * 8);
  const float s = scale_of(scales[i >> 2]);
  if constexpr (sizeof(T) == 2) {
    store16<PAST>(x + i * 8, decode8_bf16(c[0], c[1], s));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[4];
      decode4(c[h], s, v);
      store16<PAST>(x + i * 8 + 4 * h, u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                                               __float_as_uint(v[3])});
    }
  }
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

// Bound by memory (8191 x 6400 in bf16, 369 MB: 64 us; without g 47; in fp32 125): one
// exponential and one reciprocal a value fit beside it.
// du = dg * gelu'(u) and, unless g is NULL, g = gelu(u), with u in 8 bits.
template <typename T>
__global__ void __launch_bounds__(256) act8_gelu_bwd_kernel(long long chunks, const T* dg,
                                                            const uint8_t* __restrict__ q,
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
// bf16: v_mfma_f32_32x32x16_bf16, fp32 accumulators, 64 tokens a stage, two LDS
// buffers.  Both operands lie in LDS as in memory, tokens by features (swizzled, see
// gemm.hip), and are read by the transposing LDS read.  dY goes global -> LDS
// directly.  X's codes go to registers a stage ahead, 16 codes of one scale block at
// a time, and become bf16 on the way into LDS: eight conversions that take the scale
// along for 16 values.  Converting there costs each value one conversion in a
// workgroup; behind LDS every wave that shares a column would convert it again.
// Even so the conversions and their LDS writes take a fifth of a large product's time,
// so there (dw_plan) X is restored once into scratch instead and goes global -> LDS
// directly too.
//
// A stage has four sub-steps; each reads the next one's fragments between its MFMAs.
// Behind the barrier at the end of stage kt's reads its buffer is refilled with
// stage kt + 2, piece by piece between the MFMAs too: dY's loads and the loads of the
// codes of stage kt + 3 in the last sub-step, the conversions in the next two.  Every
// wait is for the loads of a whole stage ago.  A workgroup alone on its CU has nothing
// else to run meanwhile and waits for memory once a stage; it has eight waves and, from
// eight times kBK tokens on, stages of twice the length (H = 2): 4096 x 2048 x 2048 52.8 us
// with four waves and one kBK a stage, 44.6 so; 64 x 1024 x 1024 5.2, and 6.1 with H = 2;
// 512 x 1024 x 1024 9.3 either way.
// Buffers are addressed from each stage's first token, so operands may be of any
// size; tokens past the end read as zeros.
// ---------------------------------------------------------------------------
struct DwArgs {
  int tokens, n_out, n_in;
  int per_split;  // tokens of a split, a multiple of 64 (or all)
  int tiles;      // output tiles of a split
  int accumulate;
  const bf16_t* dy;
  const uint8_t* q;       // X: codes and scales, or
  const uint8_t* scales;
  const bf16_t* x;        // its values
  float* out;     // splits = 1: dw; else the splits' sums [splits][n_out][n_in]
};

// Raw buffer of `rows` rows of `ld` bytes from p, empty if rows <= 0.
__device__ __forceinline__ i32x4_t stage_rsrc(const void* p, int rows, size_t ld) {
  return operand_rsrc_words(p, rows > 0 ? (uint32_t)(min(rows, kBK) * ld) : 0u);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t stage_buffer(const void* p, int rows, size_t ld) {
  return operand_rsrc(p, rows > 0 ? (uint32_t)(min(rows, kBK) * ld) : 0u);
}

template <int BM, int BN, int WM, int WN, bool CODES, int H>
__global__ void __launch_bounds__(WM * WN * 64) act8_dw_kernel(DwArgs p) {
  constexpr int NW = WM * WN, NT = NW * 64;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  // A stage is H times kBK tokens, each kBK with its own part of the LDS buffer.
  constexpr int A_BYTES = BM * 128, PART = (BM + BN) * 128, STAGE = H * PART;
  constexpr int LA = BM / 8 / NW;         // dY loads of a wave and part
  // X: runs of 16 codes of a thread and part, or loads of a wave
  constexpr int LB = CODES ? BN * kBK / 16 / NT : BN / 8 / NW;
  constexpr int RPR = BN / 16, CPR = BN / 8;
  static_assert(!CODES || (LB * NT * 16 == BN * kBK && CPR % 16 == 0), "whole runs, slots in pairs");
  extern __shared__ __align__(16) char smem[];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // Each XCD takes neighbouring tiles, in groups of four tile rows.
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int split = id / p.tiles, tile = id - split * p.tiles;
  const int tiles_m = (p.n_out + BM - 1) / BM, tiles_n = (p.n_in + BN - 1) / BN;
  constexpr int GM = 4;
  const int group = tile / (GM * tiles_n), first_m = group * GM;
  const int gsz = min(tiles_m - first_m, GM), in_group = tile - group * GM * tiles_n;
  const int m0 = (first_m + in_group % gsz) * BM, n0 = (in_group / gsz) * BN;

  const int k0 = split * p.per_split;
  const int rows = min(p.per_split, p.tokens - k0);
  const int KT = (rows + H * kBK - 1) / (H * kBK);
  const size_t lda = (size_t)p.n_out * 2, ldx = (size_t)p.n_in * 2, ldq = p.n_in, lds = p.n_in / kScaleBlock;
  const char* pa = reinterpret_cast<const char*>(p.dy) + (size_t)k0 * lda;
  const char* px = reinterpret_cast<const char*>(p.x) + (size_t)k0 * ldx;
  const uint8_t* pq = p.q + (size_t)k0 * ldq;
  const uint8_t* ps = p.scales + (size_t)k0 * lds;

  TileLoader<true, BM, NW> la;
  TileLoader<true, BN, NW> lb;
  la.init(m0, p.n_out, wave, lane);
  la.step = lb.step = 0;  // the buffers' starts move instead
  if constexpr (!CODES) {
    lb.init(n0, p.n_in, wave, lane);
    lb.step = 0;
  }
  uint32_t qoff[LB], soff[LB], w0[LB];
  if constexpr (CODES) {
#pragma unroll
    for (int u = 0; u < LB; ++u) {
      const int i = threadIdx.x + NT * u, kr = i / RPR, run = i % RPR;
      qoff[u] = (uint32_t)(kr * p.n_in + n0 + run * 16);
      soff[u] = (uint32_t)(kr * (p.n_in / kScaleBlock) + (n0 + run * 16) / kScaleBlock);
      w0[u] = (uint32_t)(A_BYTES + kr * 2 * BN + ((run * 2 + 4 * (kr & 3)) % CPR) * 16);
    }
  }
  FragReader<true, BM> fa;
  FragReader<true, BN> fb;
  fa.init(lane);
  fb.init(lane);

  f32x16_t acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.0f;

  // The codes of the next stage to convert, and of the one after it (on their way).
  struct Codes {
    u32x4_t q[H][LB];
    uint32_t s[H][LB];
  } now, next;
  bf16x8_t a0[TM], a1[TM], b0[TN], b1[TN];  // two fragment sets
  auto load_codes = [&](Codes& c, int kt, int h, int u) {  // run u of part h of stage kt
    const int k = kt * H + h, left = rows - k * kBK;
    const __amdgpu_buffer_rsrc_t rq = stage_buffer(pq + (size_t)k * kBK * ldq, left, ldq);
    const __amdgpu_buffer_rsrc_t rc = stage_buffer(ps + (size_t)k * kBK * lds, left, lds);
    c.q[h][u] = __builtin_amdgcn_raw_buffer_load_b128(rq, qoff[u], 0, 0);
    c.s[h][u] = __builtin_amdgcn_raw_buffer_load_b8(rc, soff[u], 0, 0);
  };
  // Half run i of the stage in `now`, counted through its parts; a run's halves are neighbours
  // in LDS.
  auto write_codes = [&](char* st, int i) {
    const int h = i / (2 * LB), u = i % (2 * LB) / 2, half = i % 2;
    *reinterpret_cast<u32x4_t*>(st + h * PART + w0[u] + 16 * half) =
        decode8_bf16(now.q[h][u][2 * half], now.q[h][u][2 * half + 1], scale_of(now.s[h][u]));
  };
  // Tokens kBK k on of the split.
  auto x_rsrc = [&](int k) { return stage_rsrc(px + (size_t)k * kBK * ldx, rows - k * kBK, ldx); };
  auto dy_rsrc = [&](int k) { return stage_rsrc(pa + (size_t)k * kBK * lda, rows - k * kBK, lda); };
  // A sub-step: the MFMAs of set c, each followed by the read of one fragment of (st, ks)
  // into set n and by piece(u), in that order.
  constexpr int NMF = TM * TN;
  constexpr int RPM = (TM + TN + NMF - 1) / NMF;  // fragment reads behind an MFMA
  auto step = [&](const char* st, int ks, bf16x8_t (&na)[TM], bf16x8_t (&nb)[TN], const bf16x8_t (&ca)[TM],
                  const bf16x8_t (&cb)[TN], auto piece) {
#pragma unroll
    for (int u = 0; u < NMF; ++u) {
      acc[u / TM][u % TM] =
          __builtin_amdgcn_mfma_f32_32x32x16_bf16(cb[u / TM], ca[u % TM], acc[u / TM][u % TM], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < RPM; ++e) {
        const int f = u * RPM + e;
        if (f < TN) nb[f] = fb.read(st + A_BYTES, wn * WTN + f * 32, ks);
        else if (f < TN + TM) na[f - TN] = fa.read(st, wm * WTM + (f - TN) * 32, ks);
      }
      piece(u);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Both buffers' loads go out before the first wait.
#pragma unroll
  for (int k = 0; k < 2 * H; ++k) {
    la.issue(dy_rsrc(k), smem + k * PART, wave);
    if constexpr (!CODES) lb.issue(x_rsrc(k), smem + k * PART + A_BYTES, wave);
  }
  auto load_stage = [&](Codes& c, int kt) {
#pragma unroll
    for (int i = 0; i < H * LB; ++i) load_codes(c, kt, i / LB, i % LB);
  };
  if constexpr (CODES) {
    load_stage(now, 0);
    load_stage(next, 1);
#pragma unroll
    for (int i = 0; i < 2 * LB * H; ++i) write_codes(smem, i);
  }
  wait_vm_barrier<0>();
  if constexpr (CODES) {
    now = next;
    load_stage(next, 2);
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) b0[j] = fb.read(smem + A_BYTES, wn * WTN + j * 32, 0);
#pragma unroll
  for (int i = 0; i < TM; ++i) a0[i] = fa.read(smem, wm * WTM + i * 32, 0);
  __builtin_amdgcn_sched_barrier(0);

  // Past the last stage the loads find empty buffers: they fetch nothing and write zeros.
  for (int kt = 0; kt < KT; ++kt) {
    char* st = smem + (kt & 1) * STAGE;
    char* other = smem + ((kt + 1) & 1) * STAGE;
    // LB half runs of the next stage are converted in each of the first 2 H sub-steps.
    auto convert = [&](int i, int u) {
      if constexpr (CODES) {
        constexpr int EVERY = NMF / LB;
        static_assert(NMF % LB == 0, "conversions spread evenly over the MFMAs");
        if (i <= 2 * H && u % EVERY == 0) write_codes(other, (i - 1) * LB + u / EVERY);
      }
    };
#pragma unroll
    for (int i = 1; i < 4 * H; ++i) {
      if (i & 1) step(st + i / 4 * PART, i % 4, a1, b1, a0, b0, [&](int u) { convert(i, u); });
      else step(st + i / 4 * PART, i % 4, a0, b0, a1, b1, [&](int u) { convert(i, u); });
    }
    wait_vm_barrier<0>();  // stage kt + 1 is in LDS, `next` is there, and all have read stage kt
    if constexpr (CODES) now = next;
    i32x4_t ra[H], rx[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      ra[h] = dy_rsrc((kt + 2) * H + h);
      rx[h] = x_rsrc(CODES ? 0 : (kt + 2) * H + h);
    }
    constexpr int NP = H * (LA + LB), PER = (NP + NMF - 1) / NMF;
    step(other, 0, a0, b0, a1, b1, [&](int u) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int c = u * PER + e, h = c / (LA + LB), r = c % (LA + LB);
        if (c >= NP) continue;
        if (r < LA) la.issue_one(ra[h], st + h * PART, wave, r);
        else if constexpr (CODES) load_codes(next, kt + 3, h, r - LA);
        else lb.issue_one(rx[h], st + h * PART + A_BYTES, wave, r - LA);
      }
    });
  }
  wait_vm_barrier<0>();  // nothing is on its way into LDS any more

  // acc[j][i][r]: output lane % 32, input (r / 4) * 8 + (lane / 32) * 4 + r % 4.  Through
  // LDS, a 32-row slab of the wave's tile at a time, so that lanes write whole row segments.
  constexpr int CLD = WTN + 4, CPW = WTN / 8, CPL = 32 * CPW / 64;
  static_assert((size_t)NW * 32 * CLD * 4 <= 2 * STAGE, "epilogue staging fits in the operand buffers");
  float* stg = reinterpret_cast<float*>(smem) + wave * 32 * CLD;
  float* out = p.out + (size_t)split * p.n_out * p.n_in;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4_t*>(stg + (lane & 31) * CLD + j * 32 + g * 8 + (lane >> 5) * 4) =
            f32x4_t{acc[j][i][4 * g], acc[j][i][4 * g + 1], acc[j][i][4 * g + 2], acc[j][i][4 * g + 3]};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the staging slab is this wave's own
#pragma unroll
    for (int u = 0; u < CPL; ++u) {
      const int c = lane + 64 * u, r = c / CPW, cc = c % CPW;
      const int m = m0 + wm * WTM + i * 32 + r, n = n0 + wn * WTN + cc * 8;
      if (m < p.n_out && n < p.n_in) {
        float v[8];
        load8(stg + r * CLD + cc * 8, v);
        float* o = out + (size_t)m * p.n_in + n;
        if (p.accumulate) {
          float w[8];
          load8(o, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
        store8(o, v);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// dw (=|+=) the splits' sums.  SLICES threads of a workgroup share a chunk of four columns:
// each adds a part of the splits in order, and the parts are added in order.
template <int SLICES>
__global__ void __launch_bounds__(256) act8_dw_join_kernel(long long chunks, int splits, const float* __restrict__ part,
                                                           float* __restrict__ dw, int accumulate) {
  constexpr int CPB = 256 / SLICES;
  __shared__ f32x4_t red[SLICES > 1 ? 256 : 1];
  const int c = threadIdx.x % CPB, sl = threadIdx.x / CPB;
  const long long i = (long long)blockIdx.x * CPB + c;
  const bool live = i < chunks;
  const int per = (splits + SLICES - 1) / SLICES, end = min(splits, (sl + 1) * per);
  f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (live) {
#pragma unroll 8
    for (int k = sl * per; k < end; ++k) {
      const f32x4_t v = reinterpret_cast<const f32x4_t*>(part)[k * chunks + i];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
  }
  if constexpr (SLICES > 1) {
    red[threadIdx.x] = s;
    __syncthreads();
    if (sl > 0) return;
    for (int k = 1; k < SLICES; ++k) {
      const f32x4_t v = red[k * CPB + c];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
  }
  if (!live) return;
  f32x4_t* o = reinterpret_cast<f32x4_t*>(dw) + i;
  if (accumulate) {
    const f32x4_t v = *o;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = v[e] + s[e];
  }
  *o = s;
}

// Many splits (16 and more, of small outputs) share a chunk among eight threads: a call of
// 171 splits of 64 x 64 takes 10.9 us, 18.4 with one thread a chunk; 128 of 128 x 128 12.3
// and 17.0.
static hipError_t launch_dw_join(long long elems, int splits, const float* part, float* dw, int accumulate,
                                 hipStream_t s) {
  const long long chunks = elems / 4;
  if (splits >= 16)
    hipLaunchKernelGGL(act8_dw_join_kernel<8>, dim3((unsigned)((chunks + 31) / 32)), dim3(256), 0, s, chunks, splits,
                       part, dw, accumulate);
  else
    hipLaunchKernelGGL(act8_dw_join_kernel<1>, dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, s, chunks, splits,
                       part, dw, accumulate);
  return hipGetLastError();
}

// fp32 check mode, on the fp32 matrix instruction (32 x 32 x 2): tiles of 64 NB x 64 NB, four
// waves of 32 NB x 32 NB, 32 tokens a stage.  The next stage's operands are on their way to
// registers meanwhile, X's as codes until they go to LDS, and fragments are read ahead of
// their MFMAs.  Bound by the matrix instruction's rate: 8192 x 4096 x 4096 2.13 ms (129
// TFLOP/s; 151 is what the library reaches there), and 2.19 with NB = 1; 1000 x 3000 x 1024
// 62 us with NB = 1 and 70 with NB = 2.
constexpr int kStageF32 = 32;

template <int NB>
__global__ void __launch_bounds__(256) act8_dw_f32_kernel(DwArgs p, const float* __restrict__ dy) {
  constexpr int R = 64 * NB, KB = kStageF32, W = 32 * NB;
  __shared__ __align__(16) float sa[KB][R];
  __shared__ __align__(16) float sb[KB][R];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, hf = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  const int split = blockIdx.x / p.tiles, tile = blockIdx.x - split * p.tiles;
  const int tiles_n = (p.n_in + R - 1) / R;
  const int m0 = (tile / tiles_n) * R, n0 = (tile % tiles_n) * R;
  const int first = split * p.per_split, end = min(p.tokens, first + p.per_split);
  const int kr = threadIdx.x >> 3, c8 = (threadIdx.x & 7) * 8;  // columns c8 + 64 u of row kr
  f32x16_t acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  f32x4_t a[NB][2];
  u32x2_t codes[NB];
  uint32_t byte[NB];
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int m = m0 + 64 * u + c8, n = n0 + 64 * u + c8;
      a[u][0] = a[u][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      codes[u] = u32x2_t{0u, 0u};
      byte[u] = 0;
      if (t < end && m < p.n_out) {
        const float* q = dy + (size_t)t * p.n_out + m;
        a[u][0] = reinterpret_cast<const f32x4_t*>(q)[0];
        a[u][1] = reinterpret_cast<const f32x4_t*>(q)[1];
      }
      if (t < end && n < p.n_in) {
        codes[u] = *reinterpret_cast<const u32x2_t*>(p.q + (size_t)t * p.n_in + n);
        byte[u] = p.scales[(size_t)t * (p.n_in / kScaleBlock) + n / kScaleBlock];
      }
    }
  };
  fetch(first + kr);
  for (int k0 = first; k0 < end; k0 += KB) {
    __syncthreads();  // the stage before has been read
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      float b[8];
      decode4(codes[u][0], scale_of(byte[u]), b);
      decode4(codes[u][1], scale_of(byte[u]), b + 4);
      *reinterpret_cast<f32x4_t*>(&sa[kr][64 * u + c8]) = a[u][0];
      *reinterpret_cast<f32x4_t*>(&sa[kr][64 * u + c8 + 4]) = a[u][1];
      store8(&sb[kr][64 * u + c8], b);
    }
    __syncthreads();
    fetch(k0 + KB + kr);
    constexpr int AHEAD = NB == 1 ? 2 : 1;  // steps
    float fa[KB / 2][NB], fb[KB / 2][NB];
#pragma unroll
    for (int s = 0; s < KB / 2 + AHEAD; ++s) {
      if (s < KB / 2) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          fa[s][i] = sa[2 * s + hf][wm * W + 32 * i + l32];
          fb[s][i] = sb[2 * s + hf][wn * W + 32 * i + l32];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (s >= AHEAD) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[s - AHEAD][i], fb[s - AHEAD][j], acc[i][j], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // acc[r]: output (r / 4) * 8 + 4 * hf + r % 4, input l32
  float* dw = p.out + (size_t)split * p.n_out * p.n_in;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = m0 + wm * W + 32 * i + (r >> 2) * 8 + hf * 4 + (r & 3), n = n0 + wn * W + 32 * j + l32;
        if (m >= p.n_out || n >= p.n_in) continue;
        float* out = dw + (size_t)m * p.n_in + n;
        *out = p.accumulate ? *out + acc[i][j][r] : acc[i][j][r];
      }
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
static bool chunk_grid(int rows, int cols, long long* chunks, dim3* grid) {
  *chunks = (long long)rows * (cols / 8);
  const long long wg = (*chunks + 255) / 256;
  if (wg > max_groups(256)) return false;
  *grid = dim3((unsigned)wg);
  return true;
}

hipError_t launch_act8_save(int dtype, int rows, int cols, const void* x, uint8_t* q, uint8_t* scales, hipStream_t s) {
  long long n;
  dim3 grid;
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidConfiguration;
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
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidConfiguration;
  const bool past = (size_t)rows * cols * (dtype == DT_BF16 ? 2 : 4) >= kStreamBytes;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL((past ? act8_restore_kernel<bf16_t, true> : act8_restore_kernel<bf16_t, false>), grid,
                       dim3(256), 0, s, n, q, scales, (bf16_t*)x);
  else
    hipLaunchKernelGGL((past ? act8_restore_kernel<float, true> : act8_restore_kernel<float, false>), grid,
                       dim3(256), 0, s, n, q, scales, (float*)x);
  return hipGetLastError();
}

hipError_t launch_act8_gelu_bwd(int dtype, int rows, int cols, const void* dg, const uint8_t* q, const uint8_t* scales,
                                void* du, void* g, hipStream_t s) {
  long long n;
  dim3 grid;
  if (!chunk_grid(rows, cols, &n, &grid)) return hipErrorInvalidConfiguration;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(act8_gelu_bwd_kernel<bf16_t>, grid, dim3(256), 0, s, n, (const bf16_t*)dg, q, scales,
                       (bf16_t*)du, (bf16_t*)g);
  else
    hipLaunchKernelGGL(act8_gelu_bwd_kernel<float>, grid, dim3(256), 0, s, n, (const float*)dg, q, scales, (float*)du,
                       (float*)g);
  return hipGetLastError();
}

// How the bf16 weight gradient is cut up: tiles of bm x bn, token splits, and whether X is
// restored to bf16 first.
struct DwPlan {
  int bm, bn, tiles, splits, per_split;
  bool restore;
};

// Restoring X reads and writes it once more (3 bytes a value, and a launch); it saves
// every one of the n_out / bm tiles in its column the conversion, about 6e-10 us a
// product.  Measured, restored and converted: 16384 x 7680 x 1920 (tokens x outputs x
// inputs) 427 and 611 us, 4096 x 2048 x 2048 44.8 and 50.5, 2048 x 4096 x 1024 26.7 and 28.8,
// 512 x 7680 x 1920 29.1 and 30.9; 2048 x 1024 x 1024 19.6 and 17.9, 4096 x 1024 x 1024 24.1
// and 22.7, 333 x 1920 x 640 10.0 and 8.2.  Near the border the rule does not know how the
// product will be cut up, and takes the slower side of 16384 x 1304 x 2080 (restored, 153 and
// 137), 32768 x 2048 x 512 (restored, 105 and 96) and 16384 x 1024 x 8192 (converted, 292 and 314).
static bool dw_restore(double tokens, double n_out, double n_in) {
  return 6e-10 * tokens * n_out * n_in > 2.5 + 6.7e-7 * tokens * n_in;
}

// Tile and splits by estimated time: whole rounds of workgroups over the chip, each as
// long as its stages (and about four more for its start and end); splits add their
// sums' way through memory and a launch.  us a stage, measured: 256 x 256 1.6, 256 x 192
// 1.0 to 1.3 (one workgroup a CU); 128 x 128 0.6 alone on its CU, 0.95 for two; converting adds
// a seventh.  What it decides, with the other choice's time: 8192 x 6400 x 1600 256 x 192
// 184 us, 256 x 256 188, 128 x 128 212; 16384 x 7680 x 1920 256 x 256 428, 128 x 128 514,
// 256 x 192 541; 4096 x 2048 x 2048 128 x 128 in one split 48, in two 52.
static DwPlan dw_plan(int tokens, int n_out, int n_in) {
  struct Tile {
    int bm, bn, resident;
    double alone, full;
  };
  static const Tile tiles[] = {{128, 128, 2, 0.6, 0.92}, {256, 256, 1, 1.6, 1.6}, {256, 192, 1, 1.16, 1.16}};
  DwPlan best{};
  best.restore = dw_restore(tokens, n_out, n_in);
  const int stages = (tokens + kBK - 1) / kBK;
  double least = 0.0;
  for (const Tile& t : tiles) {
    if (t.bm != 128 && !best.restore) continue;  // converting, only 128 x 128 is ever the fastest
    const long long n = (long long)((n_out + t.bm - 1) / t.bm) * ((n_in + t.bn - 1) / t.bn);
    for (int want = 1; want == 1 || (want <= 512 && want <= stages / 2 && want * n <= 1024);
         want = want < 4 ? want + 1 : want * 4 / 3) {
      const int per = (stages + want - 1) / want, splits = (stages + per - 1) / per;
      const long long wg = n * splits, slots = 256LL * t.resident;
      const double us = (double)((wg + slots - 1) / slots) * (per + 4) * (wg <= 256 ? t.alone : t.full) *
                            (best.restore ? 1.0 : 8.0 / 7.0) +
                        (splits > 1 ? 5.0 + splits * (double)n_out * n_in * 8.0 / 7e6 : 0.0);
      if (best.bm == 0 || us < least) {
        least = us;
        best.bm = t.bm;
        best.bn = t.bn;
        best.tiles = (int)n;
        best.splits = splits;
        best.per_split = per * kBK;
      }
    }
  }
  return best;
}

// fp32: 128 x 128 tiles for products of at least 2^14 of their stages, else 64 x 64; and splits
// of at least eight stages where the tiles alone would leave CUs without work (32768 x
// 512 x 512: 2.3 ms in one split, 0.16 in 64).
static DwPlan dw_plan_f32(int tokens, int n_out, int n_in) {
  DwPlan p{};
  auto tiles = [&](long long t) { return (n_out + t - 1) / t * ((n_in + t - 1) / t); };
  const int stages = (tokens + kStageF32 - 1) / kStageF32;
  p.bm = p.bn = tiles(128) * stages >= 1 << 14 ? 128 : 64;
  p.tiles = (int)tiles(p.bm);
  const int want = std::max(1, std::min(1024 / p.tiles, stages / 8));
  const int per = (stages + want - 1) / want;
  p.splits = (stages + per - 1) / per;
  p.per_split = per * kStageF32;
  return p;
}

static DwPlan dw_plan_of(int dtype, int tokens, int n_out, int n_in) {
  return dtype == DT_BF16 ? dw_plan(tokens, n_out, n_in) : dw_plan_f32(tokens, n_out, n_in);
}

// Scratch: X's values (if they are restored), the splits' sums (if there are several).
static size_t dw_values_bytes(const DwPlan& p, int tokens, int n_in) {
  return p.restore ? ((size_t)tokens * n_in * 2 + 255) / 256 * 256 : 0;
}

size_t act8_gemm_dw_scratch_bytes(int dtype, int tokens, int n_out, int n_in) {
  const DwPlan p = dw_plan_of(dtype, tokens, n_out, n_in);
  return dw_values_bytes(p, tokens, n_in) + (p.splits > 1 ? (size_t)p.splits * n_out * n_in * sizeof(float) : 0);
}

template <int BM, int BN, int WM, int WN, bool CODES, int H>
static hipError_t run_dw(const DwArgs& a, int splits, hipStream_t s) {
  constexpr size_t lds = 2 * H * (BM + BN) * 128;
  static_assert(lds <= 160 * 1024, "LDS budget");
  auto kern = act8_dw_kernel<BM, BN, WM, WN, CODES, H>;
  static std::atomic<uint64_t> lds_set{0};
  const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kern), lds, lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.tiles * splits)), dim3(WM * WN * 64), lds, s, a);
  return hipGetLastError();
}

static hipError_t run_dw_plan(const DwPlan& p, const DwArgs& a, hipStream_t s) {
  if (p.bm == 128) {
    const bool alone = (long long)p.tiles * p.splits <= 256, longer = p.per_split >= 8 * kBK;
    if (p.restore)  // (alone, it has more than eight kBK: dw_restore)
      return alone ? run_dw<128, 128, 2, 4, false, 2>(a, p.splits, s)
                   : run_dw<128, 128, 2, 2, false, 1>(a, p.splits, s);
    if (!alone) return run_dw<128, 128, 2, 2, true, 1>(a, p.splits, s);
    return longer ? run_dw<128, 128, 2, 4, true, 2>(a, p.splits, s) : run_dw<128, 128, 2, 4, true, 1>(a, p.splits, s);
  }
  if (p.bn == 192) return run_dw<256, 192, 4, 2, false, 1>(a, p.splits, s);
  return run_dw<256, 256, 2, 4, false, 1>(a, p.splits, s);
}

hipError_t launch_act8_gemm_dw(int dtype, int tokens, int n_out, int n_in, const void* dy, const uint8_t* q,
                               const uint8_t* scales, float* dw, int accumulate, void* scratch, hipStream_t s) {
  const DwPlan p = dw_plan_of(dtype, tokens, n_out, n_in);
  if ((long long)p.tiles * p.splits > max_groups(512)) return hipErrorInvalidConfiguration;
  const bool split = p.splits > 1;
  bf16_t* values = (bf16_t*)scratch;
  float* sums = (float*)((char*)scratch + dw_values_bytes(p, tokens, n_in));
  if (p.restore) {
    const hipError_t e = launch_act8_restore(dtype, tokens, n_in, q, scales, values, s);
    if (e != hipSuccess) return e;
  }
  const DwArgs a{tokens, n_out, n_in, p.per_split, p.tiles, split ? 0 : accumulate, (const bf16_t*)dy, q, scales,
                 values, split ? sums : dw};
  hipError_t e;
  if (dtype == DT_BF16) {
    e = run_dw_plan(p, a, s);
  } else {
    hipLaunchKernelGGL((p.bm == 128 ? act8_dw_f32_kernel<2> : act8_dw_f32_kernel<1>),
                       dim3((unsigned)(p.tiles * p.splits)), dim3(256), 0, s, a, (const float*)dy);
    e = hipGetLastError();
  }
  if (e != hipSuccess || !split) return e;
  return launch_dw_join((long long)n_out * n_in, p.splits, sums, dw, accumulate, s);
}

}  // namespace merak
