// Operand tiles of the bf16 MFMA GEMMs: global -> LDS loads, fragment reads and the
// workgroup order (the LDS layouts are described at the kernel in gemm.hip).
#pragma once

#include "common.h"
#include "gemm_tiles.h"

namespace merak {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
#define MERAK_LDS __attribute__((address_space(3)))

__device__ __forceinline__ __amdgpu_buffer_rsrc_t operand_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}

// Workgroup id -> tile id such that each of the 8 XCDs (which receive
// workgroups round-robin) works on one contiguous range of tiles.
__device__ __forceinline__ int xcd_remap(int bid, int n) {
  const int per = n >> 3, rem = n & 7, x = bid & 7, idx = bid >> 3;
  return (x < rem ? x * (per + 1) : rem * (per + 1) + (x - rem) * per) + idx;
}

// One 16-byte-per-lane global -> LDS load: lane i writes LDS bytes
// [lds_addr + 16 i, lds_addr + 16 i + 16).  Issued as inline assembly: the
// compiler would otherwise treat every later LDS read that it cannot prove
// disjoint from this store (the transposing reads among them) as dependent on
// it and wait for all outstanding loads before that read, which would serialise
// the prefetch of the next K stage with the MFMAs of the current one.  The
// kernels order these loads themselves (wait_vm_barrier).  An M0 write needs
// one wait state before an LDS-DMA load.
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4_t operand_rsrc_words(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return i32x4_t{(int32_t)(uint32_t)a, (int32_t)(uint32_t)((a >> 32) & 0xffffu), (int32_t)bytes, 0x00020000};
}

__device__ __forceinline__ void lds_dma16(i32x4_t rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_addr)
               : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(const MERAK_LDS char*)p;
}

// Global -> LDS loader of one operand.  Each wave issues kInst 16-byte-per-lane
// loads per K stage.
template <bool TRANS, int R, int NW>
struct TileLoader {
  static constexpr int kInst = R / 8 / NW;
  static_assert(R / 8 % NW == 0, "tile rows must split evenly over the waves");
  static_assert(!TRANS || (R % 32 == 0 && R >= 128), "MN-contiguous tiles: width a multiple of 32, at least 128");
  uint32_t voff[kInst];
  uint32_t step;  // bytes to advance per K stage

  __device__ __forceinline__ void init(int r0, int ld, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      if constexpr (!TRANS) {
        const int row = (q * NW + wave) * 8 + (lane >> 3);
        const int chunk = (lane & 7) ^ ((row >> 1) & 7);
        voff[q] = (uint32_t)((r0 + row) * ld + chunk * 8) * 2u;
      } else {
        constexpr int CPR = R / 8;  // 16-byte chunks per k-row
        const int g = (q * NW + wave) * 64 + lane;  // chunk index within the stage
        const int kr = g / CPR, slot = g % CPR;
        const int chunk = (slot + CPR - 4 * (kr & 3)) % CPR;  // chunk stored in this slot
        voff[q] = (uint32_t)(kr * ld + r0 + chunk * 8) * 2u;
      }
    }
    step = TRANS ? (uint32_t)(kBK * ld * 2) : (uint32_t)(kBK * 2);
  }

  // Issue load q of the current K stage into `lds` (R * 128 bytes); after the
  // last one (q = kInst - 1) the loader moves on to the next stage.
  __device__ __forceinline__ void issue_one(i32x4_t rsrc, char* lds, int wave, int q) {
    const uint32_t addr = __builtin_amdgcn_readfirstlane(lds_address(lds) + (q * NW + wave) * 1024);
    lds_dma16(rsrc, addr, voff[q]);
    voff[q] += step;
  }

  // Issue the loads of the current K stage into `lds` (R * 128 bytes) and move
  // on to the next stage.
  __device__ __forceinline__ void issue(i32x4_t rsrc, char* lds, int wave) {
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const uint32_t addr = __builtin_amdgcn_readfirstlane(lds_address(lds) + (q * NW + wave) * 1024);
      lds_dma16(rsrc, addr, voff[q]);
      voff[q] += step;
    }
  }
};

// Fragment reader: the 32 x 16 (rows x k) MFMA operand block starting at tile
// row `row0` (a multiple of 32) and k = 16 * ks of an LDS stage.  Lane l gets
// row row0 + l % 32 and k = 16 ks + 8 (l / 32) + 0..7.
template <bool TRANS, int R>
struct FragReader {
  static constexpr int kInstPerFrag = TRANS ? 2 : 1;  // LDS read instructions per fragment
  int lane_off;  // lane-dependent part of the byte offset
  int key;       // lane-dependent swizzle term

  __device__ __forceinline__ void init(int lane) {
    if constexpr (!TRANS) {
      lane_off = (lane & 31) * 128;
      key = (lane >> 5) ^ (((lane & 31) >> 1) & 7);
    } else {
      const int b = lane >> 4, j = lane & 15;
      lane_off = ((b >> 1) * 8 + (j >> 2)) * (2 * R) + ((b & 1) * 2 + ((j >> 1) & 1)) * 16 + (j & 1) * 8;
      key = (j >> 2) << 2;  // slot rotation of this lane's k-row (k & 3 = j / 4)
    }
  }

  __device__ __forceinline__ bf16x8_t read(const char* lds, int row0, int ks) const {
    if constexpr (!TRANS) {
      const char* p = lds + row0 * 128 + lane_off + (((2 * ks) ^ key) << 4);
      return *reinterpret_cast<const bf16x8_t*>(p);
    } else {
      constexpr int CPR = R / 8;
      const char* p = lds + ks * 16 * (2 * R) + ((((row0 >> 3) + key) % CPR) << 4) + lane_off;
      s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MERAK_LDS s16x4_t*)(p));
      s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MERAK_LDS s16x4_t*)(p + 4 * (2 * R)));
      s16x4_t v01 = lo, v23 = hi;
      typedef short s16x8_t __attribute__((ext_vector_type(8)));
      s16x8_t v = {v01[0], v01[1], v01[2], v01[3], v23[0], v23[1], v23[2], v23[3]};
      return __builtin_bit_cast(bf16x8_t, v);
    }
  }
};

// Wait until at most N of this wave's vector-memory loads are outstanding and
// all its LDS reads have completed, then join the workgroup barrier.  (The
// buffer loads that write LDS directly are tracked by vmcnt only.)
template <int N>
__device__ __forceinline__ void wait_vm_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

}  // namespace merak
