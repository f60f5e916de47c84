// What the tiled products share: loads into LDS, waits, and the order of output tiles.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ufp4 {

// 16 bytes per lane from global memory into LDS: lane i reads sbase + voff_i, its bytes land at lds_base + 16 i. Inline
// assembly, so that the compiler does not make LDS reads wait for it; the kernel orders it itself.
__device__ __forceinline__ void to_lds16(uint32_t voff, const void* sbase, const void* lds_base) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t) reinterpret_cast<uintptr_t>(lds_base));
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(m0) : "memory");
}

// Waits until at most N vector-memory operations are outstanding and no LDS operation is (gfx9's s_waitcnt immediate).
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}

// A value that every lane has, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Place L in the launch order -> output tile. Workgroups go to the 8 XCDs round robin, and each XCD has its own L2: the first
// 8 floor(T / 8) are renumbered so that XCD k gets one run of T / 8 tiles, in bands of kBand tile rows, column by column
// within a band. (A grid holds fewer than 2^24 tiles.)
constexpr uint32_t kBand = 8;
__device__ __forceinline__ void tile_at(uint32_t L, uint32_t gy, uint32_t gx, int& tm, int& tn) {
    const uint32_t T = gx * gy, per = T / 8;
    const uint32_t t = L < 8 * per ? (L % 8) * per + L / 8 : L;
    const uint32_t band = t / (kBand * gx), first = band * kBand;
    const uint32_t rows = gy - first < kBand ? gy - first : kBand;
    const uint32_t r = t - first * gx;
    tm = (int)(first + r % rows);
    tn = (int)(r / rows);
}

}  // namespace ufp4
