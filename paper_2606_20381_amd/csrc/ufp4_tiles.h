// What the tiled products share: loads into LDS, waits, and the order of output tiles.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ufp4_internal.h"
#include "ufp4_rows.h"

namespace ufp4 {

// 16 bytes per lane from global memory into LDS: lane i reads sbase + voff_i, its bytes land at lds_base + 16 i. Inline
// assembly, so that the compiler does not make LDS reads wait for it; the kernel orders it itself.
__device__ __forceinline__ void to_lds16(uint32_t voff, const void* sbase, const void* lds_base) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t) reinterpret_cast<uintptr_t>(lds_base));
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(m0) : "memory");
}

// The same with 4 bytes per lane, landing at lds_base + 4 i.
__device__ __forceinline__ void to_lds4(uint32_t voff, const void* sbase, const void* lds_base) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t) reinterpret_cast<uintptr_t>(lds_base));
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "s"(m0) : "memory");
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

typedef float v16f __attribute__((ext_vector_type(16)));

template <int OUT, int WTM, int WTN>
struct Stored {
    static constexpr int kElems = OUT == kOutF32 ? 4 : 8;  // of a 16-byte store
    static constexpr int kStores = WTM * WTN * 32 / kElems / 2;
};

// A lane holds columns 8q + 4h .. + 3 (q < 4) of row l32 of each 32 x 32 tile. Lanes trade until a store of 16 bytes a lane
// writes whole 128-byte lines (8 rows of them; pieces of 32 or 64 bytes cost the memory system up to 1.6 times as long):
//   bf16: the halves of the wave, so that a lane has eight consecutive columns; then the 16-lane rows of the wave (16 rows x
//   64 bytes), then the 8-lane halves of those with the neighbouring tile; fp32: the same without the first step, the
//   neighbour being the tile's other 16 columns. Stored::kStores stores a wave for a tile inside the output.
// The tile begins at row row0 and column col0 of the output at c + base (elements), rows ldc apart and N wide; wave (wm, wn) holds its
// WTM x WTN part; `rows` of it are inside the output (INSIDE: all rows and columns). STREAM: nontemporally.
template <int OUT, int WTM, int WTN, bool STREAM, bool INSIDE>
__device__ __forceinline__ void store_tile(const v16f (&acc)[WTM][WTN], void* c, int64_t base, int row0, int col0, int64_t ldc, int rows, int64_t N,
                                           int wm, int wn) {
    constexpr int kElems = Stored<OUT, WTM, WTN>::kElems;
    constexpr bool kLine = OUT == kOutF32 || WTN % 2 == 0;  // a lone bf16 tile stays at 64 bytes
    const int lane = threadIdx.x & 63;
    // one store: v, at row lr and column col of the tile; at the output's right edge the pieces that are inside are still whole
    auto put = [&](const uint32_t (&v)[4], int lr, int col) __attribute__((always_inline)) {
        const int64_t off = base + (int64_t)(row0 + lr) * ldc + col0 + col;
        const int64_t left = N - col0 - col;  // columns from this lane's first
        if (INSIDE || (lr < rows && left >= kElems)) {
            const u32x4_any x = {v[0], v[1], v[2], v[3]};
            u32x4_any* const to = reinterpret_cast<u32x4_any*>(static_cast<uint8_t*>(c) + off * (OUT == kOutF32 ? 4 : 2));
            if constexpr (STREAM) __builtin_nontemporal_store(x, to);
            else *to = x;
        } else if (lr < rows) {
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
                if (e >= left) continue;
                if constexpr (OUT == kOutF32) static_cast<float*>(c)[off + e] = __uint_as_float(v[e]);
                else static_cast<uint16_t*>(c)[off + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
            }
        }
    };
    // 16 rows x 64 bytes: u = 0, 1 the tile's rows 16u ..; the wave's 16-lane rows hold the pieces 0, 2, 1, 3 of the 64 bytes
    // (fp32: half `part` of the tile's columns)
    auto quarter = [&](const v16f& c, int part, uint32_t (&v)[2][4]) __attribute__((always_inline)) {
        uint32_t x[4], y[4];
        if constexpr (OUT == kOutF32) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[t] = __float_as_uint(c[8 * part + t]);
                y[t] = __float_as_uint(c[8 * part + 4 + t]);
            }
        } else {
            auto pair = [&](int i) __attribute__((always_inline)) {
                return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)c[i]) |
                       (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)c[i + 1]) << 16;
            };
            const auto e = __builtin_amdgcn_permlane32_swap(pair(0), pair(4), false, false);
            const auto f = __builtin_amdgcn_permlane32_swap(pair(2), pair(6), false, false);
            const auto g = __builtin_amdgcn_permlane32_swap(pair(8), pair(12), false, false);
            const auto k = __builtin_amdgcn_permlane32_swap(pair(10), pair(14), false, false);
            x[0] = e[0], x[1] = f[0], x[2] = e[1], x[3] = f[1];
            y[0] = g[0], y[1] = k[0], y[2] = g[1], y[3] = k[1];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const auto r = __builtin_amdgcn_permlane16_swap(x[t], y[t], false, false);
            v[0][t] = r[0];
            v[1][t] = r[1];
        }
    };
    const int piece = ((lane >> 4) & 1) * 2 + (lane >> 5);  // of 64 bytes
    constexpr int kSteps = kLine ? (OUT == kOutF32 ? WTN : WTN / 2) : WTN;
#pragma unroll
    for (int a = 0; a < WTM; ++a) {
        const int lr = (wm * WTM + a) * 32;
#pragma unroll
        for (int b = 0; b < kSteps; ++b) {
            uint32_t v[2][4];
            if constexpr (kLine) {
                uint32_t n[2][4];
                if constexpr (OUT == kOutF32) {
                    quarter(acc[a][b], 0, v);
                    quarter(acc[a][b], 1, n);
                } else {
                    quarter(acc[a][2 * b], 0, v);
                    quarter(acc[a][2 * b + 1], 0, n);
                }
                const int col = (wn * WTN + (OUT == kOutF32 ? b : 2 * b)) * 32 + (lane & 8) / 8 * 4 * kElems + piece * kElems;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t lo[4], hi[4];  // rows 0-7 and 8-15 of the sixteen: lanes 8-15 of each sixteen have the neighbour's
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        constexpr int kRor8 = 0x128;  // rotate each sixteen lanes by eight
                        lo[t] = __builtin_amdgcn_update_dpp(v[u][t], n[u][t], kRor8, 0xF, 0xC, false);
                        hi[t] = __builtin_amdgcn_update_dpp(n[u][t], v[u][t], kRor8, 0xF, 0x3, false);
                    }
                    put(lo, lr + u * 16 + (lane & 7), col);
                    put(hi, lr + u * 16 + 8 + (lane & 7), col);
                }
            } else {
                quarter(acc[a][b], 0, v);
#pragma unroll
                for (int u = 0; u < 2; ++u) put(v[u], lr + u * 16 + (lane & 15), (wn * WTN + b) * 32 + piece * kElems);
            }
        }
    }
}

}  // namespace ufp4
