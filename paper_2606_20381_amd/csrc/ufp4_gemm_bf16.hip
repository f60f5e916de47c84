// Products of bf16 rows that lie group by group (an MoE layer's experts), W as it is stored:
//   fwd_y   Y_g [m_g, N]  = X_g [m_g, K] W_g [N, K]^T
//   bwd_dx  dX_g [m_g, K] = dY_g [m_g, N] W_g [N, K]
//   bwd_dw  dW_g [N, K]   = dY_g [m_g, N]^T X_g [m_g, K], X also as an 8-bit checkpoint
// by v_mfma_f32_32x32x16_bf16, sums in fp32.
//
// A lane of the instruction holds 8 consecutive places of the reduction of one row: 16 bytes. An operand whose memory runs along
// the reduction (X, dY and W of the forward pass) is one LDS read; of one whose memory runs across it (W of bwd_dx, both of
// bwd_dw) the LDS keeps the rows as they lie in memory and ds_read_b64_tr_b16 transposes four of them at a time on the way to the
// registers, so no tensor is transposed in memory.

#include "ufp4_internal.h"
#include "ufp4_ckpt8.h"
#include "ufp4_rows.h"
#include "ufp4_tiles.h"

#include <type_traits>

namespace ufp4 {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

#define INLINE __attribute__((always_inline))

constexpr int kStageK = 32;  // of the reduction per stage: two matrix instructions

// One stage of an operand in LDS: ROWS x kStageK values.
//   along the reduction: row r has 64 bytes, its 16-byte piece p (8 places of the reduction) at piece p ^ f(r);
//   across it: place k of the reduction has 2 ROWS bytes, their 32-byte segment s (16 rows) at segment s ^ f(k).
// Both f make what the lanes of one read touch at a time lie in different banks, whether 128 or 256 bytes are served together.
template <int ROWS, bool ACROSS>
struct Stage {
    static constexpr uint32_t kSize = ROWS * kStageK * 2;
    static constexpr int kPieces = ROWS * kStageK / 8;  // 16 bytes each
    static_assert(ROWS >= 128 || !ACROSS, "eight segments to choose from");
    static __device__ __forceinline__ uint32_t turn_row(uint32_t r) { return ((r >> 1 ^ r >> 3) & 1) | (r >> 1 & 2); }
    static __device__ __forceinline__ uint32_t turn_k(uint32_t k) { return (k & 3) | (k >> 1 & 4); }

    // Byte address of the piece of row r with places 8 p .. of the reduction.
    static __device__ __forceinline__ uint32_t along(uint32_t r, uint32_t p) { return r * 64 + (p ^ turn_row(r)) * 16; }
    // Byte address of rows 8 s .. + 7 at place k.
    static __device__ __forceinline__ uint32_t across(uint32_t k, uint32_t s) {
        return k * (ROWS * 2) + ((s >> 1 ^ turn_k(k)) * 2 + (s & 1)) * 16;
    }

    // The operand of 32 rows from row0 at places 16 ks .. + 15: lane l has row l % 32 and places 8 (l / 32) .. of those.
    static __device__ __forceinline__ v8b read(const uint8_t* stage, uint32_t row0, uint32_t ks) {
        const uint32_t lane = threadIdx.x & 63;
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const v8b*>(stage + along(row0 + (lane & 31), ks * 2 + (lane >> 5)));
        } else {
            // Each 16 lanes read four places of 16 rows, a lane 8 bytes, and get their transpose: lane t row t, four places.
            const uint32_t k = ks * 16 + (lane >> 5) * 8 + (lane >> 2 & 3), r = row0 + (lane & 16) + (lane & 3) * 4;
            typedef __attribute__((address_space(3))) v4s* LdsPtr;
            const uint8_t* const p = stage + across(k, r >> 3) + (r & 4) * 2;
            // four places on: the same segments, since turn_k does not look at bit 2
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(__attribute__((address_space(3))) void*)p);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(__attribute__((address_space(3))) void*)(p + 4 * ROWS * 2));
            return __builtin_bit_cast(v8b, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

__device__ __forceinline__ int64_t clamped(int64_t v, int64_t most) { return v < 0 ? 0 : v < most ? v : most; }

// Ragged rows: each group's first token (clamped to the tensor) and first tile row, in LDS, built by the first wave, 64 groups
// at a time. Offsets that do not rise can claim more tiles than the grid has; what they claim past it is not computed.
template <int BM>
struct GroupRows {
    static constexpr int kN = kBf16Groups + 1;
    int start[kN], rows[kN], tile[kN];

    __device__ __forceinline__ void build(const Bf16GemmJob& j) {
        const int G = j.G, lane = threadIdx.x & 63;
        int64_t tiles = 0;
        auto cut = [](int64_t v) { return v > INT32_MAX ? INT32_MAX : (int)v; };
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + lane;
            const int64_t from = g < G ? clamped(j.offsets[g], j.tokens) : 0, to = g < G ? clamped(j.offsets[g + 1], j.tokens) : 0;
            const int m = to > from ? (int)(to - from) : 0;
            const int cnt = (int)(((int64_t)m + BM - 1) / BM);
            int inc = cnt;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int v = __shfl_up(inc, d, 64);
                if (lane >= d) inc += v;
            }
            if (g < G) {
                start[g] = (int)from;
                rows[g] = m;
                tile[g] = cut(tiles + (inc - cnt));
            }
            tiles += __shfl(inc, 63, 64);
        }
        if (lane == 0) tile[G] = cut(tiles);
    }
    // The group that holds tile row t: the last one whose first tile row is at most t (empty groups share their successor's).
    __device__ __forceinline__ int of(int G, int t) const {
        int n = 0;
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + (threadIdx.x & 63);
            n += __popcll(__ballot(g < G && tile[g] <= t));
        }
        return n - 1;
    }
};

// What a pass reads: operand A's rows are the output's, B's its columns.
template <int PASS>
struct Pass {
    static constexpr bool kRagged = PASS != kBf16BwdDw;      // ragged rows; else a ragged reduction
    static constexpr bool kAcrossA = PASS == kBf16BwdDw, kAcrossB = PASS != kBf16FwdY;
};

// ------------------------------------------------------------------------------------------------
// Any size, stride and alignment: pieces go through registers, where what lies outside is zeroed.
// ------------------------------------------------------------------------------------------------
constexpr int kAnyTile = 128, kAnyThreads = 256;

template <int OUT, int PASS, bool SAVED>
__global__ __launch_bounds__(kAnyThreads, 2) void gemm_bf16_any_kernel(Bf16GemmJob j) {
    using P = Pass<PASS>;
    constexpr int BM = kAnyTile, BN = kAnyTile;
    using SA = Stage<BM, P::kAcrossA>;
    using SB = Stage<BN, P::kAcrossB>;
    constexpr uint32_t kSlot = SA::kSize + SB::kSize;
    __shared__ __align__(16) uint8_t ring[2 * kSlot];
    __shared__ typename std::conditional<P::kRagged, GroupRows<BM>, int>::type groups;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5, l32 = lane & 31;

    // This workgroup's tile: rows of A and B from row0 / col0, reduction [k0, k1).
    const uint32_t gx = (uint32_t)((j.N + BN - 1) / BN);
    int tm, tn;
    int64_t row0, rows, k0 = 0, k1 = j.red, c_base = 0;  // first row of the output, rows from there on
    const uint16_t* a = j.a;
    const uint16_t* b = j.b;
    if constexpr (P::kRagged) {
        if (tid < 64) groups.build(j);
        __syncthreads();
        const uint32_t gy = (uint32_t)uniform(groups.tile[j.G]);
        if (blockIdx.x >= (uint64_t)gx * gy) return;
        tile_at(blockIdx.x, gy, gx, tm, tn);
        const int g = groups.of(j.G, tm), lt = tm - uniform(groups.tile[g]);
        row0 = (int64_t)uniform(groups.start[g]) + (int64_t)lt * BM;
        rows = uniform(groups.rows[g]) - (int64_t)lt * BM;
        b += g * (PASS == kBf16FwdY ? j.N : j.red) * j.ldb;
    } else {
        const uint32_t gy = (uint32_t)((j.M + BM - 1) / BM), per = gx * gy, g = blockIdx.x / per;
        tile_at(blockIdx.x - g * per, gy, gx, tm, tn);
        row0 = (int64_t)tm * BM;
        rows = j.M - row0;
        k0 = clamped(j.offsets[g], j.tokens);
        k1 = clamped(j.offsets[g + 1], j.tokens);
        c_base = (int64_t)g * j.M * j.ldc;
    }
    const int64_t col0 = (int64_t)tn * BN, cols = j.N - col0;

    // Piece q of this thread: 16 bytes of operand A (B) of the stage from place k on; zero outside.
    constexpr int kEach = SA::kPieces / kAnyThreads;
    static_assert(SA::kPieces == SB::kPieces, "");
    auto fetch = [&](const uint16_t* p, int64_t ld, bool across, int64_t first, int64_t have, int64_t k, int q) INLINE {
        const int i = q * kAnyThreads + tid;
        u32x4_any zero = {0, 0, 0, 0};
        if (across) {  // place k + i / (rows / 8), rows 8 (i % (rows / 8)) ..
            const int64_t kk = k + i / (BM / 8), r = (i % (BM / 8)) * 8;
            return kk < k1 && r < have ? Piece<uint16_t>::load(p + kk * ld + first + r, have - r) : zero;
        }
        const int64_t r = i / 4, kk = k + (i % 4) * 8;
        return r < have && kk < k1 ? Piece<uint16_t>::load(p + (first + r) * ld + kk, k1 - kk) : zero;
    };
    auto place = [&](bool across, int q) INLINE {
        const uint32_t i = q * kAnyThreads + tid;
        return across ? SA::across(i / (BM / 8), i % (BM / 8)) : SA::along(i / 4, i % 4);
    };
    // A checkpoint's 16 codes: place k + i / 8, columns 16 (i % 8) ..
    auto fetch_saved = [&](int64_t k, u32x4_any& codes, uint32_t& scale) INLINE {
        const int64_t kk = k + tid / 8, c = (tid % 8) * 16;
        codes = u32x4_any{0, 0, 0, 0};
        scale = 127;
        if (kk < k1 && c < cols) {
            codes = *reinterpret_cast<const u32x4_any*>(j.b8 + kk * j.ldb + col0 + c);  // rows hold whole blocks
            scale = j.bs[kk * j.ldbs + ((col0 + c) >> 5)];
        }
    };

    v16f acc[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.0f;

    u32x4_any ra[kEach], rb[kEach];
    uint32_t scale = 127;
    auto load = [&](int64_t k) INLINE {
#pragma unroll
        for (int q = 0; q < kEach; ++q) ra[q] = fetch(a, j.lda, P::kAcrossA, row0, rows, k, q);
        if constexpr (SAVED) {
            fetch_saved(k, rb[0], scale);
        } else {
#pragma unroll
            for (int q = 0; q < kEach; ++q) rb[q] = fetch(b, j.ldb, P::kAcrossB, col0, cols, k, q);
        }
    };
    if (k0 < k1) load(k0);
    uint32_t slot = 0;
    for (int64_t k = k0; k < k1; k += kStageK) {
        uint8_t* const sa = ring + slot;
        uint8_t* const sb = sa + SA::kSize;
#pragma unroll
        for (int q = 0; q < kEach; ++q) *reinterpret_cast<u32x4_any*>(sa + place(P::kAcrossA, q)) = ra[q];
        if constexpr (SAVED) {
            u32x4_any lo, hi;
            ckpt8_to_bf16(rb[0], scale, lo, hi);
            *reinterpret_cast<u32x4_any*>(sb + SB::across(tid / 8, (tid % 8) * 2)) = lo;
            *reinterpret_cast<u32x4_any*>(sb + SB::across(tid / 8, (tid % 8) * 2 + 1)) = hi;
        } else {
#pragma unroll
            for (int q = 0; q < kEach; ++q) *reinterpret_cast<u32x4_any*>(sb + place(P::kAcrossB, q)) = rb[q];
        }
        __syncthreads();  // two slots: the next stage is written to the other one, which everyone has read
        if (k + kStageK < k1) load(k + kStageK);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            v8b fa[2], fb[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                fa[t] = SA::read(sa, wm * 64 + t * 32, ks);
                fb[t] = SB::read(sb, wn * 64 + t * 32, ks);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[y], fa[x], acc[x][y], 0, 0, 0);
        }
        slot ^= kSlot;
    }

    // B's rows are the instruction's rows: a lane holds columns 8 q + 4 h .. + 3 of row l32 of each tile.
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int64_t r = wm * 64 + x * 32 + l32;
        if (r >= rows) continue;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t c = wn * 64 + y * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
                if (c >= cols) continue;
                const int64_t at = c_base + (row0 + r) * j.ldc + col0 + c;
                if constexpr (OUT == kOutF32) static_cast<float*>(j.c)[at] = acc[x][y][i];
                else static_cast<uint16_t*>(j.c)[at] = __builtin_bit_cast(uint16_t, (__bf16)acc[x][y][i]);
            }
    }
}

// Tile rows that a launch provides for; ragged rows: every group may end in a partial tile.
int64_t tile_rows(const Bf16GemmJob& j, int bm) {
    return j.pass != kBf16BwdDw ? (j.tokens + bm - 1) / bm + j.G : (j.M + bm - 1) / bm;
}
int64_t grid_tiles(const Bf16GemmJob& j, int bm, int bn) {
    return tile_rows(j, bm) * ((j.N + bn - 1) / bn) * (j.pass == kBf16BwdDw ? j.G : 1);
}

template <int OUT>
hipError_t launch_out(const Bf16GemmJob& j, hipStream_t s) {
    const int64_t tiles = grid_tiles(j, kAnyTile, kAnyTile);
    if (tiles == 0) return hipSuccess;
    const unsigned n = (unsigned)tiles;
    switch (j.pass) {
        case kBf16FwdY: gemm_bf16_any_kernel<OUT, kBf16FwdY, false><<<n, kAnyThreads, 0, s>>>(j); break;
        case kBf16BwdDx: gemm_bf16_any_kernel<OUT, kBf16BwdDx, false><<<n, kAnyThreads, 0, s>>>(j); break;
        default:
            if (j.b8) gemm_bf16_any_kernel<OUT, kBf16BwdDw, true><<<n, kAnyThreads, 0, s>>>(j);
            else gemm_bf16_any_kernel<OUT, kBf16BwdDw, false><<<n, kAnyThreads, 0, s>>>(j);
    }
    return hipGetLastError();
}

}  // namespace

bool bf16_gemm_fits(const Bf16GemmJob& j) { return grid_tiles(j, kAnyTile, kAnyTile) < int64_t(1) << 24; }

hipError_t launch_gemm_bf16(const Bf16GemmJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_out<kOutBF16>(j, s) : launch_out<kOutF32>(j, s);
}

}  // namespace ufp4
