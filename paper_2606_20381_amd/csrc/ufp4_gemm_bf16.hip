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
//
// Four kernels: tiles of 256 x 256 and 128 x 128 fed by direct-to-LDS loads (rows of whole 16-byte pieces), tiles of 128 x 128 through
// registers (any alignment), and one for the few rows of a decode step.
//
// Bound, where the tiles fill the chip, by the matrix cores' power: the instruction alone, on registers, reaches 1.54-1.75 PFLOP/s on random
// numbers (2.3 on zeros: power takes the clock to 1.5-1.7 GHz). 8192^3 takes 0.79-0.87 ms in every pass = 1.26-1.39 (matrix cores busy 78-81%
// of the CUs' busy cycles, at 1.6-1.75 GHz; 0.79 with every load from the same L2-resident place, 0.69 without the loads). 98304 x 1408 x 2048
// of 64 experts with a power law's loads: forward and input's gradient 0.55-0.58 ms = 1.0 PFLOP/s of the products asked for (busy 64%: tiles
// that end outside of a group or of the 1408 columns, W new in every tile row, workgroups that end 12% apart), weights' gradient 0.61-0.65 ms,
// its 738 MB of results alone 0.15.

#include "ufp4_internal.h"
#include "ufp4_ckpt8.h"
#include "ufp4_rows.h"
#include "ufp4_tiles.h"

#include <math.h>

#include <type_traits>

namespace ufp4 {

namespace {

typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

#define INLINE __attribute__((always_inline))

// One stage of an operand in LDS: ROWS x K values, K places of the reduction (16 a matrix instruction).
//   along the reduction: row r has 2 K bytes, its 16-byte piece p (8 places of the reduction) at piece p ^ turn_row(r);
//   across it: place k of the reduction has 2 ROWS bytes, their 32-byte segment s (16 rows) at segment s ^ turn_k(k).
// Both turns make what the lanes of one read touch at a time lie in different banks, whether 128 or 256 bytes are served together
// (measured: no conflict).
template <int ROWS_, int K_, bool ACROSS>
struct Stage {
    static constexpr int ROWS = ROWS_, K = K_;
    static constexpr bool kAcross = ACROSS;
    static constexpr uint32_t kSize = ROWS * K * 2;
    static constexpr uint32_t kRowPieces = K / 8, kPlacePieces = ROWS / 8;
    static __device__ __forceinline__ uint32_t turn_row(uint32_t r) {
        static_assert(K == 32 || K == 64, "");
        return K == 32 ? ((r >> 1 ^ r >> 3) & 1) | (r >> 1 & 2) : (r ^ (r >> 3 & 3)) & 7;
    }
    static __device__ __forceinline__ uint32_t turn_k(uint32_t k) {
        static_assert(ROWS >= 128, "eight segments at least");
        return (k << 1 & 6) | (k >> 1 & 1);
    }

    // Byte address of the piece of row r with places 8 p .. of the reduction.
    static __device__ __forceinline__ uint32_t along(uint32_t r, uint32_t p) { return r * (K * 2) + (p ^ turn_row(r)) * 16; }
    // Byte address of rows 8 s .. + 7 at place k.
    static __device__ __forceinline__ uint32_t across(uint32_t k, uint32_t s) {
        return k * (ROWS * 2) + ((s >> 1 ^ turn_k(k)) * 2 + (s & 1)) * 16;
    }

    // What the i-th 16 bytes of the stage hold: rows from `row` at place `k` (one row and 8 places, or 8 rows and one place).
    static __device__ __forceinline__ void piece(uint32_t i, uint32_t& row, uint32_t& k) {
        if constexpr (ACROSS) {
            k = i / kPlacePieces;
            const uint32_t at = i % kPlacePieces;
            row = ((at >> 1 ^ turn_k(k)) * 2 + (at & 1)) * 8;
        } else {
            row = i / kRowPieces;
            k = (i % kRowPieces ^ turn_row(row)) * 8;
        }
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

// The rows of group g0 + lane, [from, from + m), of ragged rows: its offsets cut to the tensor and, where they fall, to no less than those
// before them (`before`: the largest start of the groups before g0, 0 at first), so that no row has two groups, and groups with rows, or
// their tiles, are never more than a grid for rising offsets holds.
__device__ __forceinline__ void group_rows(const Bf16GemmJob& j, int g0, int& before, int& from, int& m) {
    const int lane = threadIdx.x & 63, g = g0 + lane;
    const int64_t* const at = j.offsets + (g < j.G ? g : j.G - 1);  // both loads at once, without a branch
    from = (int)clamped(at[0], j.tokens);
    int to = (int)clamped(at[1], j.tokens);
    to = g < j.G ? to : from;
    if (__ballot(to < from || from < before)) {
        from = from > before ? from : before;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(from, d, 64);
            if (lane >= d) from = v > from ? v : from;
        }
    }
    m = to > from ? to - from : 0;
    before = __builtin_amdgcn_readlane(from, 63);  // of 64 groups; after fewer nothing follows
}

// Ragged rows: each group's first token and first tile row, in LDS, built by the first wave, 64 groups at a time.
template <int BM>
struct GroupRows {
    static constexpr int kN = kBf16Groups + 1;
    int start[kN], rows[kN], tile[kN];

    __device__ __forceinline__ void build(const Bf16GemmJob& j) {
        const int G = j.G, lane = threadIdx.x & 63;
        int tiles = 0, before = 0;
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + lane;
            int from, m;
            group_rows(j, g0, before, from, m);
            const int cnt = (int)(((int64_t)m + BM - 1) / BM);
            int inc = cnt;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int v = __shfl_up(inc, d, 64);
                if (lane >= d) inc += v;
            }
            if (g < G) {
                start[g] = from;
                rows[g] = m;
                tile[g] = tiles + (inc - cnt);
            }
            tiles += __shfl(inc, 63, 64);
        }
        if (lane == 0) tile[G] = tiles;
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
constexpr int kAnyTile = 128, kAnyThreads = 256, kAnyK = 32;

template <int OUT, int PASS, bool SAVED>
__global__ __launch_bounds__(kAnyThreads, 3) void gemm_bf16_any_kernel(Bf16GemmJob j) {
    using P = Pass<PASS>;
    constexpr int BM = kAnyTile, BN = kAnyTile;
    using SA = Stage<BM, kAnyK, P::kAcrossA>;
    using SB = Stage<BN, kAnyK, P::kAcrossB>;
    constexpr uint32_t kSlot = SA::kSize + SB::kSize;
    __shared__ __align__(16) uint8_t ring[2 * kSlot];
    __shared__ typename std::conditional<P::kRagged, GroupRows<BM>, int>::type groups;
    const int tid = threadIdx.x, wave = uniform(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;

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
        if (blockIdx.x >= gx * gy) return;
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

    // Pieces q of this thread: 16 bytes of operand A (B) of a stage, where they come from at the reduction's first place, and the place in
    // the stage. Rows past the last one are zeros (across the reduction) or the first one again: they only feed outputs that are not
    // stored. A piece that the row's end cuts is loaded from before its place, so that it ends with the row, and moved down on its way to
    // the LDS: loading it value by value would wait for memory in every stage.
    constexpr int kEach = SA::kSize / 16 / kAnyThreads;
    static_assert(SA::kSize == SB::kSize, "");
    struct Source {
        const uint16_t* p;
        int place, have;  // `have` of its 8 rows, across the reduction
    };
    const bool narrow_a = (P::kAcrossA ? j.M : j.red) < 8, narrow_b = (P::kAcrossB ? j.N : j.red) < 8;  // no 8 values before a row's end
    auto source = [&](auto stage, const uint16_t* base, int64_t ld, int64_t first, int64_t rows_have, bool narrow, int q) INLINE {
        using S = decltype(stage);
        uint32_t r, k;
        S::piece((uint32_t)(q * kAnyThreads + tid), r, k);
        Source s;
        s.place = (int)k;
        if constexpr (S::kAcross) {
            const int64_t left = rows_have - r;
            s.have = left < 0 ? 0 : left < 8 ? (int)left : 8;
            s.p = base + (k0 + k) * ld + first + r - (narrow || s.have == 0 ? 0 : 8 - s.have);
        } else {
            s.have = 8;
            s.p = base + (first + (r < rows_have ? r : 0)) * ld + k0 + k;
        }
        return s;
    };
    // Values of the piece that exist at place k of the reduction, where whether a whole stage is left is the same for all.
    auto existing = [&](auto stage, const Source& s, int64_t k) INLINE {
        if (k + kAnyK <= k1) return s.have;
        const int64_t left = k1 - k - s.place;
        if (decltype(stage)::kAcross) return left > 0 ? s.have : 0;
        return left < 0 ? 0 : left < 8 ? (int)left : 8;
    };
    auto fetch = [&](auto stage, const Source& s, int64_t ld, int64_t k, bool narrow) INLINE {
        using S = decltype(stage);
        const uint16_t* const p = s.p + (S::kAcross ? (k - k0) * ld : k - k0);
        const int n = existing(stage, s, k);
        u32x4_any v = {0, 0, 0, 0};
        if (narrow) v = Piece<uint16_t>::load(p, n);
        else if (n > 0) v = *reinterpret_cast<const u32x4_any*>(S::kAcross ? p : p - (8 - n));
        return v;
    };
    auto place_at = [&](auto stage, const Source& s, int64_t k, bool narrow, const u32x4_any& v, uint8_t* to) INLINE {
        const int n = existing(stage, s, k);
        u32x4_any x = v;
        if (n < 8 && !narrow) {  // down by 8 - n values; n 0: zeros already
            const int by = 8 - n;
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = by & 1 ? __builtin_amdgcn_alignbit(w < 3 ? v[w + 1] : 0, v[w], 16) : v[w];
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = by & 2 ? (w < 3 ? x[w + 1] : 0) : x[w];
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = by & 4 ? (w < 2 ? x[w + 2] : 0) : x[w];
        }
        *reinterpret_cast<u32x4_any*>(to) = x;
    };
    // A checkpoint's 16 codes: place k + tid / 8, columns 16 (tid % 8) ..
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

    Source from_a[kEach], from_b[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        from_a[q] = source(SA{}, a, j.lda, row0, rows, narrow_a, q);
        if constexpr (!SAVED) from_b[q] = source(SB{}, b, j.ldb, col0, cols, narrow_b, q);
    }
    // Two stages are on their way in registers (three or four cost the second workgroup of a CU: 8192 x 4099 x 4099 forward 497 us, 505, 581).
    struct Pieces {
        u32x4_any a[kEach], b[kEach];
        uint32_t scale;
    };
    Pieces held[2];
    auto load = [&](Pieces& h, int64_t k) INLINE {
        if (k >= k1) return;
#pragma unroll
        for (int q = 0; q < kEach; ++q) h.a[q] = fetch(SA{}, from_a[q], j.lda, k, narrow_a);
        if constexpr (SAVED) {
            fetch_saved(k, h.b[0], h.scale);
        } else {
#pragma unroll
            for (int q = 0; q < kEach; ++q) h.b[q] = fetch(SB{}, from_b[q], j.ldb, k, narrow_b);
        }
    };
    auto write = [&](const Pieces& h, int64_t k, uint32_t slot) INLINE {
        uint8_t* const sa = ring + slot;
        uint8_t* const sb = sa + SA::kSize;
#pragma unroll
        for (int q = 0; q < kEach; ++q) place_at(SA{}, from_a[q], k, narrow_a, h.a[q], sa + (q * kAnyThreads + tid) * 16);
        if constexpr (SAVED) {
            u32x4_any lo, hi;
            ckpt8_to_bf16(h.b[0], h.scale, lo, hi);
            *reinterpret_cast<u32x4_any*>(sb + SB::across(tid / 8, (tid % 8) * 2)) = lo;
            *reinterpret_cast<u32x4_any*>(sb + SB::across(tid / 8, (tid % 8) * 2 + 1)) = hi;
        } else {
#pragma unroll
            for (int q = 0; q < kEach; ++q) place_at(SB{}, from_b[q], k, narrow_b, h.b[q], sb + (q * kAnyThreads + tid) * 16);
        }
    };
    uint32_t slot = 0;
    auto stage = [&](Pieces& h, int64_t k) INLINE {
        write(h, k, slot);
        __syncthreads();  // two slots: the next stage is written to the other one, which everyone has read
        load(h, k + 2 * kAnyK);
        const uint8_t* const sa = ring + slot;
        const uint8_t* const sb = sa + SA::kSize;
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
    };
    load(held[0], k0);
    load(held[1], k0 + kAnyK);
    for (int64_t k = k0; k < k1; k += 2 * kAnyK) {
        stage(held[0], k);
        if (k + kAnyK < k1) stage(held[1], k + kAnyK);
    }
    store_tile<OUT, 2, 2, false, false>(acc, j.c, c_base, (int)row0, (int)col0, j.ldc, rows < BM ? (int)rows : BM, j.N, wm, wn);
}

// ------------------------------------------------------------------------------------------------
// Rows of whole 16-byte pieces: memory to LDS without registers between.
// ------------------------------------------------------------------------------------------------

// WM x WN waves, each with WTM x WTN matrix tiles of 32 x 32 outputs; RING stages of K places in LDS; PER_CU workgroups on a CU.
template <int WTM_, int WTN_, int WM_, int WN_, int K_, int RING_, int PER_CU>
struct Tile {
    static constexpr int WTM = WTM_, WTN = WTN_, WM = WM_, WN = WN_, K = K_, kRing = RING_;
    static constexpr int BM = 32 * WTM * WM, BN = 32 * WTN * WN;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kResident = 256 * PER_CU;    // workgroups on 256 CUs
    static constexpr int kPerEU = PER_CU * kWaves / 4;  // waves per SIMD that the registers have to allow
    static constexpr int kLoadsA = BM * K / 512 / kWaves, kLoadsB = BN * K / 512 / kWaves;  // 1 KiB loads of a stage, a wave
    static constexpr int kWaveLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * 512 * kWaves == BM * K && kLoadsB * 512 * kWaves == BN * K, "every wave issues the same loads");
    static_assert(kWaveLoads * (kRing - 1) + 32 < 64, "vmcnt has six bits");
};

// Ragged reductions by length, the longest first (of equally long ones the lower group): long tiles that begin last would run alone at
// the end. By every wave for itself.
struct Lengths {
    int start, len;  // of the lane's group among the first 64; the others' are read again each time

    __device__ __forceinline__ static void span(const Bf16GemmJob& j, int g, int& start, int& len) {
        start = 0;
        len = -1;
        if (g >= j.G) return;
        start = (int)clamped(j.offsets[g], j.tokens);
        len = (int)clamped(j.offsets[g + 1], j.tokens) - start;
        if (len < 0) len = 0;
    }
    __device__ __forceinline__ void load(const Bf16GemmJob& j) { span(j, threadIdx.x & 63, start, len); }
    // The group of this rank and its reduction: the length bit by bit, from counts of groups at least as long, then the place among equals.
    __device__ __forceinline__ int ranked(const Bf16GemmJob& j, uint32_t rank, int64_t& from, int64_t& to) const {
        const int lane = threadIdx.x & 63, rounds = (j.G + 63) / 64;
        auto count = [&](int64_t least) {  // groups of at least this length
            int n = __popcll(__ballot(len >= least));
            for (int r = 1; r < rounds; ++r) {
                int s, l;
                span(j, r * 64 + lane, s, l);
                n += __popcll(__ballot(l >= least));
            }
            return (uint32_t)uniform(n);
        };
        int64_t v = 0;  // the largest length that more than `rank` groups reach
        for (int b = 31 - __builtin_clz((uint32_t)j.tokens | 1); b >= 0; --b)
            if (count(v + (int64_t(1) << b)) > rank) v += int64_t(1) << b;
        uint32_t place = rank - count(v + 1);  // among the groups of length v
        for (int r = 0; r < rounds; ++r) {
            int s = start, l = len;
            if (r > 0) span(j, r * 64 + lane, s, l);
            uint64_t same = __ballot(l == v);
            const uint32_t n = (uint32_t)__popcll(same);
            if (place >= n) {
                place -= n;
                continue;
            }
            for (; place > 0; --place) same &= same - 1;
            const int at = uniform(__builtin_ctzll(same));
            from = __builtin_amdgcn_readlane(s, at);
            to = from + v;
            return r * 64 + at;
        }
        from = to = 0;
        return 0;
    }
};

constexpr int kCounterStride = 16;  // of 4 bytes: each XCD's counter has a line of its own

__global__ void clear_counters_kernel(uint32_t* counters) { counters[threadIdx.x] = 0; }

// The pipeline: a ring of stages in LDS, filled by direct-to-LDS loads; each wave keeps two sets of operands in registers: while the
// matrix core works on one step of a stage, the next step's operands (past the barrier, the next stage's first) are read from LDS.
// SAVED (bwd_dw): B is an 8-bit checkpoint. The ring holds its codes and scales; a stage of them becomes bf16, in one of two further slots,
// one stage before it is multiplied, 16 codes of one scale a thread.
template <int OUT, class C, int PASS, bool STREAM, bool SAVED>
__global__ __launch_bounds__(C::kThreads, C::kPerEU) void gemm_bf16_kernel(Bf16GemmJob j) {
    using P = Pass<PASS>;
    constexpr int BM = C::BM, BN = C::BN, WTM = C::WTM, WTN = C::WTN, kRing = C::kRing;
    using SA = Stage<BM, C::K, P::kAcrossA>;
    using SB = Stage<BN, C::K, P::kAcrossB>;
    static_assert(!SAVED || (C::K == 32 && C::kLoadsB == 2 && kRing >= 3), "a wave's two loads are 1 KiB of codes and the scales");
    constexpr uint32_t kCodes = C::K * BN, kScales = 256;  // bytes of a stage of a checkpoint
    constexpr uint32_t kSlot = SA::kSize + (SAVED ? kCodes + kScales : SB::kSize);
    __shared__ __align__(16) uint8_t ring[kRing * kSlot];
    __shared__ __align__(16) uint8_t unpacked[SAVED ? 2 * SB::kSize : 16];
    __shared__ typename std::conditional<P::kRagged, GroupRows<BM>, int>::type groups;
    __shared__ uint32_t s_next;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    // Where a SIMD has two waves of eight (w and w + 4), they differ in both halves of the tile, so that a tile which lies half outside
    // of the output leaves each SIMD one wave with work.
    int wm, wn;
    if constexpr (C::kWaves == 8) {
        static_assert(C::kWaves != 8 || (C::WM == 2 && C::WN == 4), "");
        wm = (wave >> 1 ^ wave >> 2) & 1;
        wn = (wave & 1) | (wave >> 1 & 2);
    } else {
        wm = (int)((unsigned)wave / C::WN);
        wn = (int)((unsigned)wave % C::WN);
    }
    const uint32_t gx = (uint32_t)((j.N + BN - 1) / BN);
    uint32_t gy, total;
    if constexpr (P::kRagged) {
        if (tid < 64) groups.build(j);
        __syncthreads();
        gy = (uint32_t)uniform(groups.tile[j.G]);
        total = gx * gy;
    } else {
        gy = (uint32_t)((j.M + BM - 1) / BM);
        total = gx * gy * (uint32_t)j.G;
    }
    Lengths lengths;
    if constexpr (!P::kRagged) lengths.load(j);

    // One output tile: its operands' places of stage 0, this lane's pieces of a stage, and where the results go. A reduction of no whole
    // stages begins inside stage 0: its first `gap` places are zeroed in LDS (memory is read from the first place on).
    struct Work {
        const uint8_t *a, *b, *s;  // s: a checkpoint's scales
        uint32_t va[C::kLoadsA], vb[C::kLoadsB];
        int nst, gap;
        int row0, rows, col0;
        int64_t c_base;
        bool idle;  // this wave's part is outside of the output: it loads with the others, and multiplies nothing
    };
    const uint32_t stepA = P::kAcrossA ? (uint32_t)(C::K * 2 * j.lda) : C::K * 2, stepB = P::kAcrossB ? (uint32_t)(C::K * (SAVED ? 1 : 2) * j.ldb) : C::K * 2;
    const uint32_t stepS = SAVED ? (uint32_t)(C::K * j.ldbs) : 0;
    // Lane's piece of load q (unit wave * loads + q of the stage: 64 pieces in the LDS's order), as an offset from the operand's first
    // row and place. Rows past the last one are replaced by it: they only feed outputs that are not stored. Places before `gap` (a
    // multiple of 8 along the reduction) are replaced by that one.
    auto offset = [&](auto stage, int unit, int64_t ld, int64_t have, int gap) INLINE {
        using S = decltype(stage);
        uint32_t r, k;
        S::piece((uint32_t)unit * 64 + lane, r, k);
        k = k < (uint32_t)gap ? (uint32_t)gap : k;
        if (S::kAcross) return (k * (uint32_t)ld + (r < have ? r : (uint32_t)have - 8)) * 2;
        return ((r < have ? r : (uint32_t)have - 1) * (uint32_t)ld + k) * 2;
    };
    auto offset_a = [&](const Work& w, int q, int gap) INLINE { return offset(SA{}, wave * C::kLoadsA + q, j.lda, w.rows, gap); };
    auto offset_b = [&](const Work& w, int q, int gap) INLINE {
        if constexpr (!SAVED) {
            return offset(SB{}, wave * C::kLoadsB + q, j.ldb, j.N - w.col0, gap);
        } else {  // 16 codes, or 4 scales; past the last block's the last ones
            constexpr uint32_t kEach = BN / 16, kWords = BN / 128;
            const uint32_t blocks = (uint32_t)((j.N - w.col0 + kCkpt8Block - 1) / kCkpt8Block);
            const uint32_t i = q == 0 ? (uint32_t)wave * 64 + lane : (uint32_t)lane % (C::K * kWords);
            uint32_t k = i / (q == 0 ? kEach : kWords), at = i % (q == 0 ? kEach : kWords);
            k = k < (uint32_t)gap ? (uint32_t)gap : k;
            const uint32_t most = q == 0 ? blocks * 2 : (blocks + 3) / 4;
            at = at < most ? at : most - 1;
            return q == 0 ? k * (uint32_t)j.ldb + at * 16 : k * (uint32_t)j.ldbs + at * 4;
        }
    };
    auto locate = [&](uint32_t L, Work& w) INLINE {
        int tm, tn;
        int64_t k0 = 0, k1 = j.red, row0, rows;
        const uint16_t* b = j.b;
        w.c_base = 0;
        if constexpr (P::kRagged) {
            tile_at(L, gy, gx, tm, tn);
            const int g = groups.of(j.G, tm), lt = tm - uniform(groups.tile[g]);
            row0 = (int64_t)uniform(groups.start[g]) + (int64_t)lt * BM;
            rows = uniform(groups.rows[g]) - (int64_t)lt * BM;
            b += (int64_t)g * (PASS == kBf16FwdY ? j.N : j.red) * j.ldb;
        } else {
            const uint32_t rank = L / (gx * gy);
            const int g = lengths.ranked(j, rank, k0, k1);
            tile_at(L - rank * (gx * gy), gy, gx, tm, tn);
            row0 = (int64_t)tm * BM;
            rows = j.M - row0;
            w.c_base = (int64_t)g * j.M * j.ldc;
        }
        w.row0 = (int)row0;
        w.rows = rows < BM ? (int)rows : BM;
        w.col0 = tn * BN;
        w.nst = (int)((k1 - k0 + C::K - 1) / C::K);
        w.gap = w.nst * C::K - (int)(k1 - k0);
        w.idle = wm * WTM * 32 >= rows || wn * WTN * 32 >= j.N - w.col0;
        const int64_t k = k0 - w.gap;
        w.a = reinterpret_cast<const uint8_t*>(j.a) + uniform64((P::kAcrossA ? k * j.lda + row0 : row0 * j.lda + k) * 2);
        if constexpr (SAVED) {
            w.b = j.b8 + uniform64(k * j.ldb + w.col0);
            w.s = j.bs + uniform64(k * j.ldbs + w.col0 / kCkpt8Block);
        } else {
            w.b = reinterpret_cast<const uint8_t*>(b) + uniform64((P::kAcrossB ? k * j.ldb + w.col0 : w.col0 * j.ldb + k) * 2);
        }
#pragma unroll
        for (int q = 0; q < C::kLoadsA; ++q) w.va[q] = offset_a(w, q, 0);
#pragma unroll
        for (int q = 0; q < C::kLoadsB; ++q) w.vb[q] = offset_b(w, q, 0);
    };
    // Load q of this wave for stage i (`first`: which is stage 0) into the slot at `slot`.
    auto issue_one = [&](const Work& w, int q, int i, uint32_t slot, auto first) INLINE {
        const bool is_a = q < C::kLoadsA;
        const int u = is_a ? q : q - C::kLoadsA;
        uint32_t v;
        if constexpr (decltype(first)::value) v = is_a ? offset_a(w, u, w.gap) : offset_b(w, u, w.gap);
        else v = is_a ? w.va[u] : w.vb[u];
        // the address in scalar registers whatever the compiler took it for
        if constexpr (SAVED) {
            if (!is_a) {
                const int64_t from = uniform64(u == 0 ? (int64_t)w.b + (int64_t)i * stepB : (int64_t)w.s + (int64_t)i * stepS);
                if (u == 0) to_lds16(v, reinterpret_cast<const void*>(from), ring + slot + SA::kSize + wave * 1024);
                else to_lds4(v, reinterpret_cast<const void*>(from), ring + slot + SA::kSize + kCodes);  // every wave the same
                return;
            }
        }
        const int64_t base = uniform64(is_a ? (int64_t)w.a + (int64_t)i * stepA : (int64_t)w.b + (int64_t)i * stepB);
        to_lds16(v, reinterpret_cast<const void*>(base), ring + slot + (is_a ? 0 : SA::kSize) + (wave * (is_a ? C::kLoadsA : C::kLoadsB) + u) * 1024);
    };
    auto fill = [&](const Work& w) INLINE {  // the first stages
        if (w.nst > 0) {
#pragma unroll
            for (int q = 0; q < C::kWaveLoads; ++q) issue_one(w, q, 0, 0, std::true_type{});
        }
        for (int i = 1; i < kRing && i < w.nst; ++i)
#pragma unroll
            for (int q = 0; q < C::kWaveLoads; ++q) issue_one(w, q, i, i * kSlot, std::false_type{});
    };
    // Zeros over the places before the gap's end, in what this wave has loaded of stage 0. (A checkpoint's codes stay, those of a row of the
    // group, no infinity among them: a NaN makes the whole column NaN with or without them, all else is multiplied by A's zeros.)
    auto close_gap = [&](const Work& w, uint32_t slot) INLINE {
        const u32x4_any zero = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < (SAVED ? C::kLoadsA : C::kWaveLoads); ++q) {
            const bool is_a = q < C::kLoadsA;
            const int unit = is_a ? wave * C::kLoadsA + q : wave * C::kLoadsB + q - C::kLoadsA;
            uint32_t r, k;
            if (is_a) SA::piece((uint32_t)unit * 64 + lane, r, k);
            else SB::piece((uint32_t)unit * 64 + lane, r, k);
            if (k < (uint32_t)w.gap) *reinterpret_cast<u32x4_any*>(ring + slot + (is_a ? 0 : SA::kSize) + unit * 1024 + lane * 16) = zero;
        }
    };

    constexpr int kTiles = WTM * WTN, kOps = WTM + WTN;  // B's WTN operands, then A's WTM
    struct Operands {
        v8b v[kOps];
    };
    const uint32_t arow = (uint32_t)wm * WTM * 32, bcol = (uint32_t)wn * WTN * 32;
    uint32_t b_slot = 0;  // SAVED: where the present stage's B is in `unpacked`; the next one's is in the other
    // Operand t of the present stage at `slot`, or (`ahead`) of the next one.
    auto read_one = [&](int t, uint32_t slot, int ks, bool ahead, Operands& f) INLINE {
        if (t >= WTN) f.v[t] = SA::read(ring + slot, arow + (t - WTN) * 32, ks);
        else if constexpr (SAVED) f.v[t] = SB::read(unpacked + (ahead ? b_slot ^ SB::kSize : b_slot), bcol + t * 32, ks);
        else f.v[t] = SB::read(ring + slot + SA::kSize, bcol + t * 32, ks);
    };
    // SAVED: this thread's 16 codes of the stage at `slot` to bf16, in `unpacked` at `to`; in two steps, reading and the rest. The two
    // writes have bank conflicts (5% of the CUs' cycles); halves swapped by bit 2 of the thread have none, but the selects cost more
    // (x saved and 64 experts' 98304 x 1408 x 2048: 828-835 us instead of 812-815).
    u32x4_any codes;
    uint32_t code_scale = 0;
    auto unpack_read = [&](uint32_t slot) INLINE {
        constexpr uint32_t kEach = BN / 16;
        const uint8_t* const from = ring + slot + SA::kSize;
        codes = *reinterpret_cast<const u32x4_any*>(from + tid * 16);
        code_scale = from[kCodes + tid / kEach * (BN / 32) + tid % kEach / 2];
    };
    auto unpack_write = [&](uint32_t to) INLINE {
        constexpr uint32_t kEach = BN / 16;
        u32x4_any lo, hi;
        ckpt8_to_bf16(codes, code_scale, lo, hi);
        *reinterpret_cast<u32x4_any*>(unpacked + to + SB::across(tid / kEach, tid % kEach * 2)) = lo;
        *reinterpret_cast<u32x4_any*>(unpacked + to + SB::across(tid / kEach, tid % kEach * 2 + 1)) = hi;
    };
    // B's rows are the instruction's rows, so that a lane gets runs of consecutive columns of one row of C.
    v16f acc[WTM][WTN];
    auto multiply_one = [&](int k, const Operands& f) INLINE {
        const int a = k / WTN, b = k % WTN;
        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v[b], f.v[WTN + a], acc[a][b], 0, 0, 0);
    };
    // Waits until at most OUTSTANDING of this wave's memory operations are in flight and its LDS reads are done, then for every
    // wave: what all have waited for is then visible to all, and nobody reads the stage before any more. `opens`: the stage that can be
    // read now is stage 0 of tile w, in the slot at `slot`.
    auto arrive = [&](auto outstanding, auto opens, const Work& w, uint32_t slot) INLINE {
        asm volatile("" ::: "memory");
        wait_loads<decltype(outstanding)::value>();
        if constexpr (decltype(opens)::value) {
            if (w.gap) {
                asm volatile("" ::: "memory");
                close_gap(w, slot);
                asm volatile("" ::: "memory");
                wait_loads<63>();
            }
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // A stage, K / 16 steps: the products of one step while the next step's operands are read. Before the last step's products comes the
    // barrier that lets the next stage be read and this one be overwritten: they cover the reads of the next stage's first operands and
    // the loads of the stage kRing ahead (stage li of tile lw, if `loads`; `first`: li is 0, `opens`: the next stage is stage 0 of lw).
    // The order is pinned: one product, then what its 32 cycles cover. OUTSTANDING: as of arrive() for the next stage, -1 if there is none.
    constexpr int kSteps = C::K / 16;
    constexpr int kOpsPer = (kOps + kTiles - 1) / kTiles, kLoadsPer = (C::kWaveLoads + kTiles - 1) / kTiles;
    Operands f[2];
    auto stage = [&](auto idle, uint32_t cur, uint32_t next, auto outstanding, const Work& lw, int li, auto loads, auto first, auto opens) INLINE {
        constexpr bool kMore = decltype(outstanding)::value >= 0, kLoads = decltype(loads)::value;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            const bool last = ks == kSteps - 1;
            if constexpr (kMore)
                if (last) arrive(outstanding, opens, lw, next);
#pragma unroll
            for (int k = 0; k < kTiles; ++k) {
                if constexpr (!decltype(idle)::value) multiply_one(k, f[ks & 1]);
                if (last ? kMore : !decltype(idle)::value) {
#pragma unroll
                    for (int t = k * kOpsPer; t < (k + 1) * kOpsPer && t < kOps; ++t)
                        read_one(t, last ? next : cur, last ? 0 : ks + 1, last, f[(ks + 1) & 1]);
                }
                if constexpr (SAVED && kMore) {  // the stage after the next, over the present one's B, which has been read
                    static_assert(!SAVED || kTiles >= 4, "");
                    if (last && k == 0) unpack_read(next == (kRing - 1) * kSlot ? 0 : next + kSlot);
                    if (last && k == kTiles - 2) unpack_write(b_slot);
                }
                if constexpr (kLoads) {
                    if (last)
#pragma unroll
                        for (int q = k * kLoadsPer; q < (k + 1) * kLoadsPer && q < C::kWaveLoads; ++q) issue_one(lw, q, li, cur, first);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    constexpr int kStores = Stored<OUT, WTM, WTN>::kStores;
    auto store = [&](const Work& w, auto inside) INLINE {
        store_tile<OUT, WTM, WTN, STREAM, decltype(inside)::value>(acc, j.c, w.c_base, w.row0, w.col0, j.ldc, w.rows, j.N, wm, wn);
    };
    auto clear = [&] INLINE {
#pragma unroll
        for (int a = 0; a < WTM; ++a)
#pragma unroll
            for (int b = 0; b < WTN; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    };
    auto is_inside = [&](const Work& w) INLINE { return w.rows == BM && (int64_t)w.col0 + BN <= j.N; };

    uint32_t L = blockIdx.x;
    // The workgroup's first tile is its own place in the order of tiles, the next one the first that no other has: one counter for each of
    // the 8 XCDs, whose workgroups and tiles are those of one remainder modulo 8. Without counters, one of every gridDim.x.
    auto take = [&] INLINE {  // by the first thread
        // (a weights' gradient has counters whenever it has more tiles than workgroups)
        if (!j.counters) return P::kRagged ? L + gridDim.x : total;
        const uint32_t x = blockIdx.x % 8;
        return (gridDim.x / 8 + atomicAdd(j.counters + x * kCounterStride, 1u)) * 8 + x;
    };
    if (L >= total) return;
    Work w;
    locate(L, w);
    fill(w);
    uint32_t cur = 0, next = kSlot;
    auto advance = [&] INLINE {
        cur = next;
        next = next == (kRing - 1) * kSlot ? 0 : next + kSlot;
        if constexpr (SAVED) b_slot ^= SB::kSize;
    };
    auto begin = [&] INLINE {
        if constexpr (SAVED) {  // the first two stages
            unpack_read(cur);
            unpack_write(b_slot);
            unpack_read(next);
            unpack_write(b_slot ^ SB::kSize);
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < kOps; ++t) read_one(t, cur, 0, false, f[0]);
    };
    using std::integral_constant;
    constexpr int L1 = C::kWaveLoads;
    constexpr std::true_type yes{};
    constexpr std::false_type no{};

    // Long tiles: the stages of one follow those of the one before without a gap. A tile's last kRing stages load the next one's first
    // (after the last tile its own first ones again, which nobody reads: a branch here makes the compiler spill the sums), and the last
    // reads the first's operands. A tile's stores are then younger than those loads, and memory operations complete in order, so the next
    // tile's first waits count them in instead of waiting for them.
    constexpr int kLong = 2 * kRing;
    constexpr int kAhead = SAVED ? 2 : 1;  // what a stage's barrier lets be read has landed up to this many stages on
    constexpr integral_constant<int, (kRing - 1 - kAhead) * L1> kept{};
    if (w.nst >= kLong) {
        arrive(integral_constant<int, (kRing - kAhead) * L1>{}, yes, w, cur);
        begin();
        bool behind = false;  // kStores stores were issued after the loads
        while (true) {
            clear();
            uint32_t taken = 0;
            if (tid == 0) taken = take();
            Work n;
            bool more, go;
            auto run = [&](auto idle) INLINE {
                int i = 0;
                if (behind) {
                    for (; i < kRing - kAhead; ++i) {
                        stage(idle, cur, next, integral_constant<int, (kRing - 1 - kAhead) * L1 + kStores>{}, w, i + kRing, yes, no, no);
                        advance();
                    }
                }
                if (tid == 0) s_next = taken;  // a barrier lies between this and its reading: kLong
                for (; i + kRing < w.nst; ++i) {
                    stage(idle, cur, next, kept, w, i + kRing, yes, no, no);
                    advance();
                }
                L = (uint32_t)uniform((int)s_next);
                more = L < total;
                n = w;
                if (more) locate(L, n);
                go = more && n.nst >= kLong;  // shorter ones, which come last where they differ, go the other way
                if (!go) n = w;
#pragma unroll
                for (int q = 0; q < kRing; ++q) {
                    if (q == 0) stage(idle, cur, next, kept, n, q, yes, yes, no);
                    else if (q == kRing - 1) stage(idle, cur, next, kept, n, q, yes, no, yes);
                    else stage(idle, cur, next, kept, n, q, yes, no, no);
                    advance();
                }
            };
            if (w.idle) run(yes);
            else run(no);
            asm volatile("" ::: "memory");
            behind = is_inside(w);
            if (behind) store(w, yes);
            else store(w, no);
            if (!go) {
                wait_loads<0>();  // the LDS must not be another tile's or workgroup's before they have landed
                if (!more) return;
                break;
            }
            w = n;
        }
        __syncthreads();
        locate(L, w);
        fill(w);
    }

    // Short tiles: one after the other.
    while (true) {
        clear();
        if (w.nst > 0) {
            cur = 0, next = kSlot, b_slot = 0;
            arrive(integral_constant<int, 0>{}, yes, w, cur);
            begin();
            auto body = [&](auto idle) INLINE {
                int i = 0;
                for (; i + kRing < w.nst; ++i) {
                    stage(idle, cur, next, kept, w, i + kRing, yes, no, no);
                    advance();
                }
                for (; i + 1 < w.nst; ++i) {  // the loads are on their way: wait for all of them
                    stage(idle, cur, next, integral_constant<int, 0>{}, w, 0, no, no, no);
                    advance();
                }
                stage(idle, cur, next, integral_constant<int, -1>{}, w, 0, no, no, no);
            };
            if (w.idle) body(yes);
            else body(no);
        }
        const Work done = w;
        if (tid == 0) s_next = take();
        __syncthreads();  // every wave has read the last stage
        L = (uint32_t)uniform((int)s_next);
        const bool more = L < total;
        if (more) {
            locate(L, w);
            __syncthreads();  // and what was taken
            fill(w);
        }
        asm volatile("" ::: "memory");
        if (is_inside(done)) store(done, yes);
        else store(done, no);
        if (!more) return;
    }
}

// Two stages of 64 places, 128 bytes of a row, or four of 32: operands along the reduction are read in whole lines by the former (8192^3
// forward 910 -> 851 us); one across it has whole lines in both, and more loads on the way in the latter (64 experts' 98304 x 1408 x
// 2048, us, 64 / 32: weights' gradient 751 / 709, input's gradient 568 / 557).
template <int PASS>
struct Depth {
    static constexpr int K = PASS == kBf16FwdY ? 64 : 32, kRing = 128 / K;
};
template <int PASS>
using Tile256 = Tile<4, 2, 2, 4, Depth<PASS>::K, Depth<PASS>::kRing, 1>;  // 256 x 256: 8 waves of 128 x 64, two per SIMD
template <int PASS>
using Tile128 = Tile<2, 2, 2, 2, Depth<PASS>::K, Depth<PASS>::kRing, 2>;  // 128 x 128: 4 waves of 64 x 64, two workgroups per CU

// ------------------------------------------------------------------------------------------------
// Few rows (a decode step): bound by reading the weights of the groups that have any.
// ------------------------------------------------------------------------------------------------

// A workgroup takes 16 CT columns of 16 RT rows of one group's product and reads its rows of W once, from memory (where other rows of the group
// came first, the L2) to the registers of v_mfma_f32_16x16x32_bf16 (16 rows x 64 consecutive bytes a load); its waves split the reduction in
// chunks of 64 places and add their sums in order. Any size, stride and alignment.
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves, kFewChunk = 64;

template <int OUT, int CT, int RT>
__global__ __launch_bounds__(kFewThreads) void gemm_bf16_few_kernel(Bf16GemmJob j) {
    constexpr int kTiles = CT * RT;
    __shared__ float4 sums[kFewWaves][kTiles * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), quarter = lane >> 4, l16 = lane & 15;
    const uint32_t chunks = (uint32_t)((j.N + 16 * CT - 1) / (16 * CT)), rank = blockIdx.x / chunks;
    const int64_t col0 = (int64_t)(blockIdx.x % chunks) * (16 * CT);
    // the group, and its rows from r0 on: the rank-th block of rows, counted over the groups
    constexpr int kRows = 16 * RT;
    int64_t start = 0, rows = 0, r0 = 0;
    int g = -1, claimed = 0;
    uint32_t before = 0;
    for (int g0 = 0; g0 < j.G && g < 0; g0 += 64) {
        int from, m;
        group_rows(j, g0, claimed, from, m);
        const uint64_t some = __ballot(m > 0);
        if (!__ballot(m > kRows)) {  // a block each
            const uint32_t n = (uint32_t)__popcll(some);
            if (before + n > rank) {
                uint64_t left = some;
                for (uint32_t skip = rank - before; skip > 0; --skip) left &= left - 1;
                g = uniform(__builtin_ctzll(left));
            }
            before += n;
        } else {
            const uint32_t n = (uint32_t)(((int64_t)m + kRows - 1) / kRows);
            uint32_t upto = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t v = __shfl_up(upto, d, 64);
                if (lane >= d) upto += v;
            }
            const uint64_t past = __ballot(before + upto > rank);
            if (past) {
                g = uniform(__builtin_ctzll(past));
                r0 = (int64_t)(rank - before - (uint32_t)__builtin_amdgcn_readlane((int)(upto - n), g)) * kRows;
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        if (g >= 0) {
            start = __builtin_amdgcn_readlane(from, g);
            rows = __builtin_amdgcn_readlane(m, g);
            g += g0;
        }
    }
    if (g < 0) return;
    const uint16_t* w[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {  // columns past the last one are not stored
        const int64_t n = col0 + t * 16 + l16;
        w[t] = j.b + ((int64_t)g * j.N + (n < j.N ? n : j.N - 1)) * j.ldb;
    }
    const uint16_t* x[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int64_t r = r0 + t * 16 + l16;
        x[t] = j.a + (start + (r < rows ? r : rows - 1)) * j.lda;
    }
    v4f acc[CT][RT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[c][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kSteps = kFewChunk / 32;
    struct Chunk {
        u32x4_any w[CT][kSteps], x[RT][kSteps];
    };
    auto load = [&](Chunk& c, int64_t k0) INLINE {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int64_t k = k0 + s * 32 + quarter * 8;
#pragma unroll
            for (int t = 0; t < CT; ++t) c.w[t][s] = Piece<uint16_t>::load(w[t] + k, j.red - k);
#pragma unroll
            for (int t = 0; t < RT; ++t) c.x[t][s] = Piece<uint16_t>::load(x[t] + k, j.red - k);
        }
    };
    auto multiply = [&](const Chunk& c) INLINE {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int n = 0; n < CT; ++n)
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, c.w[n][s]), __builtin_bit_cast(v8b, c.x[t][s]),
                                                                        acc[n][t], 0, 0, 0);
    };
    constexpr int64_t kStep = kFewWaves * kFewChunk;
    int64_t k = wave * kFewChunk;
    Chunk c0, c1;
    if (k < j.red) load(c0, k);
    for (; k + kStep < j.red; k += 2 * kStep) {
        load(c1, k + kStep);
        multiply(c0);
        if (k + 2 * kStep < j.red) load(c0, k + 2 * kStep);
        multiply(c1);
    }
    if (k < j.red) multiply(c0);
    // A lane has columns 4 quarter .. + 3 of row l16 of each tile.
#pragma unroll
    for (int n = 0; n < CT; ++n)
#pragma unroll
        for (int t = 0; t < RT; ++t) sums[wave][(n * RT + t) * 64 + lane] = make_float4(acc[n][t][0], acc[n][t][1], acc[n][t][2], acc[n][t][3]);
    __syncthreads();
    for (int i = tid; i < kTiles * 64; i += kFewThreads) {
        float4 v = sums[0][i];
#pragma unroll
        for (int o = 1; o < kFewWaves; ++o) {
            const float4 u = sums[o][i];
            v.x += u.x;
            v.y += u.y;
            v.z += u.z;
            v.w += u.w;
        }
        const int64_t r = r0 + (i / 64 % RT) * 16 + (i & 15), c = col0 + (i / 64 / RT) * 16 + (i >> 4 & 3) * 4;
        const float f[4] = {v.x, v.y, v.z, v.w};
        if (r >= rows) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= j.N) continue;
            const int64_t at = (start + r) * j.ldc + c + e;
            if constexpr (OUT == kOutF32) static_cast<float*>(j.c)[at] = f[e];
            else static_cast<uint16_t*>(j.c)[at] = __builtin_bit_cast(uint16_t, (__bf16)f[e]);
        }
    }
}

constexpr int64_t kMostGroups = int64_t(1) << 23;  // workgroups: a grid holds fewer than 2^32 threads

// Tile rows that a launch provides for; ragged rows: every group may end in a partial tile.
int64_t tile_rows(const Bf16GemmJob& j, int bm) {
    return j.pass != kBf16BwdDw ? (j.tokens + bm - 1) / bm + j.G : (j.M + bm - 1) / bm;
}
int64_t grid_tiles(const Bf16GemmJob& j, int bm, int bn) {
    return tile_rows(j, bm) * ((j.N + bn - 1) / bn) * (j.pass == kBf16BwdDw ? j.G : 1);
}

// Whether every row is whole 16-byte pieces, and a tile's rows (or a stage's) lie within 32 bits.
bool pieces(const Bf16GemmJob& j) {
    constexpr int64_t kMost = int64_t(1) << 22;
    const int64_t wide_a = j.pass == kBf16BwdDw ? j.M : j.red, wide_b = j.pass == kBf16FwdY ? j.red : j.b8 ? 0 : j.N;
    if (j.b8 && (j.ldbs % 4 != 0 || j.ldbs > kMost || reinterpret_cast<uintptr_t>(j.bs) % 4 != 0)) return false;  // codes are whole pieces
    return wide_a % 8 == 0 && wide_b % 8 == 0 && j.lda % 8 == 0 && j.ldb % 8 == 0 && j.lda <= kMost && j.ldb <= kMost &&
           reinterpret_cast<uintptr_t>(j.a) % 16 == 0 && reinterpret_cast<uintptr_t>(j.b) % 16 == 0;
}

constexpr int kCounters = 8 * kCounterStride;

// Whether the workgroups that are resident take the tiles as they get done, instead of in turn. It costs a launch that clears the counters
// (2 us) and gains where tiles differ: those of a ragged reduction, and where many have parts outside of the output. Measured, us, by counters /
// in turn: 98304 x 1408 x 2048 of 64 experts (2496 tiles) forward 556 / 571, input's gradient 557 / 566; 4096 x 4096 x 1024 of one (256)
// 36.2 / 34.4, 8192 rows of 8 (288) input's gradient 70.3 / 68.5.
bool counted(const Bf16GemmJob& j, int64_t tiles, int resident) { return tiles > (j.pass == kBf16BwdDw ? 1 : 4) * resident; }

template <int OUT, class C, int PASS, bool STREAM, bool SAVED>
hipError_t launch_tile(Bf16GemmJob j, hipStream_t s) {
    int64_t tiles = grid_tiles(j, C::BM, C::BN);
    if (counted(j, tiles, C::kResident)) clear_counters_kernel<<<1, kCounters, 0, s>>>(j.counters);
    else j.counters = nullptr;
    if (tiles > C::kResident) tiles = C::kResident;
    gemm_bf16_kernel<OUT, C, PASS, STREAM, SAVED><<<(unsigned)tiles, C::kThreads, 0, s>>>(j);
    return hipGetLastError();
}

// Which tile takes a product of whole pieces: the one with the smaller estimated time, in us, from the tiles that a CU gets (t, ragged rows
// with half a tile lost per group) and the reduction (of a weights' gradient the average group's; the longest is taken as three times that,
// and no tile of it ends sooner than alone on a CU). Measured on gfx950, 256 / 128, us:
//     one group, forward: 2048^3 43 / 25, 4096 x 4096 x 1024 36 / 39, 4096 x 2048 x 8192 143 / 123, 2048 x 8192 x 2048 60 / 68;
//     8 experts, 8192 rows, 2048 -> 1408: forward 50 / 57, gradients 71 / 64, 87 / 69; 4096 rows, 2048 -> 4096: 94 / 83, 80 / 105, 107 / 116;
//     16 experts, 16384 rows, 1312 -> 512: 37 / 45, 36 / 36, 89 / 62; 64 experts, 24576 rows, 2048 -> 1408: 181 / 202, 175 / 241, 262 / 313,
//     6144 rows: 106 / 89, 108 / 102, 156 / 178.
double estimate(const Bf16GemmJob& j, bool big) {
    const double tile = big ? 256.0 : 128.0, cols = ceil((double)j.N / tile);
    const bool dw = j.pass == kBf16BwdDw;
    const double rows = dw ? ceil((double)j.M / tile) * j.G : (double)j.tokens / tile + (j.tokens < j.G ? j.tokens : j.G) * 0.5;
    const double red = dw ? (double)j.tokens / j.G : (double)j.red, t = ceil(rows) * cols / 256.0;
    const double longest = dw && j.G > 1 ? (3.0 * red < j.tokens ? 3.0 * red : j.tokens) : red;
    double us, alone;
    if (big) {  // per 64 of the reduction: a full round of tiles 1.65, a partial one less
        const double part = t - floor(t);
        us = 9.0 + red / 64.0 * (floor(t) * 1.65 + (part > 0.0 ? 1.05 + 0.6 * part : 0.0));
        alone = 9.0 + longest / 64.0 * 1.1;
    } else {  // per 32: two tiles a CU 0.5 (many: 0.64), one 0.31
        const double part = t - 2.0 * floor(t / 2.0);
        us = 6.0 + red / 32.0 * (floor(t / 2.0) * (t <= 4.0 ? 0.5 : 0.64) + (part > 1.0 ? 0.45 : part > 0.0 ? 0.31 : 0.0));
        alone = 6.0 + longest / 32.0 * 0.31;
    }
    return us > alone ? us : alone;
}
bool large(const Bf16GemmJob& j) {
    // Many tiles of a weights' gradient are bound by their stores, which the larger ones make nontemporally, unless those cover much more than the
    // smaller ones (up to 3/2: 1024 of them are then 64 MiB of fp32 results at least). Measured, us, 256 / 128, results in fp32:
    //     1024 groups 64 x 64, 32 rows each 194 / 95, 128 rows 219 / 106; 64 groups 64 x 4096, 256 rows 60 / 45; 1024 groups 128 x 256, 64 rows
    //     205 / 204; 136 x 264 414 / 577.
    const int64_t most = grid_tiles(j, 256, 256);
    if (j.pass == kBf16BwdDw && most >= 1024 && 8 * most <= 3 * grid_tiles(j, 128, 128)) return true;
    return estimate(j, true) < estimate(j, false);
}

// Outputs that no cache holds are stored nontemporally; weights' gradients, which are read when a step's have all been computed, from
// 64 MiB on.
bool streams(const Bf16GemmJob& j) {
    const bool dw = j.pass == kBf16BwdDw;
    return (dw ? j.M * j.G : j.tokens) * j.N * (j.out_dtype == kOutF32 ? 4 : 2) >= (dw ? int64_t(64) << 20 : kStreamBytes);
}

template <int OUT, int PASS, bool SAVED = false>
hipError_t launch_pass(const Bf16GemmJob& j, hipStream_t s) {
    if (!large(j)) return launch_tile<OUT, Tile128<PASS>, PASS, false, SAVED>(j, s);
    return streams(j) ? launch_tile<OUT, Tile256<PASS>, PASS, true, SAVED>(j, s) : launch_tile<OUT, Tile256<PASS>, PASS, false, SAVED>(j, s);
}

// 32 columns a workgroup (16: 42 rows of 64 experts 21.9 us, 64: 23.5; 5120 -> 4096 2 rows 15.8, 23.8; W in the memory-side cache).
constexpr int kFewCols = 2;
// Rows of a workgroup, by the average of the groups that can have any.
int few_tiles(const Bf16GemmJob& j) {
    const int64_t groups = j.tokens < j.G ? j.tokens : j.G;
    return j.tokens <= 16 * groups ? 1 : j.tokens <= 32 * groups ? 2 : 4;
}
// Its workgroups: those of the columns for each block of rows, of which every group may leave one partial.
int64_t few_grid(const Bf16GemmJob& j) {
    const int64_t groups = j.tokens < j.G ? j.tokens : j.G;
    return (j.N + 16 * kFewCols - 1) / (16 * kFewCols) * (groups + (j.tokens - groups) / (16 * few_tiles(j)));
}

// Which products the few-row kernel takes: of 64 rows in all, or of up to 128 groups up to 8 rows a group on average and 512 in all; and where its
// grid fits. Past that its rows of W come through the L2 more than once, 128-row tiles read them less often, and finding a workgroup's group
// takes one load after the other. Measured, us, few-row kernel / 128 x 128 tiles, a power law's loads, weights that no cache holds:
//     64 experts 2048 -> 1408: 6 rows 12 / 23, 42 33 / 40, 96 44 / 49, 192 60 / 83, 384 76 / 89, 504 83 / 90;
//     8 experts 5120 -> 4096: 2 rows 20 / 72, 42 76 / 82, 64 86 / 82; 512 -> 1312: 2 rows 5.8 / 9.4, 64 7.7 / 12.0;
//     one group 2048 -> 8192: 1 row 11 / 32, 64 19 / 32;
//     128 experts 2048 -> 1408: 96 rows 51 / 53, 192 77 / 88, 512 118 / 131, 1024 158 / 150; 512 -> 512: 192 14.3 / 13.7, 512 20 / 16;
//     256 experts 1024 -> 512: 96 rows 15 / 20, 192 27 / 24, 512 47 / 43; 1024 experts 512 -> 512: 96 rows 21 / 22, 512 103 / 39;
// and all rows in one group, which the caches then hold (loads are known on the GPU only):
//     64 experts 2048 -> 1408: 42 rows 9 / 18, 192 20 / 18, 510 37 / 19 (a workgroup that takes all blocks of its group in turn: 188).
bool few(const Bf16GemmJob& j) {
    return j.pass == kBf16FwdY && (j.tokens <= 64 || (j.G <= 128 && j.tokens <= 8 * (j.G < 64 ? j.G : 64))) && few_grid(j) < kMostGroups;
}

template <int OUT>
hipError_t launch_few(const Bf16GemmJob& j, hipStream_t s) {
    const unsigned n = (unsigned)few_grid(j);
    switch (few_tiles(j)) {
        case 1: gemm_bf16_few_kernel<OUT, kFewCols, 1><<<n, kFewThreads, 0, s>>>(j); break;
        case 2: gemm_bf16_few_kernel<OUT, kFewCols, 2><<<n, kFewThreads, 0, s>>>(j); break;
        default: gemm_bf16_few_kernel<OUT, kFewCols, 4><<<n, kFewThreads, 0, s>>>(j);
    }
    return hipGetLastError();
}

template <int OUT>
hipError_t launch_any(const Bf16GemmJob& j, hipStream_t s) {
    const unsigned n = (unsigned)grid_tiles(j, kAnyTile, kAnyTile);
    switch (j.pass) {
        case kBf16FwdY: gemm_bf16_any_kernel<OUT, kBf16FwdY, false><<<n, kAnyThreads, 0, s>>>(j); break;
        case kBf16BwdDx: gemm_bf16_any_kernel<OUT, kBf16BwdDx, false><<<n, kAnyThreads, 0, s>>>(j); break;
        default:
            if (j.b8) gemm_bf16_any_kernel<OUT, kBf16BwdDw, true><<<n, kAnyThreads, 0, s>>>(j);
            else gemm_bf16_any_kernel<OUT, kBf16BwdDw, false><<<n, kAnyThreads, 0, s>>>(j);
    }
    return hipGetLastError();
}

template <int OUT>
hipError_t launch_out(const Bf16GemmJob& j, hipStream_t s) {
    if (grid_tiles(j, kAnyTile, kAnyTile) == 0) return hipSuccess;
    if (few(j)) return launch_few<OUT>(j, s);
    if (!pieces(j)) return launch_any<OUT>(j, s);
    switch (j.pass) {
        case kBf16FwdY: return launch_pass<OUT, kBf16FwdY>(j, s);
        case kBf16BwdDx: return launch_pass<OUT, kBf16BwdDx>(j, s);
        default: return j.b8 ? launch_pass<OUT, kBf16BwdDw, true>(j, s) : launch_pass<OUT, kBf16BwdDw>(j, s);
    }
}

}  // namespace

int64_t bf16_gemm_workspace(const Bf16GemmJob& j) {
    if (few(j)) return 0;
    const int tile = large(j) ? 256 : 128, resident = large(j) ? Tile256<kBf16FwdY>::kResident : Tile128<kBf16FwdY>::kResident;
    return counted(j, grid_tiles(j, tile, tile), resident) ? kCounters * 4 : 0;
}

bool bf16_gemm_fits(const Bf16GemmJob& j) { return grid_tiles(j, kAnyTile, kAnyTile) < kMostGroups; }

hipError_t launch_gemm_bf16(const Bf16GemmJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_out<kOutBF16>(j, s) : launch_out<kOutF32>(j, s);
}

}  // namespace ufp4

namespace {

ufp4::Bf16GemmJob planned(int pass, int64_t tokens, int64_t N, int64_t K, int32_t G) {
    ufp4::Bf16GemmJob j{};
    j.pass = pass;
    j.tokens = tokens;
    j.M = pass == ufp4::kBf16BwdDw ? N : 0;
    j.N = pass == ufp4::kBf16FwdY ? N : K;
    j.red = pass == ufp4::kBf16FwdY ? K : pass == ufp4::kBf16BwdDx ? N : 0;
    j.G = G;
    return j;
}

}  // namespace

extern "C" int ufp4_plan_gemm_bf16(int pass, int64_t tokens, int64_t N, int64_t K, int32_t G, int whole_pieces) {
    const ufp4::Bf16GemmJob j = planned(pass, tokens, N, K, G);
    return ufp4::few(j) ? 0 : !whole_pieces ? 1 : ufp4::large(j) ? 3 : 2;
}

extern "C" int ufp4_plan_gemm_bf16_streams(int pass, int64_t tokens, int64_t N, int64_t K, int32_t G, int out_dtype) {
    ufp4::Bf16GemmJob j = planned(pass, tokens, N, K, G);
    j.out_dtype = out_dtype;
    return !ufp4::few(j) && ufp4::large(j) && ufp4::streams(j);
}
