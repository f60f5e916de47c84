// GEMM on microscaled 4-bit operands: C[i, j] = sum_k A[i,k] 2^(eA[i,k/32] - 127) B[j,k] 2^(eB[j,k/32] - 127), A and B E2M1
// levels in the layout of ufp4_mxfp4.hip, sums in fp32 by v_mfma_scale_f32_32x32x64_f8f6f4, which applies both scales.
//
// A lane of the instruction holds the 32 codes of one row and one 32-block: 16 bytes, one LDS read. K advances 128 (four
// blocks) per stage; a panel's stage is 8 KiB of codes and 512 bytes of scales, both contiguous, copied unchanged into a
// three-deep LDS ring by direct-to-LDS loads (a fourth slot measured the same at 16384^3). Each wave keeps two sets of operands
// in registers: while the matrix core works on one half of a stage, the other half (or, past the barrier, the next stage's first
// half) is read from LDS, so that neither the barrier nor the LDS latency stands between two matrix instructions.
//
// Bound by the matrix cores and their power where the reduction is long: the instruction alone, on registers, reaches 6.3 PFLOP/s
// on codes of normal numbers (9.8 on zeros: power takes the clock to 1.5 GHz), 16384^3 with bf16 output takes 1.75-1.87 ms = 4.7-5.0
// (matrix cores busy 73% of the time at 1.5 GHz). Where it is short, by the stores, which take the memory system from the loads:
// 16384 x 16384 x 2048 takes 0.29 ms = 3.8 PFLOP/s, without its stores 0.235 ms.

#include "ufp4_internal.h"
#include "ufp4_mxfp4.h"
#include "ufp4_rows.h"
#include "ufp4_tiles.h"

#include <math.h>

#include <type_traits>

namespace ufp4 {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));

#define INLINE __attribute__((always_inline))

constexpr int kStage = 4;  // 32-blocks per stage

// WM x WN waves, each with WTM x WTN matrix tiles of 32 x 32 outputs; RING stages in LDS; PER_CU workgroups on a CU. SPLIT > 1:
// as many such teams of waves per workgroup, each with a ring of its own, take every SPLIT-th stage of one tile.
template <int WTM_, int WTN_, int WM_, int WN_, int RING_, int PER_CU, int SPLIT = 1>
struct Tile {
    static constexpr int WTM = WTM_, WTN = WTN_, WM = WM_, WN = WN_, kRing = RING_, kSplit = SPLIT;
    static constexpr int BM = 32 * WTM * WM, BN = 32 * WTN * WN;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves * SPLIT;  // kWaves of a team
    static constexpr int kResident = 256 * PER_CU;      // workgroups on 256 CUs
    static constexpr int kPerEU = PER_CU * kWaves * SPLIT / 4;  // waves per SIMD that the registers have to allow
    // Panels (of a 64-row tile: halves of one) of A and B; 1 KiB direct-to-LDS loads of a panel's stage, dealt to the waves;
    // and the 16-byte pieces of its scales, in units of kScaleLanes. A wave left over loads a unit that another one loads, too.
    static constexpr int kRowsP = BM < 128 ? BM : 128, kPanelsA = BM / kRowsP, kPanels = kPanelsA + BN / kRowsP;
    static constexpr int kPanelLoads = kRowsP / 16, kWaveCodes = kPanels * kPanelLoads / kWaves;
    static constexpr int kPieces = kRowsP / 4, kNeed = kPanels * kPieces;
    static constexpr int kScaleLanes = kNeed <= kWaves * 8 ? 8 : kNeed <= kWaves * 16 ? 16 : 32;
    static constexpr int kWaveLoads = kWaveCodes + 1;
    static_assert(kPanelLoads % kWaves == 0 && BN >= kRowsP && kPieces % kScaleLanes == 0 && kNeed <= kWaves * kScaleLanes,
                  "every wave issues the same loads");
    static_assert(kWaveLoads * (kRing - 1) < 64, "vmcnt has six bits");
};

// A slot of the ring: A's codes [panel][block][row] 16 bytes, as in memory (of a 64-row tile [block][row]), B's, then the scales
// of A and of B [panel][block % 2][row][2].
template <class C>
struct Slot {
    static constexpr uint32_t kB = C::BM * 64, kScales = kB + C::BN * 64, kSize = kScales + (C::BM + C::BN) * 4;
};

// The same by the first N lanes of a wave whose lanes are all active. Not an `if`: a branch would split the main loop into
// blocks between which the compiler moves products and operands.
template <int N>
__device__ __forceinline__ void to_lds16_first(uint32_t voff, const void* sbase, const void* lds_base) {
    static_assert(N <= 32, "the upper half is off");
    const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t) reinterpret_cast<uintptr_t>(lds_base));
    asm volatile(
        "s_mov_b32 m0, %2\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, 0\n\tglobal_load_lds_dwordx4 %0, %1\n\t"
        "s_mov_b64 exec, -1" ::"v"(voff), "s"(sbase), "s"(m0), "i"((int)(0xFFFFFFFFu >> (32 - N)))
        : "memory");
}

// Tile rows of a grid; ragged-M: a bound over all groups, each of which may end in a partial tile.
__host__ __device__ inline int64_t tile_rows(const MxGemmJob& j, int bm) {
    return j.mode == kGemmRaggedM ? (j.a_rows + bm - 1) / bm + j.G : (j.M + bm - 1) / bm;
}

// Ragged rows: the groups' first panel of the padded rows, first token, and, where a tile is two panels, first tile row, in LDS,
// built by the first wave, 64 groups at a time. (A 64-row tile is half a panel: a group's tile rows are
// then twice its panels, the last of which may hold none of its rows.) Operands and outputs hold fewer than 2^31 rows; what
// offsets claim past that is cut.
template <int BM>
struct Groups {
    static constexpr int kN = kMxfp4Groups + 1;
    int unit[kN], token[kN], tile[BM > 128 ? kN : 1];
    static constexpr int kTilesPerPanel = BM > 128 ? 1 : 128 / BM;

    __device__ __forceinline__ void build(const MxGemmJob& j) {
        const int G = j.G, lane = threadIdx.x & 63;
        int64_t tiles = 0, units = 0;  // what offsets claim can sum to more than 32 bits; 64 groups of it cannot
        auto cut = [](int64_t v) { return v > INT32_MAX ? INT32_MAX : (int)v; };
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + lane;
            const int64_t start = g < G ? j.offsets[g] : 0;
            int64_t m = g < G ? j.offsets[g + 1] - start : 0;
            m = m < 0 ? 0 : m > INT32_MAX ? INT32_MAX : m;
            const uint32_t cnt = (uint32_t)((m + BM - 1) / BM), n = (uint32_t)((m + 127) / 128);
            uint32_t ti = cnt, ni = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t vt = __shfl_up(ti, d, 64), vn = __shfl_up(ni, d, 64);
                if (lane >= d) {
                    ti += vt;
                    ni += vn;
                }
            }
            if (g < G) {
                unit[g] = cut(units + (ni - n));
                token[g] = start < 0 ? -1 : cut(start);
                if constexpr (BM > 128) tile[g] = cut(tiles + (ti - cnt));
            }
            tiles += (uint32_t)__shfl(ti, 63, 64);
            units += (uint32_t)__shfl(ni, 63, 64);
        }
        if (lane == 0) {
            const int64_t end = j.offsets[G];
            unit[G] = cut(units);
            token[G] = end < 0 ? -1 : cut(end);
            if constexpr (BM > 128) tile[G] = cut(tiles);
        }
    }
    __device__ __forceinline__ int first_tile(int g) const {
        if constexpr (BM > 128) return tile[g];
        else return unit[g] > INT32_MAX / kTilesPerPanel ? INT32_MAX : unit[g] * kTilesPerPanel;
    }
    // The group that holds tile row t: the last one whose first tile row is at most t (empty groups share their successor's).
    __device__ __forceinline__ int of(int G, int t) const {
        int n = 0;
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + (threadIdx.x & 63);
            n += __popcll(__ballot(g < G && first_tile(g) <= t));
        }
        return n - 1;
    }
};

// Ragged reduction: the first 32-block of group g and the one past its last, by a sum over the lanes of each wave.
__device__ __forceinline__ void group_blocks(const MxGemmJob& j, int g, int& first, int& end) {
    const int lane = threadIdx.x & 63;
    auto blocks = [&](int h) {
        const int64_t m = j.offsets[h + 1] - j.offsets[h];
        return m <= 0 ? 0 : m > INT32_MAX ? int64_t(1) << 26 : (m + 31) / 32;
    };
    int64_t sum = 0;
    for (int h = lane; h < g; h += 64) sum += blocks(h);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
    const int64_t stop = sum + blocks(g);  // clamped to the operands: fewer than 2^31 blocks
    first = uniform((int)(sum < j.nkb ? sum : j.nkb));
    end = uniform((int)(stop < j.nkb ? stop : j.nkb));
}

template <int OUT, class C, int MODE, bool STREAM>
__global__ __launch_bounds__(C::kThreads, C::kPerEU) void gemm_mxfp4_kernel(MxGemmJob j) {
    using S = Slot<C>;
    constexpr int kRing = C::kRing;
    __shared__ __align__(16) uint8_t rings[C::kSplit * kRing * S::kSize];
    __shared__ typename std::conditional<MODE == kGemmRaggedM, Groups<C::BM>, int>::type groups;
    constexpr int BM = C::BM, BN = C::BN, WTM = C::WTM, WTN = C::WTN;
    constexpr int kRowsP = C::kRowsP;     // rows of a panel in LDS
    constexpr bool kHalf = kRowsP < 128;  // half a panel per operand
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int kSplit = C::kSplit;
    const int team = kSplit > 1 ? (int)((unsigned)uniform(tid >> 6) / C::kWaves) : 0;
    const int wave = uniform(tid >> 6) - team * C::kWaves;  // of the team
    uint8_t* const ring = rings + team * kRing * S::kSize;
    const int h = lane >> 5, l32 = lane & 31;
    const int wm = (int)((unsigned)wave / C::WN), wn = (int)((unsigned)wave % C::WN);
    const uint32_t gx = (uint32_t)((j.N + BN - 1) / BN);
    uint32_t gy = (uint32_t)tile_rows(j, BM), total = gx * gy;
    if constexpr (MODE == kGemmRaggedM) {
        if (tid < 64) groups.build(j);
        __syncthreads();
        const uint32_t have = (uint32_t)uniform(groups.first_tile(j.G));
        gy = have < gy ? have : gy;
        total = gx * gy;
    } else if constexpr (MODE == kGemmRaggedK) {
        total *= (uint32_t)j.G;
    }

    // One output tile: the panels of its operands (A's, then B's) at the reduction's first block, this wave's scales, the stages,
    // and where the results go.
    struct Work {
        const uint8_t* gw[C::kPanels];
        const uint8_t* gs;
        int st0, nst, kbf, kbe;  // first stage, stages, blocks [kbf, kbe) of them
        int row0, rows, col0;    // first row of the output, rows that exist, first column
        int64_t c_base;
    };
    constexpr int kUnits = C::kPieces / C::kScaleLanes;
    const int unit = wave % (C::kPanels * kUnits), spanel = unit / kUnits;  // this wave's unit of the scales
    auto locate = [&](uint32_t L, Work& w) INLINE {
        int tm, tn, g = 0;
        if constexpr (MODE == kGemmRaggedK) {
            g = (int)(L / (gx * gy));
            L -= (uint32_t)g * (gx * gy);
        }
        tile_at(L, gy, gx, tm, tn);
        int64_t arow0 = (int64_t)tm * BM, brow0 = (int64_t)tn * BN, b_kb0 = 0, kbf = 0, kbe = j.nkb;
        int64_t row0 = arow0, rows = j.M - arow0;
        w.c_base = 0;
        if constexpr (MODE == kGemmRaggedM) {
            g = groups.of(j.G, tm);
            const int lt = tm - uniform(groups.first_tile(g));
            arow0 = (int64_t)uniform(groups.unit[g]) * 128 + lt * BM;
            const int start = uniform(groups.token[g]), end = uniform(groups.token[g + 1]);
            row0 = (int64_t)start + lt * BM;
            rows = end - row0 < j.M - row0 ? end - row0 : j.M - row0;  // token rows past the output are not stored
            if (start < 0) rows = 0;
            brow0 += g * j.b_group_rows;
            b_kb0 = g * j.b_group_kb;
        } else if constexpr (MODE == kGemmRaggedK) {
            int first, end;
            group_blocks(j, g, first, end);
            kbf = first;
            kbe = end;
            w.c_base = (int64_t)g * j.M * j.ldc;
        }
        // Stages are whole groups of four blocks (the scales' unit). A ragged reduction may begin and end inside one.
        w.kbf = (int)kbf;
        w.kbe = (int)kbe;
        w.st0 = (int)(kbf / kStage);
        w.nst = kbe > kbf ? (int)((kbe + kStage - 1) / kStage) - w.st0 : 0;
        if constexpr (kSplit > 1) {  // the team's stages: all teams take as many, those past the reduction masked
            w.nst = (w.nst + kSplit - 1) / kSplit;
            w.st0 += team;
        }
        w.row0 = (int)row0;
        w.rows = rows < BM ? (int)rows : BM;
        w.col0 = tn * BN;
        // A panel past the operand's last one (a tile over the edge) is replaced by the last one: its rows only feed outputs that
        // are not stored.
        const int64_t pa_last = (j.a_rows - 1) / 128, pb_last = (j.b_rows - 1) / 128;
#pragma unroll
        for (int p = 0; p < C::kPanels; ++p) {
            const bool isb = p >= C::kPanelsA;
            const int64_t first = isb ? brow0 : arow0, last = isb ? pb_last : pa_last;
            const int64_t want = first / 128 + (isb ? p - C::kPanelsA : p), panel = want < last ? want : last;
            const int half = kHalf ? (int)((first / 64) & 1) : 0;
            w.gw[p] = (isb ? j.b + b_kb0 * 2048 : j.a) + panel * (isb ? j.b_pld : j.a_pld) + half * 1024;
            const uint8_t* const sp = (isb ? j.bs + b_kb0 * 128 : j.as) + panel * (isb ? j.bs_pld : j.as_pld) + half * 128;
            if (p == 0 || spanel == p) w.gs = sp;
        }
    };
    const uint32_t sc = (uint32_t)(unit % kUnits * C::kScaleLanes + lane);
    const uint32_t lane_s = kHalf ? (sc >> 3) * 256 + (sc & 7) * 16 : sc * 16;
    const uint32_t ls = S::kScales + unit * C::kScaleLanes * 16;
    const uint32_t lane16 = (uint32_t)lane * 16;
    const int kb_last = (int)j.nkb - 1, st_last = kb_last / kStage;  // last block and stage that A (and B from b_kb0) holds

    // Load q of this wave for stage i into the slot at `slot`. In a partial last stage a block that the operand lacks is replaced
    // by the last one; its scales are masked.
    auto issue_one = [&](const Work& w, int q, int i, uint32_t slot) INLINE {
        if (q < C::kWaveCodes) {
            constexpr int kEach = C::kPanelLoads / C::kWaves;  // loads of a panel per wave
            const int p = q / kEach, L = wave * kEach + q % kEach;
            const int kb = (w.st0 + i * kSplit) * kStage + (kHalf ? L : L >> 1);
            to_lds16(lane16 + (uint32_t)(kb < kb_last ? kb : kb_last) * 2048u, w.gw[p] + (kHalf ? 0 : (L & 1) * 1024),
                     ring + slot + (p * C::kPanelLoads + L) * 1024);
        } else {
            const int st = w.st0 + i * kSplit;
            to_lds16_first<C::kScaleLanes>(lane_s + (uint32_t)(kSplit == 1 || st < st_last ? st : st_last) * 512u, w.gs,
                                           ring + slot + ls);
        }
    };
    auto fill = [&](const Work& w) INLINE {  // the first stages
        for (int i = 0; i < kRing && i < w.nst; ++i)
#pragma unroll
            for (int q = 0; q < C::kWaveLoads; ++q) issue_one(w, q, i, i * S::kSize);
    };

    static_assert(kRowsP % (32 * WTM) == 0 && kRowsP % (32 * WTN) == 0, "a wave's rows lie in one panel");
    const unsigned arow = (unsigned)wm * WTM * 32, bcol = (unsigned)wn * WTN * 32;
    const unsigned ap = arow / kRowsP, ar = arow % kRowsP + l32, bp = bcol / kRowsP, br = bcol % kRowsP + l32;
    constexpr int kTiles = WTM * WTN, kOps = WTM + WTN;  // B's WTN operands, then A's WTM
    struct Operands {
        v4i v[kOps];
    };
    struct Scales {
        int v[kOps];
    };
    // what this lane reads of a slot: its row of operand 0, block h
    const uint32_t lb = S::kB + ((bp * kStage + h) * kRowsP + br) * 16, la = ((ap * kStage + h) * kRowsP + ar) * 16;
    const uint32_t lsb = S::kScales + BM * 4 + ((bp * 2 + h) * kRowsP + br) * 2, lsa = S::kScales + ((ap * 2 + h) * kRowsP + ar) * 2;
    auto read_one = [&](int t, uint32_t slot, int ks, Operands& f) INLINE {
        const uint8_t* const p = ring + slot + (t < WTN ? lb : la) + (ks * 2 * kRowsP + (t < WTN ? t : t - WTN) * 32) * 16;
        f.v[t] = *reinterpret_cast<const v4i*>(p);
    };
    auto read_scale = [&](int t, uint32_t slot, Scales& f) INLINE {  // the bytes of both halves
        const uint8_t* const p = ring + slot + (t < WTN ? lsb : lsa) + (t < WTN ? t : t - WTN) * 64;
        f.v[t] = *reinterpret_cast<const uint16_t*>(p);
    };
    // Scales of blocks outside the reduction are 0 (2^-127) on both sides: their products vanish.
    auto mask_scales = [&](const Work& w, int i, Scales& f) INLINE {
        const int kb0 = (w.st0 + i * kSplit) * kStage + h;  // this lane's blocks: kb0 and kb0 + 2
        const int m = (kb0 >= w.kbf && kb0 < w.kbe ? 0x00FF : 0) | (kb0 + 2 >= w.kbf && kb0 + 2 < w.kbe ? 0xFF00 : 0);
#pragma unroll
        for (int t = 0; t < kOps; ++t) f.v[t] &= m;
    };
    // B's rows are the instruction's rows, so that a lane gets runs of consecutive columns of one row of C. Format 4: E2M1.
    v16f acc[WTM][WTN];
    auto multiply_one = [&](int k, const Operands& f, const Scales& s, auto half) INLINE {
        constexpr int byte = decltype(half)::value;
        const int a = k / WTN, b = k % WTN;
        const v4i x = f.v[b], y = f.v[WTN + a];
        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0},
                                                                    v8i{y[0], y[1], y[2], y[3], 0, 0, 0, 0}, acc[a][b], 4, 4, byte,
                                                                    s.v[b], byte, s.v[WTN + a]);
    };

    // Waits until at most OUTSTANDING of this wave's memory operations are in flight and its LDS reads are done, then for every
    // wave: what all have waited for is then visible to all, and nobody reads the stage before any more.
    auto arrive = [&](auto outstanding) INLINE {
        asm volatile("" ::: "memory");
        wait_loads<decltype(outstanding)::value>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // A stage: the first half's products while the second half's operands are read; then, past the barrier that lets the next
    // stage be read and this one be overwritten, the second half's products while the next stage's first half is read and the
    // stage kRing ahead is loaded. The order is pinned: one product, then what its 32 cycles cover. There is no branch inside:
    // the compiler would move products across it. The next stage is stage ni of tile nw, the one loaded (if `loads`) stage li of
    // tile lw. OUTSTANDING: as of arrive() for the next stage, -1 if there is none.
    constexpr int kOpsPer = (kOps + kTiles - 1) / kTiles, kLoadsPer = (C::kWaveLoads + kTiles - 1) / kTiles;
    Operands f0, f1;
    Scales s;
    auto stage = [&](uint32_t cur, uint32_t next, const Work& nw, int ni, auto outstanding, const Work& lw, int li, auto loads) INLINE {
        constexpr bool kMore = decltype(outstanding)::value >= 0, kLoads = decltype(loads)::value;
        Scales sn;
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
            multiply_one(k, f0, s, std::integral_constant<int, 0>{});
#pragma unroll
            for (int t = k * kOpsPer; t < (k + 1) * kOpsPer && t < kOps; ++t) read_one(t, cur, 1, f1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kMore) arrive(outstanding);
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
            multiply_one(k, f1, s, std::integral_constant<int, 1>{});
            if constexpr (kMore) {
#pragma unroll
                for (int t = k * kOpsPer; t < (k + 1) * kOpsPer && t < kOps; ++t) {
                    read_one(t, next, 0, f0);
                    read_scale(t, next, sn);
                }
            }
            if constexpr (kLoads) {
#pragma unroll
                for (int q = k * kLoadsPer; q < (k + 1) * kLoadsPer && q < C::kWaveLoads; ++q) issue_one(lw, q, li, cur);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kMore) {
            mask_scales(nw, ni, sn);
            s = sn;
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
    constexpr int L1 = C::kWaveLoads;
    uint32_t L = blockIdx.x;
    if (L >= total) return;
    Work w;
    locate(L, w);
    fill(w);
    uint32_t cur = 0, next = S::kSize;
    auto advance = [&] INLINE {
        cur = next;
        next = next == (kRing - 1) * S::kSize ? 0 : next + S::kSize;
    };
    auto begin = [&] INLINE {
#pragma unroll
        for (int t = 0; t < kOps; ++t) {
            read_one(t, cur, 0, f0);
            read_scale(t, cur, s);
        }
        mask_scales(w, 0, s);
    };
    using std::integral_constant;
    // The last kRing stages of a tile, whose loads are on their way; nothing follows them.
    auto finish = [&](int i) INLINE {
        static_assert(kRing == 3, "");
        if (i + 2 < w.nst) {
            stage(cur, next, w, i + 1, integral_constant<int, L1>{}, w, 0, std::false_type{});
            advance();
            ++i;
        }
        if (i + 1 < w.nst) {
            stage(cur, next, w, i + 1, integral_constant<int, 0>{}, w, 0, std::false_type{});
            advance();
            ++i;
        }
        stage(cur, next, w, 0, integral_constant<int, -1>{}, w, 0, std::false_type{});
    };

    // The workgroup's tiles, all of as many stages. The stages of one tile follow those of the one before without a gap: its last
    // kRing stages load the next tile's first ones (after the last tile its own first ones again, which nobody reads: a branch here
    // makes the compiler spill the sums), and the last reads the first's operands. A tile's stores are then younger than those
    // loads, and memory operations complete in order, so the next tile's first waits count them in instead of waiting for them.
    // (Filling the ring anew for each tile: 8192 x 8192 x 2048 92 us instead of 79, 98304 x 2048 x 1408 182 instead of 168.)
    if constexpr (kSplit == 1 && MODE != kGemmRaggedK) {
        if (w.nst >= kRing) {
            arrive(integral_constant<int, (kRing - 1) * L1>{});
            begin();
            bool behind = false;  // kStores stores were issued after the loads
            while (true) {
                clear();
                L += gridDim.x;
                const bool more = L < total;
                Work n = w;
                if (more) locate(L, n);
                int i = 0;
                if (behind && w.nst >= 2 * kRing) {
                    for (; i < kRing - 1; ++i) {
                        stage(cur, next, w, i + 1, integral_constant<int, (kRing - 2) * L1 + kStores>{}, w, i + kRing, std::true_type{});
                        advance();
                    }
                }
                for (; i + kRing < w.nst; ++i) {
                    stage(cur, next, w, i + 1, integral_constant<int, (kRing - 2) * L1>{}, w, i + kRing, std::true_type{});
                    advance();
                }
                constexpr integral_constant<int, (kRing - 2) * L1> kept{};
                stage(cur, next, w, i + 1, kept, n, 0, std::true_type{});
                advance();
                stage(cur, next, w, i + 2, kept, n, 1, std::true_type{});
                advance();
                stage(cur, next, n, 0, kept, n, 2, std::true_type{});
                advance();
                asm volatile("" ::: "memory");
                behind = is_inside(w);
                if (behind) store(w, std::true_type{});
                else store(w, std::false_type{});
                if (!more) {
                    wait_loads<0>();  // the LDS must not be another workgroup's before they have landed
                    return;
                }
                w = n;
            }
        }
    }

    // Tiles of different length, or of few stages, or of several teams: one after the other.
    while (true) {
        clear();
        if (w.nst > 0) {
            cur = 0, next = S::kSize;
            arrive(integral_constant<int, 0>{});
            begin();
            int i = 0;
            for (; i + kRing < w.nst; ++i) {
                stage(cur, next, w, i + 1, integral_constant<int, (kRing - 2) * L1>{}, w, i + kRing, std::true_type{});
                advance();
            }
            finish(i);
        }
        L += gridDim.x;
        const bool more = L < total;
        const Work done = w;
        if constexpr (kSplit > 1) {
            // the other teams' sums, added by the first in the order of the teams
            static_assert(kSplit == 1 || (kSplit - 1) * C::kWaves * 64 * kTiles * 16 * 4 <= kSplit * kRing * S::kSize, "");
            float* const sums = reinterpret_cast<float*>(rings) + (wave * 64 + lane) * 4;
            constexpr int kTeam = C::kWaves * 64 * 4, kQuads = kTiles * 4;  // one float4 of every lane; float4s of a lane
            __syncthreads();  // every wave has read the last stage
            if (team > 0) {
#pragma unroll
                for (int k = 0; k < kQuads; ++k) {
                    const v16f& c = acc[k / 4 / WTN][k / 4 % WTN];
                    *reinterpret_cast<float4*>(sums + ((team - 1) * kQuads + k) * kTeam) =
                        make_float4(c[k % 4 * 4], c[k % 4 * 4 + 1], c[k % 4 * 4 + 2], c[k % 4 * 4 + 3]);
                }
            }
            __syncthreads();
            if (team == 0) {
#pragma unroll
                for (int t = 1; t < kSplit; ++t)
#pragma unroll
                    for (int k = 0; k < kQuads; ++k) {
                        v16f& c = acc[k / 4 / WTN][k / 4 % WTN];
                        const float4 v = *reinterpret_cast<const float4*>(sums + ((t - 1) * kQuads + k) * kTeam);
                        c[k % 4 * 4] += v.x;
                        c[k % 4 * 4 + 1] += v.y;
                        c[k % 4 * 4 + 2] += v.z;
                        c[k % 4 * 4 + 3] += v.w;
                    }
            }
        }
        if (more) {
            locate(L, w);
            __syncthreads();  // every wave has read the last stage (the first team: the other teams' sums)
            fill(w);
        }
        asm volatile("" ::: "memory");
        if (kSplit == 1 || team == 0) {
            if (is_inside(done)) store(done, std::true_type{});
            else store(done, std::false_type{});
        }
        if (!more) return;
    }
}

using Tile256 = Tile<4, 2, 2, 4, 3, 1>;      // 256 x 256: 8 waves of 128 x 64, two per SIMD
using Tile128 = Tile<2, 2, 2, 2, 3, 2>;      // 128 x 128: 4 waves of 64 x 64, two workgroups per CU
using Tile64 = Tile<1, 1, 2, 2, 3, 4>;       // 64 x 64: 4 waves of 32 x 32, four workgroups per CU
using Tile64K = Tile<1, 1, 2, 2, 3, 1, 4>;   // 64 x 64 by four teams of 4 waves, each a quarter of the reduction

int64_t grid_tiles(const MxGemmJob& j, int bm, int bn) { return ((j.N + bn - 1) / bn) * tile_rows(j, bm); }

template <int OUT, class C, bool STREAM>
hipError_t launch_tile(const MxGemmJob& j, hipStream_t s) {
    int64_t tiles = grid_tiles(j, C::BM, C::BN);
    if (tiles == 0) return hipSuccess;
    // One workgroup per tile where tiles differ in length (ragged reduction: the next free CU takes the next one); otherwise the
    // workgroups that are resident take the tiles in turn.
    if (j.mode == kGemmRaggedK) tiles *= j.G;
    else if (tiles > C::kResident) tiles = C::kResident;
    switch (j.mode) {
        case kGemmRaggedM: gemm_mxfp4_kernel<OUT, C, kGemmRaggedM, STREAM><<<(unsigned)tiles, C::kThreads, 0, s>>>(j); break;
        case kGemmRaggedK: gemm_mxfp4_kernel<OUT, C, kGemmRaggedK, STREAM><<<(unsigned)tiles, C::kThreads, 0, s>>>(j); break;
        default: gemm_mxfp4_kernel<OUT, C, kGemmDense, STREAM><<<(unsigned)tiles, C::kThreads, 0, s>>>(j); break;
    }
    return hipGetLastError();
}

// Outputs of kStreamBytes and more are stored nontemporally: they cannot stay in a cache, and
// in the L2's recency order they push the operands out. Measured, us, nontemporal / plain: 16384 x 16384 x 2048 bf16 311 / 398,
// fp32 393 / 602 (190 MB read instead of 425), x 512 bf16 150 / 205, 64 experts' 98304 x 1408 x 2048 forward 200 / 251 and weight
// gradient 259 / 322; at 256 MiB 8192 x 8192 fp32 of 1024 74 / 97, of 2048 107 / 99, of 8192 254 / 267; below, 8192 x 8192 x 2048
// bf16 83 / 77. The 64-row tiles store everything plainly: outputs of that size are theirs only where one side is narrow (up to about
// 320 rows or columns, of weight gradients 570: 64 x 2^20 x 128, 256 experts of 192 x 2048 over 64 tokens each).
// A weights' gradient is read when the whole step's have been computed, hundreds of MB later, so it is stored so from 64 MiB on. Whole
// steps (quantizers and the three products), us, nontemporal / plain: 16 experts 4823 x 1920 x 1600 (188 MiB of gradients) 132 / 150, 8
// experts 1602 x 3456 x 1600 (169) 106 / 119, 16508 x 4736 x 1344 (194) 403 / 418, 16 experts 2069 x 7552 x 256 (118) 102 / 106, dense
// 5120 x 6016 x 2976 (68) 202 / 208-214; below 32 MiB the same within 1%. (The 64-row tiles: as above.)
constexpr int64_t kStreamGradBytes = int64_t(64) << 20;
bool streams(const MxGemmJob& j) {
    return j.M * j.N * (j.mode == kGemmRaggedK ? j.G : 1) * (j.out_dtype == kOutF32 ? 4 : 2) >= (j.weight_grad ? kStreamGradBytes : kStreamBytes);
}

// Which tile takes a problem: the one with the smallest estimated time
//     fixed + (R - 1) * again + stages * max(alone, R * busy),
// R the most tiles that one of 256 CUs takes, `alone` the time of a stage (128 of the reduction) on a CU with one tile, `busy`
// what each tile's stage costs where they queue. Microseconds, measured on gfx950; the largest tile moves the fewest bytes per
// product and wins where its tiles fill the chip. Measured, us, 256 / 128 / 64 / 64 in four teams:
//     8192 x 8192 x 2048 78 / 89 / 155 / 266, 8192 x 4096 x 1024 31 / 30 / 46 / 99, 4096^3 36 / 42 / 68 / 100,
//     2048^3 16.3 / 9.5 / 11.3 / 17.9, 256 x 8192 x 2048 15.8 / 9.0 / 7.5 / 10.4, 64 x 2048 x 8192 38 / 20 / 14.8 / 11.7,
//     256 x 256 x 32768 133 / 67 / 49 / 33.
// The four teams are bound by what one CU can load (64 bytes a clock); more would need sums across workgroups.
enum { kTile256, kTile128, kTile64, kTile64K, kKernels };
struct Cost {
    int tile, threads;
    double fixed, again, alone, busy;
};
constexpr Cost kCost[kKernels] = {
    {Tile256::BM, Tile256::kThreads, 9.0, 4.5, 0.48, 0.85},
    {Tile128::BM, Tile128::kThreads, 6.2, 0.75, 0.24, 0.30},
    {Tile64::BM, Tile64::kThreads, 5.4, 0.2, 0.15, 0.115},
    {Tile64K::BM, Tile64K::kThreads, 6.2, 3.0, 0.10, 0.10},
};

int pick_tile(const MxGemmJob& j) {
    const int64_t groups = j.mode == kGemmRaggedK ? j.G : 1;
    const int64_t blocks = j.mode == kGemmRaggedK ? (j.nkb + j.G - 1) / j.G : j.nkb;  // ragged reduction: an average group
    const double stages = (double)((blocks + kStage - 1) / kStage);
    int best = kTile256;
    double best_us = 0.0;
    for (int k = 0; k < kKernels; ++k) {
        const Cost& c = kCost[k];
        const int64_t tiles = grid_tiles(j, c.tile, c.tile) * groups;
        // a grid holds fewer than 2^32 threads: what fits with the largest tile must not fail on a smaller one's grid
        if (k != kTile256 && tiles * c.threads > int64_t(UINT32_MAX)) continue;
        // Ragged rows: the operand is padded to panels, and every other group leaves half of a 256-row tile empty.
        const double rows = j.mode == kGemmRaggedM ? (double)j.a_rows / c.tile + (c.tile > 128 ? j.G / 4.0 : 0.0) : 0.0;
        const double some = j.mode == kGemmRaggedM ? rows * (double)((j.N + c.tile - 1) / c.tile) : (double)tiles;
        const double R = ceil(some / 256.0);
        const double us = c.fixed + (R - 1.0) * c.again + stages * (R * c.busy > c.alone ? R * c.busy : c.alone);
        if (k == 0 || us < best_us) {
            best = k;
            best_us = us;
        }
    }
    return best;
}

template <int OUT>
hipError_t launch_out(const MxGemmJob& j, hipStream_t s) {
    switch (pick_tile(j)) {
        case kTile256: return streams(j) ? launch_tile<OUT, Tile256, true>(j, s) : launch_tile<OUT, Tile256, false>(j, s);
        case kTile128: return streams(j) ? launch_tile<OUT, Tile128, true>(j, s) : launch_tile<OUT, Tile128, false>(j, s);
        case kTile64: return launch_tile<OUT, Tile64, false>(j, s);
        default: return launch_tile<OUT, Tile64K, false>(j, s);
    }
}

}  // namespace

hipError_t launch_gemm_mxfp4(const MxGemmJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_out<kOutBF16>(j, s) : launch_out<kOutF32>(j, s);
}

}  // namespace ufp4

extern "C" int ufp4_plan_gemm_mxfp4(int mode, int64_t M, int64_t N, int64_t red, int32_t G, int64_t a_rows) {
    ufp4::MxGemmJob j{};
    j.mode = mode;
    j.M = M;
    j.N = N;
    j.nkb = red / 32;
    j.G = G;
    j.a_rows = a_rows;
    return ufp4::pick_tile(j);
}
