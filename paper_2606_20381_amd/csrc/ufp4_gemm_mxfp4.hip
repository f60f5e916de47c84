// GEMM on microscaled 4-bit operands: C[i, j] = sum_k A[i,k] 2^(eA[i,k/32] - 127) B[j,k] 2^(eB[j,k/32] - 127), A and B E2M1
// levels in the layout of ufp4_mxfp4.hip, sums in fp32 by v_mfma_scale_f32_32x32x64_f8f6f4, which applies both scales.
//
// A lane of the instruction holds the 32 codes of one row and one 32-block: 16 bytes, one LDS read. K advances 128 (four
// blocks) per stage; a panel's stage is 8 KiB of codes and 512 bytes of scales, both contiguous, copied unchanged into a
// four-deep LDS ring by direct-to-LDS loads. Each wave keeps two sets of operands in registers: while the matrix core works
// on one half of a stage, the other half (or, past the barrier, the next stage's first half) is read from LDS, so that
// neither the barrier nor the LDS latency stands between two matrix instructions.

#include "ufp4_internal.h"
#include "ufp4_mxfp4.h"

#include <type_traits>

namespace ufp4 {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kStage = 4;  // 32-blocks per stage
constexpr int kRing = 4;   // stages in LDS

// WM x WN waves, each with WTM x WTN matrix tiles of 32 x 32 outputs.
template <int WTM_, int WTN_, int WM_, int WN_, int PER_CU>
struct Tile {
    static constexpr int WTM = WTM_, WTN = WTN_, WM = WM_, WN = WN_;
    static constexpr int BM = 32 * WTM * WM, BN = 32 * WTN * WN;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int kPerEU = PER_CU * kWaves / 4;  // waves per SIMD that the registers have to allow
    static constexpr int kLoadsA = BM / 16, kLoadsB = BN / 16;  // 1 KiB direct-to-LDS loads per stage
    static constexpr int kWaveCodes = (kLoadsA + kLoadsB) / kWaves;
    static constexpr int kScaleLanes = (BM + BN) / 4 / kWaves;  // 16-byte pieces of scales per wave and stage
    static constexpr int kWaveLoads = kWaveCodes + 1;
    static_assert(BM == BN && (kLoadsA + kLoadsB) % kWaves == 0 && kWaves % 2 == 0, "every wave issues the same loads");
    static_assert(kScaleLanes <= 64 && kWaveLoads * (kRing - 1) < 64, "one scale load per wave; vmcnt has six bits");
};

template <class C>
struct Slot {
    uint8_t a[C::BM * 64];  // [panel][block][row] 16 bytes, as in memory; of a 64-row tile [block][row]
    uint8_t b[C::BN * 64];
    uint8_t s[(C::BM + C::BN) * 4];  // A's, then B's [panel][block % 2][row][2]
};

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

__device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Workgroup -> output tile. Workgroups go to the 8 XCDs round robin, and each XCD has its own L2: the first 8 floor(T / 8)
// are renumbered so that XCD k gets one run of T / 8 tiles, in bands of kBand tile rows, column by column within a band.
constexpr int kBand = 8;
__device__ __forceinline__ void tile_at(int64_t L, int64_t gy, int64_t gx, int64_t& tm, int64_t& tn) {
    const int64_t T = gx * gy, per = T / 8;
    const int64_t t = L < 8 * per ? (L % 8) * per + L / 8 : L;
    const int64_t band = t / (kBand * gx), first = band * kBand;
    const int64_t rows = gy - first < kBand ? gy - first : kBand;
    const int64_t r = t - first * gx;
    tm = first + r % rows;
    tn = r / rows;
}

// Tile rows of the grid; ragged-M: a bound over all groups, each of which may end in a partial tile.
__host__ __device__ inline int64_t tile_rows(const MxGemmJob& j, int bm) {
    return j.mode == kGemmRaggedM ? (j.a_rows + bm - 1) / bm + j.G : (j.M + bm - 1) / bm;
}

// Ragged-M: the group of tile row t, with its first row among the padded rows (groups start on panels) and the tokens.
struct GroupTile {
    int64_t g, prow, trow, rows;
};
template <int BM>
__device__ __forceinline__ bool group_tile(const MxGemmJob& j, int64_t t, GroupTile& r) {
    const int lane = threadIdx.x & 63;
    int64_t tiles = 0, pads = 0;
    for (int g0 = 0; g0 < j.G; g0 += 64) {
        const int g = g0 + lane;
        const int64_t start = g < j.G ? j.offsets[g] : 0;
        int64_t m = g < j.G ? j.offsets[g + 1] - start : 0;
        if (m < 0) m = 0;
        const int64_t cnt = (m + BM - 1) / BM, pad = (m + 127) / 128 * 128;
        int64_t ti = cnt, pi = pad;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t vt = __shfl_up(ti, d, 64), vp = __shfl_up(pi, d, 64);
            if (lane >= d) {
                ti += vt;
                pi += vp;
            }
        }
        const int64_t te = tiles + ti - cnt;
        const uint64_t hit = __ballot(te <= t && t < te + cnt);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            const int64_t lt = t - __shfl(te, at, 64);
            r.g = g0 + at;
            r.prow = __shfl(pads + pi - pad, at, 64) + lt * BM;
            r.trow = __shfl(start, at, 64) + lt * BM;
            r.rows = __shfl(m, at, 64) - lt * BM;
            return true;
        }
        tiles += __shfl(ti, 63, 64);
        pads += __shfl(pi, 63, 64);
    }
    return false;
}

// Ragged-K: the first 32-block of group g along the padded reduction, and its blocks.
__device__ __forceinline__ void group_blocks(const int64_t* off, int g, int64_t& first, int64_t& n) {
    const int lane = threadIdx.x & 63;
    int64_t sum = 0;
    for (int h = lane; h < g; h += 64) {
        const int64_t c = off[h + 1] - off[h];
        sum += c > 0 ? (c + 31) / 32 : 0;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
    first = sum;
    const int64_t c = off[g + 1] - off[g];
    n = c > 0 ? (c + 31) / 32 : 0;
}

template <int OUT, class C>
__global__ __launch_bounds__(C::kThreads, C::kPerEU) void gemm_mxfp4_kernel(MxGemmJob j) {
    // separate objects: loads in flight into one do not alias reads of another
    __shared__ Slot<C> sm0, sm1, sm2, sm3;
    constexpr int BM = C::BM, BN = C::BN, WTM = C::WTM, WTN = C::WTN;
    constexpr bool kHalf = BM < 128;                  // half a panel per operand
    constexpr int kRowsP = kHalf ? BM : 128;          // rows of a panel in LDS
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31;
    const int wm = (int)((unsigned)wave / C::WN), wn = (int)((unsigned)wave % C::WN);
    int64_t tm, tn;
    tile_at(blockIdx.x, tile_rows(j, BM), (j.N + BN - 1) / BN, tm, tn);
    // A rows from arow0 and B rows from brow0; blocks kb_first .. kb_end - 1 of A (B's lie b_kb0 further); output rows out_row0
    // .. out_row0 + mrows - 1 at c_base
    int64_t arow0 = tm * BM, brow0 = tn * BN, b_kb0 = 0, kb_first = 0, kb_end = j.nkb;
    int64_t out_row0 = tm * BM, mrows = j.M - tm * BM, c_base = 0;
    if (j.mode == kGemmRaggedM) {
        GroupTile r;
        if (!group_tile<BM>(j, tm, r)) return;  // the whole workgroup agrees
        arow0 = r.prow;
        out_row0 = r.trow;
        mrows = r.rows < j.M - r.trow ? r.rows : j.M - r.trow;  // token rows past the output are not stored
        if (r.trow < 0) mrows = 0;
        brow0 = r.g * j.b_group_rows + tn * BN;
        b_kb0 = r.g * j.b_group_kb;
    } else if (j.mode == kGemmRaggedK) {
        int64_t n;
        group_blocks(j.offsets, (int)blockIdx.y, kb_first, n);
        kb_end = kb_first + n < j.nkb ? kb_first + n : j.nkb;  // clamped to the operands
        c_base = (int64_t)blockIdx.y * j.M * j.ldc;
    }
    arow0 = uniform64(arow0);
    brow0 = uniform64(brow0);
    b_kb0 = uniform64(b_kb0);
    const int kbf = (int)uniform64(kb_first), kbe = (int)uniform64(kb_end);
    // Stages are whole groups of four blocks (the scales' unit). A ragged reduction may begin and end inside one: the scales
    // of blocks outside are taken as 0 (2^-127) on both sides, so that their products vanish. Elsewhere the reduction
    // begins at 0, and the quantizers wrote 0 for the scales that fill up its last group.
    const int st0 = kbf / kStage;
    const int nst = kbe > kbf ? (kbe + kStage - 1) / kStage - st0 : 0;
    // The tile's panels. One past the operand's last (a tile over the edge) is replaced by the last one: its rows only feed
    // outputs that are not stored.
    const int64_t pa_last = (j.a_rows - 1) / 128, pb_last = (j.b_rows - 1) / 128;
    const int64_t pa0 = arow0 / 128 < pa_last ? arow0 / 128 : pa_last, pb0 = brow0 / 128 < pb_last ? brow0 / 128 : pb_last;
    const int64_t pa1 = pa0 + 1 < pa_last ? pa0 + 1 : pa_last, pb1 = pb0 + 1 < pb_last ? pb0 + 1 : pb_last;
    const int a_half = kHalf ? (int)((arow0 / 64) & 1) : 0, b_half = kHalf ? (int)((brow0 / 64) & 1) : 0;
    const uint8_t* const ga0 = j.a + pa0 * j.a_pld + a_half * 1024;
    const uint8_t* const ga1 = j.a + pa1 * j.a_pld;
    const uint8_t* const gb0 = j.b + pb0 * j.b_pld + b_kb0 * 2048 + b_half * 1024;
    const uint8_t* const gb1 = j.b + pb1 * j.b_pld + b_kb0 * 2048;
    // this wave's scales: pieces sc0 .. of its operand (the first half of the waves take A's)
    const int sop = wave >= C::kWaves / 2;
    const int sc0 = (wave - sop * (C::kWaves / 2)) * C::kScaleLanes;
    const int spanel = kHalf ? 0 : sc0 / 32;
    const uint8_t* const gs = sop == 0 ? j.as + (spanel ? pa1 : pa0) * j.as_pld + a_half * 128
                                       : j.bs + (spanel ? pb1 : pb0) * j.bs_pld + b_kb0 * 128 + b_half * 128;
    const int kb_last = (int)j.nkb - 1;  // last block that A (and B from b_kb0) holds

    auto issue = [&](int i, Slot<C>& d) {
        const int kb0 = (st0 + i) * kStage;
#pragma unroll
        for (int q = 0; q < C::kWaveCodes; ++q) {
            const int all = q * C::kWaves + wave;
            const bool isb = C::kLoadsA % C::kWaves == 0 ? q >= C::kLoadsA / C::kWaves : all >= C::kLoadsA;
            const int L = isb ? all - C::kLoadsA : all;
            const int blk = kHalf ? L : (L & 7) >> 1;
            const int kb = kb0 + blk < kb_last ? kb0 + blk : kb_last;  // past the reduction: any codes, their scales are 0
            const uint8_t* const g = kHalf || L < 8 ? (isb ? gb0 : ga0) : (isb ? gb1 : ga1);
            to_lds16((uint32_t)lane * 16, g + (int64_t)kb * 2048 + (kHalf ? 0 : (L & 1) * 1024), (isb ? d.b : d.a) + L * 1024);
        }
        if (lane < C::kScaleLanes) {
            const int c = sc0 + lane;
            const uint32_t at = kHalf ? (uint32_t)((c >> 3) * 256 + (c & 7) * 16) : (uint32_t)((c & 31) * 16);
            to_lds16(at, gs + (int64_t)(st0 + i) * 512, d.s + sop * BM * 4 + sc0 * 16);
        }
    };

    v16f acc[WTM][WTN];
#pragma unroll
    for (int a = 0; a < WTM; ++a)
#pragma unroll
        for (int b = 0; b < WTN; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;

    static_assert(kRowsP % (32 * WTM) == 0 && kRowsP % (32 * WTN) == 0, "a wave's rows lie in one panel");
    const unsigned arow = (unsigned)wm * WTM * 32, bcol = (unsigned)wn * WTN * 32;
    const unsigned ap = arow / kRowsP, ar = arow % kRowsP + l32, bp = bcol / kRowsP, br = bcol % kRowsP + l32;

    struct Operands {
        v8i a[WTM], b[WTN];
    };
    struct Scales {
        int a[WTM], b[WTN];
    };
    auto read = [&](const Slot<C>& d, int ks, Operands& f) {
        auto one = [](const uint8_t* p) {
            const uint4 x = *reinterpret_cast<const uint4*>(p);
            const v8i v = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
            return v;
        };
#pragma unroll
        for (int b = 0; b < WTN; ++b) f.b[b] = one(d.b + ((bp * kStage + 2 * ks + h) * kRowsP + br + b * 32) * 16);
#pragma unroll
        for (int a = 0; a < WTM; ++a) f.a[a] = one(d.a + ((ap * kStage + 2 * ks + h) * kRowsP + ar + a * 32) * 16);
    };
    auto read_scales = [&](const Slot<C>& d, int i, Scales& f) {
        constexpr int kS = kRowsP * 2;  // bytes of one half
#pragma unroll
        for (int b = 0; b < WTN; ++b)
            f.b[b] = *reinterpret_cast<const uint16_t*>(d.s + BM * 4 + (bp * 2 + h) * kS + (br + b * 32) * 2);
#pragma unroll
        for (int a = 0; a < WTM; ++a)
            f.a[a] = *reinterpret_cast<const uint16_t*>(d.s + (ap * 2 + h) * kS + (ar + a * 32) * 2);
        const int kb0 = (st0 + i) * kStage + h;  // this lane's blocks: kb0 and kb0 + 2
        if (j.mode == kGemmRaggedK && ((st0 + i) * kStage < kbf || (st0 + i + 1) * kStage > kbe)) {
            const int m = (kb0 >= kbf && kb0 < kbe ? 0x00FF : 0) | (kb0 + 2 >= kbf && kb0 + 2 < kbe ? 0xFF00 : 0);
#pragma unroll
            for (int b = 0; b < WTN; ++b) f.b[b] &= m;
#pragma unroll
            for (int a = 0; a < WTM; ++a) f.a[a] &= m;
        }
    };
    auto multiply = [&](const Operands& f, const Scales& s, auto half) {
        constexpr int kHalfStage = decltype(half)::value;  // byte of the scales
#pragma unroll
        for (int a = 0; a < WTM; ++a)
#pragma unroll
            for (int b = 0; b < WTN; ++b)  // format 4: E2M1 for both operands
                acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.a[a], f.b[b], acc[a][b], 4, 4, kHalfStage, s.a[a],
                                                                            kHalfStage, s.b[b]);
    };
    // Waits for this wave's loads of stage i (those of up to kRing - 2 later stages stay in flight) and its LDS reads, then for
    // every wave: stage i is then visible to all, and nobody reads stage i - 1 any more.
    auto arrive = [&](int i) {
        const int later = nst - 1 - i;
        asm volatile("" ::: "memory");
        if (later >= 2) wait_loads<2 * C::kWaveLoads>();
        else if (later == 1) wait_loads<C::kWaveLoads>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    Operands f0, f1;
    Scales s0, s1;
    auto stage = [&](int i, Slot<C>& cur, Slot<C>& next) {
        read(cur, 1, f1);
        multiply(f0, s0, std::integral_constant<int, 0>{});
        s1 = s0;
        if (i + 1 < nst) {
            arrive(i + 1);
            if (i + kRing < nst) issue(i + kRing, cur);
            read(next, 0, f0);
            read_scales(next, i + 1, s0);
        }
        multiply(f1, s1, std::integral_constant<int, 1>{});
    };

    if (nst > 0) {
        issue(0, sm0);
        if (nst > 1) issue(1, sm1);
        if (nst > 2) issue(2, sm2);
        if (nst > 3) issue(3, sm3);
        if (nst > 3) {
            asm volatile("" ::: "memory");
            wait_loads<3 * C::kWaveLoads>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        } else {
            arrive(0);
        }
        read(sm0, 0, f0);
        read_scales(sm0, 0, s0);
        for (int i = 0; i < nst; i += 4) {
            stage(i, sm0, sm1);
            if (i + 1 < nst) stage(i + 1, sm1, sm2);
            if (i + 2 < nst) stage(i + 2, sm2, sm3);
            if (i + 3 < nst) stage(i + 3, sm3, sm0);
        }
    }

    // Lane (l32, h) holds rows 8q + 4h + t (q, t < 4) of column l32 of each 32 x 32 tile.
    const int64_t N = j.N, ldc = j.ldc;
    auto store = [&](int64_t row, int64_t col, float v) {
        const int64_t off = c_base + row * ldc + col;
        if constexpr (OUT == kOutF32) static_cast<float*>(j.c)[off] = v;
        else static_cast<uint16_t*>(j.c)[off] = __builtin_bit_cast(uint16_t, (__bf16)v);
    };
    const bool inside = mrows >= BM && (tn + 1) * BN <= N;
#pragma unroll
    for (int a = 0; a < WTM; ++a) {
#pragma unroll
        for (int b = 0; b < WTN; ++b) {
            const int64_t col = tn * BN + (wn * WTN + b) * 32 + l32;
            const int64_t lr0 = (wm * WTM + a) * 32 + 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t lr = lr0 + 8 * (i >> 2) + (i & 3);
                if (inside || (col < N && lr < mrows)) store(out_row0 + lr, col, acc[a][b][i]);
            }
        }
    }
}

using Tile256 = Tile<4, 4, 2, 2, 1>;  // 256 x 256: 4 waves of 128 x 128, one per SIMD
using Tile128 = Tile<2, 2, 2, 2, 2>;  // 128 x 128: 4 waves of 64 x 64, two workgroups per CU
using Tile64 = Tile<1, 1, 2, 2, 4>;   // 64 x 64: 4 waves of 32 x 32, four workgroups per CU

int64_t grid_tiles(const MxGemmJob& j, int bm) { return ((j.N + bm - 1) / bm) * tile_rows(j, bm); }

template <int OUT, class C>
hipError_t launch_tile(const MxGemmJob& j, hipStream_t s) {
    const int64_t tiles = grid_tiles(j, C::BM);
    if (tiles == 0) return hipSuccess;
    gemm_mxfp4_kernel<OUT, C><<<dim3((unsigned)tiles, j.mode == kGemmRaggedK ? (unsigned)j.G : 1u), C::kThreads, 0, s>>>(j);
    return hipGetLastError();
}

enum { kTile256, kTile128, kTile64 };

int pick_tile(const MxGemmJob& j) {
    const int64_t groups = j.mode == kGemmRaggedK ? j.G : 1;
    if (grid_tiles(j, 256) * groups >= 200) return kTile256;
    if (grid_tiles(j, 128) * groups >= 256) return kTile128;
    return kTile64;
}

template <int OUT>
hipError_t launch_out(const MxGemmJob& j, hipStream_t s) {
    switch (pick_tile(j)) {
        case kTile256: return launch_tile<OUT, Tile256>(j, s);
        case kTile128: return launch_tile<OUT, Tile128>(j, s);
        default: return launch_tile<OUT, Tile64>(j, s);
    }
}

}  // namespace

hipError_t launch_gemm_mxfp4(const MxGemmJob& j, hipStream_t s) {
    return j.out_dtype == kOutBF16 ? launch_out<kOutBF16>(j, s) : launch_out<kOutF32>(j, s);
}

}  // namespace ufp4
