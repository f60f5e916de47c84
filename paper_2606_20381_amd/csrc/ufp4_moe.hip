// Tokens sorted by expert and back.
//
// sort: ids [T, k] -> every slot (t, j)'s place in the order by (expert, t, j). A stable counting sort of n = T k slots by E
//   keys, in runs of kRun slots per workgroup. Within a wave the slots of one expert find each other by ballots over the
//   bits of the key, so a slot's rank is a count of lanes and no atomic decides an order.
// dispatch: out[rows[t, j]] = w[t, j] x[t]; combine: out[t] = sum_j w[t, j] y[rows[t, j]]; each the other's adjoint.
// combine_bwd: dy[rows[t, j]] = w[t, j] dout[t] and dw[t, j] = <dout[t], y[rows[t, j]]> from one read of both.
//   All three are HBM bound: a wave takes one token, or a 4 KiB segment of one, reads its row once for all k experts and sums in
//   fp32. Short rows (one or two 16-byte pieces a lane) leave registers for several of a token's rows at a time, without which a
//   token takes k times a read's latency: 32768 tokens x 8 x 128 bf16 dispatch 53 -> 22 us, combine 61 -> 26. The gradient of
//   longer rows (more than a segment) takes a workgroup per token, of few tokens one per slot.
//
// Measured, 16384 tokens to 6 of 64 experts, 2048 bf16 columns: sort 4.7 + 7.7 us (two launches of 24 workgroups, bound by their
// own latency), dispatch 78 us and combine 80 us (470 MB each: 5.9 TB/s; a copy of 1 GiB runs at 5.1), combine_bwd 172 us (873 MB:
// 5.1 TB/s; among a layer step's other kernels 189; 5003 x 2 x 5120 fp32 91 us, 512 MB: 5.6 TB/s).

#include "ufp4_internal.h"
#include "ufp4_rows.h"

#include <type_traits>

namespace ufp4 {

namespace {

// ------------------------------------------------------------------------------------------------
// sort
// ------------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kRounds = 4;                       // slots per thread
constexpr int kRun = kSortThreads * kRounds;     // slots per workgroup
constexpr int kWaveRun = 64 * kRounds;           // contiguous slots per wave

// Expert of slot i, E where it has none (or lies past the last slot).
__device__ __forceinline__ int sort_key(const MoeSortJob& j, int64_t i) {
    if (i >= j.n) return j.E;
    const int64_t id = j.ids64 ? static_cast<const int64_t*>(j.ids)[i] : static_cast<const int32_t*>(j.ids)[i];
    return id >= 0 && id < j.E ? (int)id : j.E;
}

// Each workgroup's slots per expert: counts [workgroup][E].
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(MoeSortJob j) {
    extern __shared__ int32_t s_count[];  // [E]
    for (int e = threadIdx.x; e < j.E; e += kSortThreads) s_count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kRun;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int key = sort_key(j, first + r * kSortThreads + threadIdx.x);
        if (key < j.E) atomicAdd(&s_count[key], 1);  // a count: the order of the additions does not show
    }
    __syncthreads();
    for (int e = threadIdx.x; e < j.E; e += kSortThreads) j.counts[(int64_t)blockIdx.x * j.E + e] = s_count[e];
}

// Counts of many workgroups: an exclusive sum over the workgroups per expert, in place, and the totals in row `runs`.
// One wave per expert, 64 workgroups at a time.
__global__ __launch_bounds__(256) void sort_scan_kernel(MoeSortJob j) {
    const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e >= j.E) return;
    int32_t base = 0;
    for (int64_t b0 = 0; b0 < j.runs; b0 += 64) {
        const int64_t b = b0 + lane;
        const int32_t c = b < j.runs ? j.counts[b * j.E + e] : 0;
        int32_t inc = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t v = __shfl_up(inc, d, 64);
            if (lane >= d) inc += v;
        }
        if (b < j.runs) j.counts[b * j.E + e] = base + inc - c;
        base += __shfl(inc, 63, 64);
    }
    if (lane == 0) j.counts[j.runs * j.E + e] = base;
}

// Places. MANY: the counts have been summed over the workgroups (sort_scan_kernel); otherwise the workgroup adds them up
// itself, or (one workgroup) they are its own.
template <bool MANY>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(MoeSortJob j) {
    extern __shared__ char s_raw[];
    const int E = j.E;
    int32_t* const s_base = reinterpret_cast<int32_t*>(s_raw);        // [E] first place of this workgroup's slots
    int32_t* const s_total = s_base + E;                              // [E] slots in all workgroups
    uint16_t* const s_wave = reinterpret_cast<uint16_t*>(s_total + E);  // [wave][E] slots, then their exclusive sum
    __shared__ int32_t s_scan[kSortWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t first = (int64_t)blockIdx.x * kRun + wave * kWaveRun;
    int key[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) key[r] = sort_key(j, first + r * 64 + lane);
    for (int i = tid; i < kSortWaves * E; i += kSortThreads) s_wave[i] = 0;
    if (!MANY && j.runs > 1)
        for (int e = tid; e < E; e += kSortThreads) s_base[e] = s_total[e] = 0;
    __syncthreads();
    if (!MANY && j.runs > 1) {  // a workgroup's counts per wave (integers: the order of the additions does not show)
        for (int64_t b = wave; b < j.runs; b += kSortWaves)
            for (int e = lane; e < E; e += 64) {
                const int32_t c = j.counts[b * E + e];
                if (c == 0) continue;
                atomicAdd(&s_total[e], c);
                if (b < blockIdx.x) atomicAdd(&s_base[e], c);
            }
    }
    int bits = 0;
    while ((1 << bits) <= E) ++bits;
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        uint64_t peers = ~0ull;  // the lanes with this lane's key
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((key[r] >> b) & 1);
            peers &= (key[r] >> b) & 1 ? set : ~set;
        }
        rank[r] = 0;
        if (key[r] < E) {
            volatile uint16_t* const c = s_wave + wave * E + key[r];  // other lanes of the wave write it between the rounds
            const int before = *c;
            rank[r] = before + __popcll(peers & below);
            if ((peers & below) == 0) *c = (uint16_t)(before + __popcll(peers));  // one lane per key, after all have read
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();

    // Per expert: the waves' counts to their exclusive sum; the slots of this expert in earlier workgroups and in all.
    // A thread takes expert tid (E <= kSortThreads).
    int32_t before = 0, total = 0;
    if (tid < E) {
        int32_t own = 0;
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t c = s_wave[w * E + tid];
            s_wave[w * E + tid] = (uint16_t)own;
            own += c;
        }
        if constexpr (MANY) {
            before = j.counts[(int64_t)blockIdx.x * E + tid];
            total = j.counts[j.runs * E + tid];
        } else if (j.runs > 1) {
            before = s_base[tid];
            total = s_total[tid];
        } else {
            total = own;
        }
    }
    // exclusive sum of the totals over the experts
    int32_t inc = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t v = __shfl_up(inc, d, 64);
        if (lane >= d) inc += v;
    }
    if (lane == 63) s_scan[wave] = inc;
    __syncthreads();
    int32_t waves = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        if (w < wave) waves += s_scan[w];
        all += s_scan[w];
    }
    const int32_t start = waves + inc - total;
    if (tid < E) {
        s_base[tid] = start + before;
        if (blockIdx.x == 0) j.offsets[tid] = start;
    }
    if (blockIdx.x == 0 && tid == 0) j.offsets[E] = all;
    __syncthreads();

#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = first + r * 64 + lane;
        if (i < j.n) {
            int32_t place = -1;
            if (key[r] < E) {
                place = s_base[key[r]] + s_wave[wave * E + key[r]] + rank[r];
                if (j.source) j.source[place] = (int32_t)i;
            }
            j.rows[i] = place;
            if (j.source && i >= all) j.source[i] = -1;  // places that no slot takes
        }
    }
}

// ------------------------------------------------------------------------------------------------
// dispatch, combine
// ------------------------------------------------------------------------------------------------
constexpr int kSegPieces = 4;  // 16-byte pieces per lane of a segment: 4 KiB per wave

// out rows [first, rows_out) zero, in segments: the rows that no slot takes. Called by every wave of a grid of `tokens` waves
// per segment.
template <typename T, int PIECES>
__device__ __forceinline__ void zero_rows(T* out, int64_t ldo, int64_t first, int64_t rows_out, int64_t token, int64_t tokens,
                                          int64_t c0, int64_t cols) {
    using P = Piece<T>;
    const u32x4_any zero = {0, 0, 0, 0};
    for (int64_t r = (first < 0 ? 0 : first) + token; r < rows_out; r += tokens)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int64_t c = c0 + p * 64 * P::V;
            P::store(out + r * ldo + c, cols - c, zero);
        }
}

// A token's rows and weights, one a lane (k <= 64), all read at once: row(q) is -1 for a slot that has none. Every lane of the wave
// takes part.
struct Slots {
    int32_t mine;
    float w;
    __device__ __forceinline__ Slots(const int32_t* rows, const float* weights, int64_t t, int k, int64_t rows_y) {
        const int lane = threadIdx.x & 63;
        const int32_t r = lane < k ? rows[t * k + lane] : -1;
        mine = r < rows_y ? r : -1;
        w = weights && lane < k ? weights[t * k + lane] : 1.0f;
    }
    __device__ __forceinline__ int32_t row(int q) const { return __builtin_amdgcn_readlane(mine, q); }
    __device__ __forceinline__ float weight(int q) const {
        return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), q));
    }
};

// A wave takes PIECES pieces a lane of a token.
template <typename T, bool STREAM, int PIECES>
__global__ __launch_bounds__(256) void dispatch_kernel(MoeRowsJob j) {
    using P = Piece<T>;
    constexpr int V = P::V;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= j.tokens * j.segs) return;
    const int64_t t = item / j.segs, c0 = (item - t * j.segs) * (PIECES * 64 * V) + (threadIdx.x & 63) * V;
    const T* const x = static_cast<const T*>(j.in) + t * j.ldi;
    T* const out = static_cast<T*>(j.out);
    const int64_t used = j.offsets[j.E];
    const Slots slots(j.rows, j.w, t, j.k, j.rows_y);
    u32x4_any raw[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int64_t c = c0 + p * 64 * V;
        raw[p] = P::load(x + c, j.cols - c);
    }
    for (int q = 0; q < j.k; ++q) {
        const int32_t row = slots.row(q);
        if (row < 0) continue;
        const float w = slots.weight(q);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int64_t c = c0 + p * 64 * V;
            u32x4_any r = raw[p];
            if (j.w) {
                float f[V];
                P::unpack(r, f);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= w;
                r = P::pack(f);
            }
            P::template store<STREAM>(out + row * j.ldo + c, j.cols - c, r);
        }
    }
    zero_rows<T, PIECES>(out, j.ldo, used, j.rows_y, t, j.tokens, c0, j.cols);
}

// A wave takes PIECES pieces a lane of a token and reads kSegPieces / PIECES of its rows at a time: short rows leave the registers
// for it, and need it (a row after the other is k times a read's latency).
template <typename T, bool STREAM, int PIECES>
__global__ __launch_bounds__(256) void combine_kernel(MoeRowsJob j) {
    using P = Piece<T>;
    constexpr int V = P::V, kAtOnce = kSegPieces / PIECES;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= j.tokens * j.segs) return;
    const int64_t t = item / j.segs, c0 = (item - t * j.segs) * (PIECES * 64 * V) + (threadIdx.x & 63) * V;
    const T* const y = static_cast<const T*>(j.in);
    const Slots slots(j.rows, j.w, t, j.k, j.rows_y);
    float acc[PIECES][V];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[p][i] = 0.0f;
    for (int q0 = 0; q0 < j.k; q0 += kAtOnce) {
        u32x4_any raw[kAtOnce][PIECES];
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int32_t row = q0 + s < j.k ? slots.row(q0 + s) : -1;
            if (row < 0) continue;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int64_t c = c0 + p * 64 * V;
                raw[s][p] = P::template load<STREAM>(y + row * j.ldi + c, j.cols - c);
            }
        }
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            if (q0 + s >= j.k || slots.row(q0 + s) < 0) continue;
            const float w = slots.weight(q0 + s);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                float f[V];
                P::unpack(raw[s][p], f);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[p][i] = __builtin_fmaf(w, f[i], acc[p][i]);
            }
        }
    }
    T* const out = static_cast<T*>(j.out) + t * j.ldo;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int64_t c = c0 + p * 64 * V;
        P::store(out + c, j.cols - c, P::pack(acc[p]));
    }
}

// The combine's gradient for rows that a wave holds in PIECES pieces a lane: a wave per token, rows read as above.
template <typename T, bool STREAM, int PIECES>
__global__ __launch_bounds__(256) void combine_bwd_wave_kernel(MoeBwdJob j) {
    using P = Piece<T>;
    constexpr int V = P::V, kAtOnce = kSegPieces / PIECES;
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= j.tokens) return;
    const T* const dout = static_cast<const T*>(j.dout) + t * j.lddo;
    const T* const y = static_cast<const T*>(j.y);
    T* const dy = static_cast<T*>(j.dy);
    const int64_t used = j.offsets[j.E];
    const Slots slots(j.rows, j.w, t, j.k, j.rows_y);
    u32x4_any raw[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int64_t c = (p * 64 + lane) * V;
        raw[p] = P::load(dout + c, j.cols - c);
    }
    float dots = 0.0f;  // lane q: slot q's
    for (int q0 = 0; q0 < j.k; q0 += kAtOnce) {
        u32x4_any ry[kAtOnce][PIECES];
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int32_t row = q0 + s < j.k ? slots.row(q0 + s) : -1;
            if (row < 0) continue;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int64_t c = (p * 64 + lane) * V;
                ry[s][p] = P::load(y + row * j.ldy + c, j.cols - c);
            }
        }
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int32_t row = q0 + s < j.k ? slots.row(q0 + s) : -1;
            if (row < 0) continue;
            const float w = slots.weight(q0 + s);
            float dot = 0.0f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int64_t c = (p * 64 + lane) * V;
                float d[V], f[V];
                P::unpack(raw[p], d);
                P::unpack(ry[s][p], f);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dot = __builtin_fmaf(d[i], f[i], dot);
                    d[i] *= w;
                }
                P::template store<STREAM>(dy + row * j.lddy + c, j.cols - c, P::pack(d));
            }
            dot = wave_sum(dot);
            if (lane == q0 + s) dots = dot;
        }
    }
    if (lane < j.k) j.dw[t * j.k + lane] = dots;
    const u32x4_any zero = {0, 0, 0, 0};
    for (int64_t r = (used < 0 ? 0 : used) + t; r < j.rows_y; r += j.tokens)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int64_t c = (p * 64 + lane) * V;
            P::store(dy + r * j.lddy + c, j.cols - c, zero);
        }
}

// One workgroup per token (where tokens are few, per slot: gridDim.y = k): dout's segment in registers, each expert's row of y against
// it, the dot products added over the lanes, then over the waves in order.
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void combine_bwd_kernel(MoeBwdJob j) {
    using P = Piece<T>;
    constexpr int V = P::V;
    __shared__ float s_dot[4][kMoeMaxK];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t t = blockIdx.x;
    const int q0 = gridDim.y > 1 ? (int)blockIdx.y : 0, q1 = gridDim.y > 1 ? q0 + 1 : j.k;  // this workgroup's slots
    const T* const dout = static_cast<const T*>(j.dout) + t * j.lddo;
    const T* const y = static_cast<const T*>(j.y);
    T* const dy = static_cast<T*>(j.dy);
    const int64_t used = j.offsets[j.E];
    for (int q = tid; q < 4 * kMoeMaxK; q += 256) s_dot[q / kMoeMaxK][q % kMoeMaxK] = 0.0f;
    __syncthreads();
    for (int64_t seg = 0; seg < j.cols; seg += kSegPieces * 256 * V) {
        const int64_t c0 = seg + (int64_t)tid * V;
        u32x4_any raw[kSegPieces];
#pragma unroll
        for (int p = 0; p < kSegPieces; ++p) {
            const int64_t c = c0 + p * 256 * V;
            raw[p] = P::load(dout + c, j.cols - c);
        }
        for (int q = q0; q < q1; ++q) {
            const int32_t row = j.rows[t * j.k + q];
            if (row < 0 || row >= j.rows_y) continue;
            const float w = j.w ? j.w[t * j.k + q] : 1.0f;
            float dot = 0.0f;
#pragma unroll
            for (int p = 0; p < kSegPieces; ++p) {
                const int64_t c = c0 + p * 256 * V;
                float d[V], f[V];
                P::unpack(raw[p], d);
                P::unpack(P::load(y + row * j.ldy + c, j.cols - c), f);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dot = __builtin_fmaf(d[i], f[i], dot);
                    d[i] *= w;
                }
                P::template store<STREAM>(dy + row * j.lddy + c, j.cols - c, P::pack(d));
            }
            dot = wave_sum(dot);
            if (lane == 0) s_dot[wave][q] += dot;
        }
    }
    __syncthreads();
    for (int q = q0 + tid; q < q1; q += 256)
        j.dw[t * j.k + q] = (s_dot[0][q] + s_dot[1][q]) + (s_dot[2][q] + s_dot[3][q]);
    const u32x4_any zero = {0, 0, 0, 0};
    for (int64_t r = (used < 0 ? 0 : used) + t * gridDim.y + blockIdx.y; r < j.rows_y; r += j.tokens * gridDim.y)
        for (int64_t c = (int64_t)tid * V; c < j.cols; c += 256 * V) P::store(dy + r * j.lddy + c, j.cols - c, zero);
}

template <typename T>
int64_t segments(int64_t cols) {
    constexpr int64_t seg = kSegPieces * 64 * Piece<T>::V;
    return (cols + seg - 1) / seg;
}

}  // namespace

int64_t moe_sort_runs(int64_t n) { return n > 0 ? (n + kRun - 1) / kRun : 1; }

// Up to this many workgroups each adds up the others' counts itself; more have them summed by a launch of their own.
constexpr int64_t kAddUp = 64;

hipError_t launch_moe_sort(const MoeSortJob& j, hipStream_t s) {
    if (j.runs > 1) {
        sort_count_kernel<<<(unsigned)j.runs, kSortThreads, j.E * sizeof(int32_t), s>>>(j);
        if (j.runs > kAddUp) sort_scan_kernel<<<(unsigned)((j.E + 3) / 4), 256, 0, s>>>(j);
    }
    const size_t lds = 2 * j.E * sizeof(int32_t) + kSortWaves * j.E * sizeof(uint16_t);
    if (j.runs > kAddUp) sort_place_kernel<true><<<(unsigned)j.runs, kSortThreads, lds, s>>>(j);
    else sort_place_kernel<false><<<(unsigned)j.runs, kSortThreads, lds, s>>>(j);
    return hipGetLastError();
}

// Pieces a lane of rows of `cols`: 1, 2 or 4.
template <typename T, typename F>
void for_pieces(int64_t cols, F&& kernel) {
    using std::integral_constant;
    const int64_t pieces = (cols + 64 * Piece<T>::V - 1) / (64 * Piece<T>::V);
    if (pieces <= 1) kernel(integral_constant<int, 1>{});
    else if (pieces <= 2) kernel(integral_constant<int, 2>{});
    else kernel(integral_constant<int, kSegPieces>{});
}

// Rows by expert of kStreamBytes and more are stored (dispatch) and read (combine) nontemporally: no cache holds them until they
// are used again, and kept in order of recency they push out what is. bf16, 16384 tokens x 6 x 2048 (403 MB), us, nontemporal /
// plain: dispatch 80 / 92, combine 80 / 95, one after the other 160 / 204; 8192 tokens (201 MB) 42 / 35, 42 / 36, 84 / 72.
// combine_bwd reads one such tensor and writes another, so its stores take half the size (a workgroup per token: 16384 tokens 217 /
// 222, 8192 94 / 117, 4096 51 / 52).
template <typename T>
hipError_t launch_dispatch_t(MoeRowsJob j, hipStream_t s) {
    j.segs = segments<T>(j.cols);
    const unsigned g = (unsigned)((j.tokens * j.segs + 3) / 4);
    const bool stream = j.rows_y * j.cols * (int64_t)sizeof(T) >= kStreamBytes;
    for_pieces<T>(j.cols, [&](auto pieces) {
        constexpr int kP = decltype(pieces)::value;
        stream ? dispatch_kernel<T, true, kP><<<g, 256, 0, s>>>(j) : dispatch_kernel<T, false, kP><<<g, 256, 0, s>>>(j);
    });
    return hipGetLastError();
}

hipError_t launch_moe_dispatch(MoeRowsJob j, hipStream_t s) {
    return j.bf16 ? launch_dispatch_t<uint16_t>(j, s) : launch_dispatch_t<float>(j, s);
}

template <typename T>
hipError_t launch_combine_t(MoeRowsJob j, hipStream_t s) {
    j.segs = segments<T>(j.cols);
    const unsigned g = (unsigned)((j.tokens * j.segs + 3) / 4);
    const bool stream = j.rows_y * j.cols * (int64_t)sizeof(T) >= kStreamBytes;
    for_pieces<T>(j.cols, [&](auto pieces) {
        constexpr int kP = decltype(pieces)::value;
        stream ? combine_kernel<T, true, kP><<<g, 256, 0, s>>>(j) : combine_kernel<T, false, kP><<<g, 256, 0, s>>>(j);
    });
    return hipGetLastError();
}

hipError_t launch_moe_combine(MoeRowsJob j, hipStream_t s) {
    return j.bf16 ? launch_combine_t<uint16_t>(j, s) : launch_combine_t<float>(j, s);
}

// Up to this many slots (workgroups that 256 CUs hold at once) the gradient takes a workgroup per slot: a token's k rows one after
// the other are k times a read's latency. us, so / a workgroup per token, bf16: 7 tokens x 6 x 2048 4.5 / 12.0, 64 x 8 x 7168 5.2 /
// 13.3, 256 x 6 x 2048 7.7 / 12.5; 1024 x 6 x 2048 21.7 / 18.8 (dout is read k times).
constexpr int64_t kFewSlots = 2048;

template <typename T>
hipError_t launch_combine_bwd_t(const MoeBwdJob& j, hipStream_t s) {
    const bool stream = 2 * j.rows_y * j.cols * (int64_t)sizeof(T) >= kStreamBytes, few = j.tokens * j.k <= kFewSlots;
    if (!few && segments<T>(j.cols) <= 1) {
        const unsigned g = (unsigned)((j.tokens + 3) / 4);
        for_pieces<T>(j.cols, [&](auto pieces) {
            constexpr int kP = decltype(pieces)::value;
            stream ? combine_bwd_wave_kernel<T, true, kP><<<g, 256, 0, s>>>(j) : combine_bwd_wave_kernel<T, false, kP><<<g, 256, 0, s>>>(j);
        });
    } else {
        const dim3 g((unsigned)j.tokens, few ? (unsigned)j.k : 1u);
        stream ? combine_bwd_kernel<T, true><<<g, 256, 0, s>>>(j) : combine_bwd_kernel<T, false><<<g, 256, 0, s>>>(j);
    }
    return hipGetLastError();
}

hipError_t launch_moe_combine_bwd(const MoeBwdJob& j, hipStream_t s) {
    return j.bf16 ? launch_combine_bwd_t<uint16_t>(j, s) : launch_combine_bwd_t<float>(j, s);
}

}  // namespace ufp4
