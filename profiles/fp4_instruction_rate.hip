// v_mfma_scale_f32_32x32x64_f8f6f4 on registers alone, as the product kernel issues it: two waves per SIMD, 4 x 2 tiles a wave,
// operands that change from one product of a tile to the next (SETS sets of them, and of scales).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <random>
#include <vector>
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));
constexpr int kGroups = 256, kThreads = 512, kProducts = 128000;  // of a wave
template <int SETS>
__global__ __launch_bounds__(kThreads, 2) void rate(const int4* in, const int* scales, float* out) {
    const int at = blockIdx.x * kThreads + threadIdx.x;
    int4 f[SETS][6];
    int s[SETS];
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        s[i] = scales[at * 4 + i];
#pragma unroll
        for (int k = 0; k < 6; ++k) f[i][k] = in[(at * 4 + i) * 6 + k];
    }
    v16f c[4][2] = {};
#pragma unroll 1
    for (int k = 0; k < kProducts / (8 * SETS); ++k)
#pragma unroll
        for (int i = 0; i < 8 * SETS; ++i) {
            const int set = i >> 3, a = (i >> 1) & 3, b = i & 1;
            const int4 p = f[set][b], q = f[set][2 + a];
            c[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v8i{p.x, p.y, p.z, p.w, 0, 0, 0, 0}, v8i{q.x, q.y, q.z, q.w, 0, 0, 0, 0},
                                                                      c[a][b], 4, 4, 0, s[set], 1, s[set]);
        }
    float sum = 0;
    for (int i = 0; i < 8; ++i)
        for (int e = 0; e < 16; ++e) sum += c[i >> 1][i & 1][e];
    out[at] = sum;
}
int main() {
    const size_t n = (size_t)kGroups * kThreads;
    std::vector<uint32_t> host(n * 96);
    std::vector<int> sc(n * 4);
    std::mt19937 g(1);
    std::normal_distribution<float> normal(0.0f, 2.5f);  // of a block of 32 the largest lies in 4 .. 8
    int4* in; int* scales; float* out;
    if (hipMalloc(&in, host.size() * 4) != hipSuccess || hipMalloc(&scales, n * 16) != hipSuccess || hipMalloc(&out, n * 4) != hipSuccess) return 1;
    hipEvent_t t0, t1;
    if (hipEventCreate(&t0) != hipSuccess || hipEventCreate(&t1) != hipSuccess) return 1;
    for (int kind = 0; kind < 3; ++kind) {  // normal codes, scales of one binade or of five; zeros
        for (auto& v : host) {
            v = 0;
            for (int i = 0; i < 8 && kind < 2; ++i) {
                const float x = normal(g), a = fabsf(x);
                const uint32_t c = a < 0.25f ? 0 : a < 0.75f ? 1 : a < 1.25f ? 2 : a < 1.75f ? 3 : a < 2.5f ? 4 : a < 3.5f ? 5 : a < 5.0f ? 6 : 7;
                v |= (c | (x < 0 ? 8 : 0)) << (4 * i);
            }
        }
        for (auto& v : sc) v = kind == 1 ? (125 + (int)(g() % 5)) | (125 + (int)(g() % 5)) << 8 : 127 | 127 << 8;
        if (hipMemcpy(in, host.data(), host.size() * 4, hipMemcpyHostToDevice) != hipSuccess) return 1;
        if (hipMemcpy(scales, sc.data(), n * 16, hipMemcpyHostToDevice) != hipSuccess) return 1;
        for (int sets = 2; sets <= 4; sets += 2) {
            auto go = [&] { sets == 2 ? rate<2><<<kGroups, kThreads>>>(in, scales, out) : rate<4><<<kGroups, kThreads>>>(in, scales, out); };
            for (int i = 0; i < 50; ++i) go();
            (void)hipEventRecord(t0);
            for (int i = 0; i < 150; ++i) go();
            (void)hipEventRecord(t1);
            if (hipEventSynchronize(t1) != hipSuccess) return 1;
            float ms = 0;
            (void)hipEventElapsedTime(&ms, t0, t1);
            const double flops = (double)kGroups * (kThreads / 64) * kProducts * 150 * 2 * 32 * 32 * 64;
            printf("%s, %d sets of operands: %.2f ms a launch, %.2f PFLOP/s\n",
                   kind == 0 ? "normal codes, one scale" : kind == 1 ? "normal codes, scales of five binades" : "zeros", sets, ms / 150,
                   flops / (ms * 1e-3) / 1e15);
            fflush(stdout);
        }
    }
    return hipDeviceSynchronize() == hipSuccess ? 0 : 1;
}
