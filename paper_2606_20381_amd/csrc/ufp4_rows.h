// Rows of bf16 or fp32 numbers in 16-byte pieces, for the kernels that take any row length, leading dimension and base
// address (layer norm, expert dispatch and combine).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ufp4_device.h"

namespace ufp4 {

// 16 bytes at the alignment of one element: gfx950's global loads and stores take any address, so an odd row length needs
// no second kernel. Only a row's last, partial piece goes element by element.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
struct Piece;

template <>
struct Piece<float> {
    static constexpr int V = 4;
    // S: nontemporally
    template <bool S = false>
    static __device__ __forceinline__ u32x4_any load(const float* p, int64_t left) {
        if (left >= V) {
            const u32x4_any* const q = reinterpret_cast<const u32x4_any*>(p);
            if constexpr (S) return __builtin_nontemporal_load(q);
            else return *q;
        }
        u32x4_any r = {0, 0, 0, 0};
        if (left > 0) r[0] = __float_as_uint(p[0]);
        if (left > 1) r[1] = __float_as_uint(p[1]);
        if (left > 2) r[2] = __float_as_uint(p[2]);
        return r;
    }
    static __device__ __forceinline__ void unpack(const u32x4_any& r, float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = __uint_as_float(r[i]);
    }
    static __device__ __forceinline__ u32x4_any pack(const float (&f)[V]) {
        return u32x4_any{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    template <bool S = false>
    static __device__ __forceinline__ void store(float* p, int64_t left, const u32x4_any& r) {
        if (left >= V) {
            if constexpr (S) __builtin_nontemporal_store(r, reinterpret_cast<u32x4_any*>(p));
            else *reinterpret_cast<u32x4_any*>(p) = r;
            return;
        }
        if (left > 0) p[0] = __uint_as_float(r[0]);
        if (left > 1) p[1] = __uint_as_float(r[1]);
        if (left > 2) p[2] = __uint_as_float(r[2]);
    }
};

template <>
struct Piece<uint16_t> {  // bf16 bits
    static constexpr int V = 8;
    template <bool S = false>
    static __device__ __forceinline__ u32x4_any load(const uint16_t* p, int64_t left) {
        if (left >= V) {
            const u32x4_any* const q = reinterpret_cast<const u32x4_any*>(p);
            if constexpr (S) return __builtin_nontemporal_load(q);
            else return *q;
        }
        u32x4_any r = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < left) r[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        return r;
    }
    static __device__ __forceinline__ void unpack(const u32x4_any& r, float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(r[i]);
            f[2 * i + 1] = bf16_hi(r[i]);
        }
    }
    // one rounding, to nearest even; NaN and infinity keep their kind
    static __device__ __forceinline__ u32x4_any pack(const float (&f)[V]) {
        u32x4_any r;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[2 * i]) |
                   (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[2 * i + 1]) << 16;
        return r;
    }
    template <bool S = false>
    static __device__ __forceinline__ void store(uint16_t* p, int64_t left, const u32x4_any& r) {
        if (left >= V) {
            if constexpr (S) __builtin_nontemporal_store(r, reinterpret_cast<u32x4_any*>(p));
            else *reinterpret_cast<u32x4_any*>(p) = r;
            return;
        }
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < left) p[i] = (uint16_t)(r[i >> 1] >> (16 * (i & 1)));
    }
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

}  // namespace ufp4
