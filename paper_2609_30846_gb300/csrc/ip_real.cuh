// Element types of the operators with real-valued inputs or outputs (f32, f16, bf16):
// loads to and stores from f32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace ipr {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
    return __float2bfloat16_rn(x);
}

// Eight consecutive elements; `vec`: p is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T *p, bool vec, float (&v)[8]) {
    if (vec) {
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            const uint4 w = *reinterpret_cast<const uint4 *>(p + i * W);
            const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
            for (int j = 0; j < W; ++j) v[i * W + j] = to_f32(e[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(p[i]);
    }
}

// p is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8 / W; ++i) {
        struct alignas(16) Vec { T e[W]; } w;
#pragma unroll
        for (int j = 0; j < W; ++j) w.e[j] = from_f32<T>(v[i * W + j]);
        *reinterpret_cast<Vec *>(p + i * W) = w;
    }
}

// Eight elements as they lie in memory.
template <typename T>
struct Raw8 {
    static constexpr int WORDS = 2 * sizeof(T);
    uint32_t w[WORDS];

    template <bool VEC>
    __device__ __forceinline__ void load(const T *p, int n) {      // the first n, the others 0
        if (VEC) {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(p) + i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
        } else {
            zero();
            for (int i = 0; i < n && i < 8; ++i) {
                if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
                else w[i >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << (16 * (i & 1));
            }
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    // largest magnitude so far, as the bits of T (two halves for the 16-bit types): magnitudes
    // order as integers, a NaN above an infinity above every number
    __device__ __forceinline__ void largest(uint32_t &top) const {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            top = sizeof(T) == 4 ? max(top, w[i] & 0x7fffffffu) : __vmaxu2(top, w[i] & 0x7fff7fffu);
    }
    // `top` of a thread as bits of an f32 of the same order and value
    static __device__ __forceinline__ uint32_t value(uint32_t top) {
        if constexpr (sizeof(T) == 4) return top;
        const uint16_t h = static_cast<uint16_t>(max(top >> 16, top & 0xffffu));
        return __float_as_uint(to_f32(*reinterpret_cast<const T *>(&h))) & 0x7fffffffu;
    }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        const uint16_t h = static_cast<uint16_t>(i & 1 ? w[i >> 1] >> 16 : w[i >> 1]);
        return to_f32(*reinterpret_cast<const T *>(&h));
    }
};

}  // namespace ipr
