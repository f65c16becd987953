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

// Four consecutive elements, in one access where p is aligned to their size.
template <typename T>
__device__ __forceinline__ void load4(const T *p, float (&v)[4]) {
    struct alignas(4 * sizeof(T)) Vec { T e[4]; };
    if ((reinterpret_cast<uintptr_t>(p) & (sizeof(Vec) - 1)) == 0) {
        const Vec w = *reinterpret_cast<const Vec *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32(w.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32(p[i]);
    }
}
// p is aligned to four elements.
template <typename T>
__device__ __forceinline__ void store4(T *p, const float (&v)[4]) {
    struct alignas(4 * sizeof(T)) Vec { T e[4]; };
    Vec w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.e[i] = from_f32<T>(v[i]);
    *reinterpret_cast<Vec *>(p) = w;
}

}  // namespace ipr
