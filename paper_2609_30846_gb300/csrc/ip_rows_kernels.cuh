// Device code of a decoder's rows for sm_103a: the root-mean-square norm with the residual's
// addition, rows quantised to int8 or to microscaled 4-bit floating point (e2m1 codes, an e4m3
// scale for each 16 of them, an f32 scale a row) in the same pass, and the values of such rows.
#pragma once

#include <stdint.h>

#include "ip_scaled_kernels.cuh"

namespace ipw {

using namespace ipk;
using namespace ipr;

// ---- 4-bit rows ----------------------------------------------------------
//
// With amax the row's largest magnitude: r = 2^e, the least power of two with amax <= 2688 r
// (2688 = 6 x 448, the largest e2m1 times the largest e4m3 number) and e >= -126; a block's scale
// is s = e4m3(amax_b / (6 r)), a code c = e2m1(x / (s r)), both to nearest, ties to even, as exactly
// stated: x / r is exact, and what is rounded to 4 or 2 bits is the f32 quotient rounded to
// nearest.  That is right although it rounds twice: the midpoints m of both formats have at most
// five significant bits, so x and m s are neighbours in f32 at best, |x - m s| >= 2^-24 m s, and the
// f32 quotient of an x that is not m s falls on the side of m that x / s is on.
// The quotient: q = x i, i the reciprocal of s rounded to nearest, then q - i (q s - x), the
// remainder exact in one fma (Markstein's correction).
// The e4m3 scales lie in blocks of 512 bytes for 128 rows x 64 elements (4 scales a row), byte
// 16 (row mod 32) + 4 ((row mod 128) / 32) + (block mod 4): 32 lanes of four words, as the tensor
// cores take them.

__device__ __forceinline__ uint32_t e4m3_of(float x) {      // 0 <= x, at most 448 (larger: 448)
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(0.0f), "f"(x));
    return v;
}
__device__ __forceinline__ float e4m3_value(uint32_t b) {   // of a byte below 0x80
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(b)));
    return __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
}
__device__ __forceinline__ uint32_t e2m1_of8(const float (&q)[8]) {      // eight codes, the first lowest
    uint32_t w;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}\n"
        : "=r"(w)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return w;
}
__device__ __forceinline__ void e2m1_values8(uint32_t w, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2 p = *reinterpret_cast<const __half2 *>(&h[j]);
        v[2 * j] = __low2float(p);
        v[2 * j + 1] = __high2float(p);
    }
}
// Byte offset of the four scales of chunk kc (64 elements) of a row, kcs chunks a row.
__device__ __forceinline__ long long scale_at(long long row, int kc, int kcs) {
    return ((row >> 7) * kcs + kc) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// ---- norm and rows -------------------------------------------------------
//
// h = x + residual, rounded to the elements' type (it is the next residual); z = h weight in f32;
// the output row is z / sqrt(mean(h^2) + eps), quantised.  The row's factor 1 / sqrt(...) leaves the
// codes as they are, so they are z's, exactly as the definitions of the rows say, and only the
// row's scale carries it.
//
// What bounds it: DRAM; a row stays in registers between the passes up to 8 UNITS elements a
// thread (a longer one is read again, from L2).
//
// The squares are summed in f32.  Sums that leave the middle of its range (bf16 and f32 rows
// beyond 2^55 or below 2^-35) are formed again from elements scaled by 2^-80 or 2^96, and the
// row's magnitude is divided by that root first, so that 1 / root need not be an f32.

constexpr int UNITS = 4;      // units of eight elements that a thread keeps

struct RowsParams {
    const void *x, *res, *weight;
    long long rows, ldx, ldres, ldsum, ldq;
    int d;
    float eps;
    void *sum;
    uint8_t *q;
    uint8_t *blocks;          // 4-bit rows: their e4m3 scales
    float *scale;
};

enum { OUT_I8 = 0, OUT_FP4 = 1 };

template <int WARPS>
__device__ __forceinline__ float row_sum(float v, float *red) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (WARPS > 1) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) v += red[i];
    }
    return v;
}
template <int WARPS>
__device__ __forceinline__ uint32_t row_max(uint32_t v, float *red) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (WARPS > 1) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = __uint_as_float(v);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WARPS; ++i) v = max(v, __float_as_uint(red[i]));
    }
    return v;
}

// x + r rounded to T, as bits.
template <typename T>
__device__ __forceinline__ void add8(Raw8<T> &x, const Raw8<T> &r) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const T h = from_f32<T>(x.at(j) + r.at(j));
        if constexpr (sizeof(T) == 4) {
            x.w[j] = __float_as_uint(h);
        } else {
            const uint32_t b = *reinterpret_cast<const uint16_t *>(&h);
            x.w[j >> 1] = j & 1 ? (x.w[j >> 1] & 0xffffu) | (b << 16) : (x.w[j >> 1] & 0xffff0000u) | b;
        }
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_raw(T *p, const Raw8<T> &v, int n) {
    if (VEC) {
#pragma unroll
        for (int i = 0; i < Raw8<T>::WORDS; i += 4)
            *reinterpret_cast<uint4 *>(reinterpret_cast<uint32_t *>(p) + i) = make_uint4(v.w[i], v.w[i + 1], v.w[i + 2], v.w[i + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = from_f32<T>(v.at(j));
    }
}

// Eight elements to int8 (ip_scaled_kernels.cuh has the argument; f, inv, top of the row).
__device__ __forceinline__ uint2 to_i8(const float (&z)[8], float f, float inv, float top, bool far) {
    uint32_t k[8];
    float off = far ? 1.0f : 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        k[j] = __float_as_uint(__fmaf_rn(z[j], inv, 12582912.0f));
        off = fmaxf(off, fabsf(__fmaf_rn(z[j], inv, -__fsub_rn(__uint_as_float(k[j]), 12582912.0f))));
    }
    if (off > 0.5f - 0x1p-14f) {
        Raw8<float> raw;
#pragma unroll
        for (int j = 0; j < 8; ++j) raw.w[j] = __float_as_uint(z[j]);
        return ips::quant_look<float>(raw, f, inv, top);
    }
    return ips::low_bytes(k);
}

// TPR threads a row: 32 (four rows a CTA), 128 or 256 (the CTA).  VEC: rows of x, residual, sum and
// the weight start on 16 bytes (q's on 8) and d is a multiple of eight.  NORM: with weight and
// norm, else the rows of x as they are (4-bit rows only).
template <typename T, int TPR, bool VEC, int OUT, bool NORM>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) rows_kernel(const RowsParams prm) {
    constexpr int RPC = TPR < 128 ? 128 / TPR : 1, WARPS = TPR / 32;
    __shared__ float red[WARPS];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const int d = prm.d, kcs = (d + 63) / 64;
    const bool with_res = NORM && prm.res != nullptr;
    const T *g = static_cast<const T *>(prm.weight);
    for (long long row = static_cast<long long>(blockIdx.x) * RPC + threadIdx.x / TPR; row < prm.rows;
         row += static_cast<long long>(gridDim.x) * RPC) {
        const T *x = static_cast<const T *>(prm.x) + row * prm.ldx;
        const T *res = with_res ? static_cast<const T *>(prm.res) + row * prm.ldres : nullptr;
        T *sum = with_res ? static_cast<T *>(prm.sum) + row * prm.ldsum : nullptr;
        Raw8<T> h[UNITS], w[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int c = (i * TPR + t) * 8;
            h[i].zero();
            if (NORM) w[i].zero();
            if (c < d) {
                h[i].template load<VEC>(x + c, d - c);
                if (NORM) w[i].template load<VEC>(g + c, d - c);
            }
        }
        if (with_res) {
            Raw8<T> r[UNITS];
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 8;
                r[i].zero();
                if (c < d) r[i].template load<VEC>(res + c, d - c);
            }
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 8;
                add8(h[i], r[i]);
                if (c < d) store_raw<VEC>(sum + c, h[i], d - c);
            }
        }
        // elements behind those that a thread keeps: read and added here, read again below
        constexpr int KEPT = UNITS * TPR * 8;
        float ss = 0.0f;
        uint32_t top = 0;
        auto take = [&](const Raw8<T> &v, const Raw8<T> &u, float f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float a = v.at(j);
                const float b = NORM ? a * f : 0.0f;
                ss = __fmaf_rn(b, b, ss);
                top = max(top, __float_as_uint(NORM ? __fmul_rn(a, u.at(j)) : a) & 0x7fffffffu);
            }
        };
#pragma unroll
        for (int i = 0; i < UNITS; ++i) take(h[i], w[i], 1.0f);
        for (int c = KEPT + t * 8; c < d; c += TPR * 8) {
            Raw8<T> v, u;
            v.template load<VEC>(x + c, d - c);
            if (with_res) {
                u.template load<VEC>(res + c, d - c);
                add8(v, u);
                store_raw<VEC>(sum + c, v, d - c);
            }
            if (NORM) u.template load<VEC>(g + c, d - c);
            take(v, u, 1.0f);
        }
        const T *again = with_res ? sum : x;
        const uint32_t bits = row_max<WARPS>(top, red);
        const bool finite = bits < 0x7f800000u;
        const float amax = __uint_as_float(bits);
        float root = 1.0f, up = 1.0f;      // the row is divided by root / up
        if (NORM) {
            ss = row_sum<WARPS>(ss, red);
            float eps = prm.eps;
            const bool large = !(ss < 0x1p110f), small = ss < 0x1p-70f && prm.eps < 0x1p-80f;
            if (sizeof(T) == 4 || !std::is_same<T, __half>::value)
                if (large || small) {
                    up = large ? 0x1p-80f : 0x1p96f;
                    eps = eps * up * up;
                    ss = 0.0f;
                    uint32_t unused = top;
#pragma unroll
                    for (int i = 0; i < UNITS; ++i) take(h[i], w[i], up);
                    for (int c = KEPT + t * 8; c < d; c += TPR * 8) {
                        Raw8<T> v;
                        v.template load<VEC>(again + c, d - c);
                        take(v, v, up);
                    }
                    top = unused;
                    ss = row_sum<WARPS>(ss, red);
                }
            root = __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, static_cast<float>(d)), eps));
        }
        const bool zero = !finite || bits == 0;
        const int e = static_cast<int>(bits >> 23);
        uint8_t *q = prm.q + row * prm.ldq;
        if (OUT == OUT_I8) {
            if (t == 0)
                prm.scale[row] = finite ? (bits == 0 ? 0.0f : __fdiv_rn(__fmul_rn(__fdiv_rn(amax, root), up), 127.0f)) : __uint_as_float(0x7fc00000u);
            // rows near the ends of the range are brought to the middle by a power of two
            const bool far = e < 32 || e > 222;
            const int fe = 254 - e < 1 ? 1 : (254 - e > 253 ? 253 : 254 - e);
            const float f = far ? __uint_as_float(static_cast<unsigned>(fe) << 23) : 1.0f;
            const float ntop = amax * f, inv = zero ? 0.0f : __fdiv_ru(127.0f, ntop);
            auto put = [&](int c, const Raw8<T> &v, const Raw8<T> &u) {
                float z[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = __fmul_rn(v.at(j), u.at(j));
                const uint2 b = zero ? make_uint2(0u, 0u) : to_i8(z, f, inv, ntop, far);
                if (VEC) {
                    *reinterpret_cast<uint2 *>(q + c) = b;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < d) q[c + j] = static_cast<uint8_t>((j < 4 ? b.x : b.y) >> (8 * (j & 3)));
                }
            };
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 8;
                if (c < d) put(c, h[i], w[i]);
            }
            for (int c = KEPT + t * 8; c < d; c += TPR * 8) {
                Raw8<T> v, u;
                v.template load<VEC>(again + c, d - c);
                u.template load<VEC>(g + c, d - c);
                put(c, v, u);
            }
        } else {
            // amax = m 2^(e - 127), 1 <= m < 2, is at most 2688 r = 1.3125 2^11 r
            int ex = e - 127 - ((bits & 0x7fffffu) <= 0x280000u ? 11 : 10);
            ex = ex < -126 ? -126 : ex;
            const float f = __uint_as_float(static_cast<unsigned>(127 - ex) << 23);
            const float r = __uint_as_float(static_cast<unsigned>(127 + ex) << 23);
            if (t == 0) prm.scale[row] = finite ? (bits == 0 ? 0.0f : NORM ? __fmul_rn(__fdiv_rn(r, root), up) : r) : __uint_as_float(0x7fc00000u);
            // all lanes of a warp come here together: four blocks of eight lanes make one word
            auto put = [&](int c, const Raw8<T> &v, const Raw8<T> &u) {
                float z[8], big = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    z[j] = (NORM ? __fmul_rn(v.at(j), u.at(j)) : v.at(j)) * f;
                    big = fmaxf(big, fabsf(z[j]));
                }
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                const uint32_t sb = zero ? 0u : e4m3_of(__fdiv_rn(big, 6.0f));
                uint32_t word = lane & 1 ? 0u : sb << (4 * (lane & 6));
                word |= __shfl_xor_sync(0xffffffffu, word, 2);
                word |= __shfl_xor_sync(0xffffffffu, word, 4);
                if ((lane & 7) == 0 && c < d)
                    *reinterpret_cast<uint32_t *>(prm.blocks + scale_at(row, c >> 6, kcs)) = word;
                if (c >= d) return;
                uint32_t code = 0;
                if (sb != 0) {
                    const float s = e4m3_value(sb), i = __frcp_rn(s);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float y = z[j] * i;
                        z[j] = __fmaf_rn(-__fmaf_rn(y, s, -z[j]), i, y);      // so that -0 stays -0
                    }
                    code = e2m1_of8(z);
                }
                if (c + 8 <= d) {
                    *reinterpret_cast<uint32_t *>(q + (c >> 1)) = code;
                } else {
                    for (int j = 0; c + 2 * j < d; ++j) q[(c >> 1) + j] = static_cast<uint8_t>(code >> (8 * j));
                }
            };
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 8;
                if (c - lane * 8 < d) put(c, h[i], w[i]);
            }
            for (int c = KEPT + t * 8; c - lane * 8 < d; c += TPR * 8) {
                Raw8<T> v, u;
                v.zero();
                if (NORM) u.zero();
                if (c < d) {
                    v.template load<VEC>(again + c, d - c);
                    if (NORM) u.template load<VEC>(g + c, d - c);
                }
                put(c, v, u);
            }
        }
    }
}

// ---- values of rows ------------------------------------------------------

struct ValuesParams {
    const uint8_t *q, *blocks;
    const float *scale;
    long long rows, ldq, ldy;
    int d;
    void *y;
    unsigned long long magic;      // of the units a row
    int units;
};

// code x scale (a 4-bit row's: code x block scale, exact, x row scale), rounded once.  A thread
// takes 16 elements.  VEC: rows of q and y start on 16 bytes and d is a multiple of 16.
template <typename T, bool VEC, int IN>
__global__ void __launch_bounds__(256) values_kernel(const ValuesParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    const long long n = prm.rows * prm.units;
    for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<long long>(gridDim.x) * 256) {
        const long long row = i < (1ll << 32) ? static_cast<long long>(udiv_magic(static_cast<uint32_t>(i), prm.magic)) : i / prm.units;
        const int c = static_cast<int>(i - row * prm.units) * 16, d = prm.d;
        const float scale = prm.scale[row];
        float v[16];
        if (IN == OUT_I8) {
            const uint8_t *q = prm.q + row * prm.ldq + c;
            uint32_t w[4] = {0, 0, 0, 0};
            if (VEC) {
                const uint4 u = *reinterpret_cast<const uint4 *>(q);
                w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
            } else {
                for (int j = 0; j < 16 && c + j < d; ++j) w[j >> 2] |= static_cast<uint32_t>(q[j]) << (8 * (j & 3));
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = static_cast<float>(sbyte(w[j >> 2], j & 3)) * scale;
        } else {
            const uint8_t *q = prm.q + row * prm.ldq + (c >> 1);
            uint32_t w[2] = {0, 0};
            if (VEC) {
                const uint2 u = *reinterpret_cast<const uint2 *>(q);
                w[0] = u.x, w[1] = u.y;
            } else {
                for (int j = 0; j < 8 && c + 2 * j < d; ++j) w[j >> 2] |= static_cast<uint32_t>(q[j]) << (8 * (j & 3));
            }
            const float s = e4m3_value(prm.blocks[scale_at(row, c >> 6, (d + 63) / 64) + ((c >> 4) & 3)]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float u[8];
                e2m1_values8(w[k], u);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[8 * k + j] = u[j] * s * scale;
            }
        }
        T *y = static_cast<T *>(prm.y) + row * prm.ldy + c;
        if (VEC) {
            float a[8], b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = v[j], b[j] = v[8 + j];
            store8<T>(y, a);
            store8<T>(y + 8, b);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < d) y[j] = from_f32<T>(v[j]);
        }
    }
}

}  // namespace ipw
