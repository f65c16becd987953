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
// A quotient: y = x i, i the reciprocal of s rounded to nearest, then y - i (y s - x), the
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
__device__ __forceinline__ uint32_t e2m1_of8(const uint32_t *h) {      // of eight f16 numbers
    uint32_t w;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f16x2 a, %1;\n cvt.rn.satfinite.e2m1x2.f16x2 b, %2;\n"
        " cvt.rn.satfinite.e2m1x2.f16x2 c, %3;\n cvt.rn.satfinite.e2m1x2.f16x2 d, %4;\n"
        " mov.b32 %0, {a, b, c, d};\n}\n"
        : "=r"(w)
        : "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]));
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
// What bounds it: DRAM, and close behind it the instructions: 12000 x 1024 bf16 with residual 13.4-13.8 us, 6.3 TB/s, to 4 bits
// 13.0 (17.5 while each element's operations were done twice).  f32 rows hold twice the bytes in registers: 6000 x 1024 with residual 16.1
// us, 5.0 TB/s.  Not so where rows are short, a warp each whatever their length (12000 x 40 6.2 us, 96000 x 128 42), or not on
// 16 bytes (6000 x 1023 bf16 16.8, x 1024 7.7; f32 25 and 16).  A row stays in registers between the passes up to 16 UNITS elements a thread (a longer one is read again, from L2).
//
// The squares are summed in f32.  Sums that leave the middle of its range (bf16 and f32 rows
// beyond 2^55 or below 2^-35) are formed again from elements scaled by 2^-80 or 2^96, and the
// row's magnitude is divided by that root first, so that 1 / root need not be an f32.

struct RowsParams {
    const void *x, *res, *weight;
    long long rows, ldx, ldres, ldsum, ldq;
    int d;
    float eps;
    void *sum;
    uint8_t *q;
    uint8_t *blocks;          // 4-bit rows: their e4m3 scales
    float *scale;
    bool q16;                 // rows of q start on 16 bytes
};

enum { OUT_I8 = 0, OUT_FP4 = 1 };

// Sum and maximum over a row's warps; red: two buffers that successive calls take in turn.
template <int WARPS>
__device__ __forceinline__ void reduce(float &sum, uint32_t &top, float2 (*red)[WARPS], int &turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    top = __reduce_max_sync(0xffffffffu, top);
    if (WARPS > 1) {
        if ((threadIdx.x & 31) == 0) red[turn][threadIdx.x >> 5] = make_float2(sum, __uint_as_float(top));
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const float2 v = red[turn][i];
            sum += v.x;
            top = max(top, __float_as_uint(v.y));
        }
        turn ^= 1;
    }
}

// Sixteen elements as they lie in memory, the first n of them, the others 0.
template <typename T>
struct Raw16 {
    Raw8<T> h[2];

    // p: c elements into its row, of which n are left.  Rows that are not on 16 bytes: the aligned vectors that hold the
    // elements, where all of them lie within the row, turned by the words and bytes that p is off.
    template <bool VEC>
    __device__ __forceinline__ void load(const T *p, int n, int c) {
        if constexpr (!VEC) {
            constexpr int ES = sizeof(T), WORDS = Raw8<T>::WORDS;
            const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15;
            const int before = off / ES;
            if (before <= c && 16 + (off ? 16 / ES - before : 0) <= n) {
                const uint4 *from = reinterpret_cast<const uint4 *>(p - before);
                uint32_t x[4 * ES + 4];
#pragma unroll
                for (int i = 0; i <= ES; ++i) {
                    const uint4 u = i < ES || off ? from[i] : make_uint4(0, 0, 0, 0);
                    x[4 * i] = u.x, x[4 * i + 1] = u.y, x[4 * i + 2] = u.z, x[4 * i + 3] = u.w;
                }
#pragma unroll
                for (int i = 0; i < 4 * ES + 3; ++i) x[i] = off & 4 ? x[i + 1] : x[i];
#pragma unroll
                for (int i = 0; i < 4 * ES + 1; ++i) x[i] = off & 8 ? x[i + 2] : x[i];
#pragma unroll
                for (int i = 0; i < 4 * ES; ++i)
                    h[i / WORDS].w[i % WORDS] = ES == 4 ? x[i] : __funnelshift_r(x[i], x[i + 1], 8 * (off & 2));
                return;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (8 * k < n) h[k].template load<VEC>(p + 8 * k, n - 8 * k);
            else h[k].zero();
        }
    }
    // p on 16 bytes, n a multiple of eight
    __device__ __forceinline__ void store(T *p, int n) const {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (8 * k < n)
#pragma unroll
                for (int i = 0; i < Raw8<T>::WORDS; i += 4)
                    *reinterpret_cast<uint4 *>(reinterpret_cast<uint32_t *>(p + 8 * k) + i) =
                        make_uint4(h[k].w[i], h[k].w[i + 1], h[k].w[i + 2], h[k].w[i + 3]);
    }
    __device__ __forceinline__ float at(int j) const { return h[j >> 3].at(j & 7); }
    // + r, rounded to T once (the sum of two 16-bit numbers by an instruction that rounds the exact one)
    __device__ __forceinline__ void add(const Raw16 &r) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < Raw8<T>::WORDS; ++i) {
                if constexpr (sizeof(T) == 4) {
                    h[k].w[i] = __float_as_uint(__fadd_rn(__uint_as_float(h[k].w[i]), __uint_as_float(r.h[k].w[i])));
                } else if constexpr (std::is_same<T, __half>::value) {
                    asm("add.rn.f16x2 %0, %0, %1;" : "+r"(h[k].w[i]) : "r"(r.h[k].w[i]));
                } else {
                    asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(h[k].w[i]) : "r"(r.h[k].w[i]));
                }
            }
    }
};

// Rows that are not on 16 bytes leave through shared memory, so that a warp's lanes write neighbours (a lane's own sixteen
// one by one: values of 6000 x 1023 29.6 us for 8.9, norm with residual 42 for 19).  Per warp, sixteen elements a lane.
template <typename T>
struct Turn {
    static constexpr int LD = sizeof(T) == 4 ? 17 : 18;
    T e[32 * LD];
};

// The larger magnitude, NaN above all; the sign is of no use.
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The same of two pairs of 16-bit numbers.
template <typename T>
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
    uint32_t r;
    if (std::is_same<T, __half>::value) asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Sixteen elements to int8 (ip_scaled_kernels.cuh has the argument; f, inv, top of the row).
__device__ __forceinline__ uint2 to_i8(const float *z, float f, float inv, float top, bool far) {
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

__device__ __forceinline__ float largest16(const float (&z)[16]) {
    float big = fabsf(z[0]);
#pragma unroll
    for (int j = 1; j < 16; ++j) big = fmaxf(big, fabsf(z[j]));
    return big;
}

// What a row's blocks are coded with: their largest magnitude comes to [0, 2688] times `down`; a block scale s
// stands for s `up` in units of the elements.
struct Fp4Row {
    float down, up;
};
// Block scale byte and codes of sixteen elements whose largest magnitude is `big`.  SHORT: elements of 11 bits at most.  The
// quotient of one that is not m s is 2^-11 m from m at least (m s has seven bits), so that f16, whose
// half step at m is less, keeps it on its side, and takes an f32 quotient 2^-22 m from m to m: no remainder is needed.
template <bool SHORT>
__device__ __forceinline__ uint32_t to_fp4(const float (&z)[16], float big, Fp4Row row, uint2 &code) {
    // big down / 6, the quotient rounded to nearest (Markstein, as below)
    const float b = big * row.down, sixth = 0.16666667f, y6 = b * sixth;
    const uint32_t sb = e4m3_of(__fmaf_rn(-__fmaf_rn(y6, 6.0f, -b), sixth, y6));
    code = make_uint2(0u, 0u);
    if (sb == 0) return 0;
    const float s = e4m3_value(sb);
    // the reciprocal of the four-bit s to nearest: one Newton step
    float i;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(i) : "f"(s));
    if (SHORT) {
        i *= row.down;
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)      // both products by one instruction
            asm("{\n .reg .b64 p, q;\n .reg .f32 a, b;\n mov.b64 p, {%1, %2};\n mov.b64 q, {%3, %3};\n mul.rn.f32x2 p, p, q;\n"
                " mov.b64 {a, b}, p;\n cvt.rn.f16x2.f32 %0, b, a;\n}\n"
                : "=r"(h[j])
                : "f"(z[2 * j]), "f"(z[2 * j + 1]), "f"(i));
        code = make_uint2(e2m1_of8(h), e2m1_of8(h + 4));
        return sb;
    }
    i = __fmaf_rn(i, __fmaf_rn(-s, i, 1.0f), i) * row.down;
    const float su = s * row.up;
    float q[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float y = z[j] * i;
        q[j] = __fmaf_rn(-__fmaf_rn(y, su, -z[j]), i, y);      // so that -0 stays -0
    }
    code = make_uint2(e2m1_of8(*reinterpret_cast<const float (*)[8]>(q)), e2m1_of8(*reinterpret_cast<const float (*)[8]>(q + 8)));
    return sb;
}

// CTAs that an SM is to hold, which bounds the registers: a row's bytes in flight are what hides DRAM's latency
// (rows to 4 bits, us, at 6 / 8 / 10 CTAs: 12000 x 4096 f16 29.3 / 24.8 / 24.5, x 2048 21.9 / 17.4 / 15.7; norm of 12000 x
// 1024 bf16 17.8 / 20.3 / 25.9, its registers spill).  What is left of spills at these bounds, bytes stored a thread: none in 16-bit
// norms up to 4096, up to 140 beyond; 16 to 112 in f32 norms of more than 2048 on 16 bytes, 28 to 712 off 16 bytes.
template <typename T, int TPR, int UNITS, bool NORM>
constexpr int rows_ctas() {
    constexpr bool WIDE = sizeof(T) == 4;
    if (TPR == 256) return NORM ? (WIDE ? 3 : 4) : (WIDE ? 3 : 5);
    if (UNITS == 1) return NORM || WIDE ? 8 : 12;
    return NORM ? (WIDE ? 5 : 6) : (WIDE ? 6 : 8);
}

// TPR threads a row: 32 (four rows a CTA), 128 or 256 (the CTA), UNITS of sixteen elements each in
// registers.  VEC: rows of x, residual, sum, the weight and q start on 16 bytes and d is a multiple
// of eight.  NORM: with weight and norm, else the rows of x as they are (4-bit rows only).
template <typename T, int TPR, int UNITS, bool VEC, int OUT, bool NORM>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, rows_ctas<T, TPR, UNITS, NORM>()) rows_kernel(const RowsParams prm) {
    constexpr int RPC = TPR < 128 ? 128 / TPR : 1, WARPS = TPR / 32, KEPT = UNITS * TPR * 16;
    __shared__ float2 red[2][WARPS];
    __shared__ Turn<T> turns[NORM && !VEC ? (TPR < 128 ? 4 : WARPS) : 1];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const int d = prm.d, kcs = (d + 63) / 64;
    const bool with_res = NORM && prm.res != nullptr;
    const T *g = static_cast<const T *>(prm.weight);
    // the sum's elements from c on, by all lanes of a warp together
    auto store_sum = [&](const Raw16<T> &h, T *sum, int c) {
        if constexpr (VEC) {
            h.store(sum + c, d - c);
        } else {
            Turn<T> &own = turns[threadIdx.x >> 5];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) own.e[lane * Turn<T>::LD + j] = from_f32<T>(h.at(j));
            __syncwarp();
            const int c0 = c - lane * 16;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int e = 32 * k + lane;
                if (c0 + e < d) sum[c0 + e] = own.e[(e >> 4) * Turn<T>::LD + (e & 15)];
            }
            __syncwarp();
        }
    };
    int turn = 0;
    for (long long row = static_cast<long long>(blockIdx.x) * RPC + threadIdx.x / TPR; row < prm.rows;
         row += static_cast<long long>(gridDim.x) * RPC) {
        const T *x = static_cast<const T *>(prm.x) + row * prm.ldx;
        const T *res = with_res ? static_cast<const T *>(prm.res) + row * prm.ldres : nullptr;
        T *sum = with_res ? static_cast<T *>(prm.sum) + row * prm.ldsum : nullptr;
        const T *again = with_res ? sum : x;
        float ss = 0.0f, top = 0.0f;
        uint32_t bits = 0;
        // h's elements: their squares and, in z, what is quantised
        auto take = [&](const Raw16<T> &h, const Raw16<T> &w, float (&z)[16]) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float a = h.at(j);
                ss = __fmaf_rn(a, a, ss);
                z[j] = __fmul_rn(a, w.at(j));
                top = larger(top, z[j]);
            }
        };
        Raw16<T> raw[NORM ? 1 : UNITS];
        uint32_t most[NORM ? 1 : UNITS];      // of a unit's elements, as Raw8::largest has it
        float z[NORM ? UNITS : 1][16];
        if constexpr (NORM) {
            Raw16<T> h[UNITS], w[UNITS];
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 16;
                h[i].template load<VEC>(x + c, d - c, c);
                w[i].template load<VEC>(g + c, d - c, c);
            }
            if (with_res) {
                Raw16<T> r[UNITS];
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int c = (i * TPR + t) * 16;
                    r[i].template load<VEC>(res + c, d - c, c);
                }
#pragma unroll
                for (int i = 0; i < UNITS; ++i) {
                    const int c = (i * TPR + t) * 16;
                    h[i].add(r[i]);
                    store_sum(h[i], sum, c);
                }
            }
#pragma unroll
            for (int i = 0; i < UNITS; ++i) take(h[i], w[i], z[i]);
            // elements behind those that a thread keeps: added here, read again below
            for (int c = KEPT + t * 16; c - lane * 16 < d; c += TPR * 16) {
                Raw16<T> v, u;
                float unused[16];
                v.template load<VEC>(x + c, d - c, c);
                if (with_res) {
                    u.template load<VEC>(res + c, d - c, c);
                    v.add(u);
                    store_sum(v, sum, c);
                }
                u.template load<VEC>(g + c, d - c, c);
                take(v, u, unused);
            }
            bits = __float_as_uint(top) & 0x7fffffffu;
        } else {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 16;
                raw[i].template load<VEC>(x + c, d - c, c);
            }
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                most[i] = 0;
                if constexpr (sizeof(T) == 4) {
                    raw[i].h[0].largest(most[i]), raw[i].h[1].largest(most[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) most[i] = larger2<T>(most[i], raw[i].h[j >> 2].w[j & 3]);
                    most[i] &= 0x7fff7fffu;
                }
                bits = sizeof(T) == 4 ? max(bits, most[i]) : __vmaxu2(bits, most[i]);
            }
            for (int c = KEPT + t * 16; c < d; c += TPR * 16) {
                Raw16<T> v;
                v.template load<VEC>(x + c, d - c, c);
                v.h[0].largest(bits), v.h[1].largest(bits);
            }
            bits = Raw8<T>::value(bits);
        }
        reduce<WARPS>(ss, bits, red, turn);
        const bool finite = bits < 0x7f800000u;
        const float amax = __uint_as_float(bits);
        float root = 1.0f, up = 1.0f;      // the row is divided by root / up
        if constexpr (NORM) {
            float eps = prm.eps;
            const bool large = !(ss < 0x1p110f), small = ss < 0x1p-70f && prm.eps < 0x1p-80f;
            if (!std::is_same<T, __half>::value && (large || small)) {
                up = large ? 0x1p-80f : 0x1p96f;
                eps = eps * up * up;
                ss = 0.0f;
                uint32_t unused = 0;
                for (int c = t * 16; c < d; c += TPR * 16) {
                    Raw16<T> v;
                    v.template load<VEC>(again + c, d - c, c);
#pragma unroll
                    for (int j = 0; j < 16; ++j) ss = __fmaf_rn(v.at(j) * up, v.at(j) * up, ss);
                }
                reduce<WARPS>(ss, unused, red, turn);
            }
            root = __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, static_cast<float>(d)), eps));
            // of a large row half of the power on either side of the quotient, so that a large weight's stays in range
            if (up < 1.0f) root *= 0x1p40f, up = 0x1p-40f;
        }
        // v / (root / up); of a small row a small v is scaled first
        auto over_root = [&](float v) {
            return up > 1.0f && v < 1.0f ? __fdiv_rn(__fmul_rn(v, up), root) : __fmul_rn(__fdiv_rn(v, root), up);
        };
        const bool zero = !finite || bits == 0;
        const int e = static_cast<int>(bits >> 23);
        uint8_t *q = prm.q + row * prm.ldq;
        // the elements from c on: those that are kept, or read again
        auto again16 = [&](int c, float (&v)[16]) {
            Raw16<T> h, w;
            h.template load<VEC>(again + c, d - c, c);
            if (NORM) w.template load<VEC>(g + c, d - c, c);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = NORM ? __fmul_rn(h.at(j), w.at(j)) : h.at(j);
        };
        if constexpr (OUT == OUT_I8) {
            if (t == 0)
                prm.scale[row] = finite ? (bits == 0 ? 0.0f : __fdiv_rn(over_root(amax), 127.0f)) : __uint_as_float(0x7fc00000u);
            // rows near the ends of the range are brought to the middle by a power of two
            const bool far = e < 32 || e > 222;
            const int fe = 254 - e < 1 ? 1 : (254 - e > 253 ? 253 : 254 - e);
            const float f = far ? __uint_as_float(static_cast<unsigned>(fe) << 23) : 1.0f;
            const float ntop = amax * f, inv = zero ? 0.0f : __fdiv_ru(127.0f, ntop);
            auto put = [&](int c, const float (&v)[16]) {
                uint2 b[2] = {make_uint2(0u, 0u), make_uint2(0u, 0u)};
                if (!zero) b[0] = to_i8(v, f, inv, ntop, far), b[1] = to_i8(v + 8, f, inv, ntop, far);
                if (VEC || (prm.q16 && c + 16 <= d)) {
                    if (c + 16 <= d) *reinterpret_cast<uint4 *>(q + c) = make_uint4(b[0].x, b[0].y, b[1].x, b[1].y);
                    else *reinterpret_cast<uint2 *>(q + c) = b[0];
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < d) q[c + j] = static_cast<uint8_t>(((j & 7) < 4 ? b[j >> 3].x : b[j >> 3].y) >> (8 * (j & 3)));
                }
            };
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 16;
                if (c < d) put(c, z[i]);
            }
            for (int c = KEPT + t * 16; c < d; c += TPR * 16) {
                float v[16];
                again16(c, v);
                put(c, v);
            }
        } else {
            // amax = m 2^(e - 127), 1 <= m < 2, is at most 2688 r = 1.3125 2^11 r
            int ex = e - 127 - ((bits & 0x7fffffu) <= 0x280000u ? 11 : 10);
            ex = ex < -126 ? -126 : ex;
            const float f = __uint_as_float(static_cast<unsigned>(127 - ex) << 23);
            const float r = __uint_as_float(static_cast<unsigned>(127 + ex) << 23);
            if (t == 0) prm.scale[row] = finite ? (bits == 0 ? 0.0f : NORM ? over_root(r) : r) : __uint_as_float(0x7fc00000u);
            // a row near the ends of the range is scaled by f itself, others' elements stay as they are
            const bool far = ex < -100 || ex > 100;
            const Fp4Row fr{far ? 1.0f : f, far ? 1.0f : r};
            // all lanes of a warp come here together: the scales of four make one word
            auto put = [&](int c, float (&v)[16], float big) {
                uint32_t sb = 0;
                uint2 code = make_uint2(0u, 0u);
                if (!zero) {
                    if (far) {
                        big *= f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] *= f;
                    }
                    sb = to_fp4<!NORM && sizeof(T) == 2>(v, big, fr, code);
                }
                uint32_t word = sb << (8 * (lane & 3));
                word |= __shfl_xor_sync(0xffffffffu, word, 1);
                word |= __shfl_xor_sync(0xffffffffu, word, 2);
                if ((lane & 3) == 0 && c < d) *reinterpret_cast<uint32_t *>(prm.blocks + scale_at(row, c >> 6, kcs)) = word;
                if (c + 16 <= d) {
                    *reinterpret_cast<uint2 *>(q + (c >> 1)) = code;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + 2 * j < d) q[(c >> 1) + j] = static_cast<uint8_t>((j < 4 ? code.x : code.y) >> (8 * (j & 3)));
                }
            };
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int c = (i * TPR + t) * 16;
                if (c - lane * 16 < d) {
                    if constexpr (NORM) {
                        put(c, z[i], largest16(z[i]));
                    } else {
                        float v[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = raw[i].at(j);
                        put(c, v, __uint_as_float(Raw8<T>::value(most[i])));
                    }
                }
            }
            for (int c = KEPT + t * 16; c - lane * 16 < d; c += TPR * 16) {
                float v[16];
                again16(c, v);
                put(c, v, largest16(v));
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
    int wide;                      // rows of y start on 32 bytes
    bool qvec;                     // those of q on 16 (4-bit rows: 8)
};

// code x scale (a 4-bit row's: code x block scale, exact, x row scale), rounded once.  A thread
// takes 16 elements and writes them in whole sectors.  VEC: rows of y start on 8 bytes, q's on 16 (4-bit
// rows: 8); EVEN: d is a multiple of 16.
template <typename T, bool VEC, bool EVEN, int IN>
__global__ void __launch_bounds__(256) values_kernel(const ValuesParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ Turn<T> turns[VEC ? 1 : 8];
    const long long n = prm.rows * prm.units;
    const int lane = threadIdx.x & 31;
    // VEC: each lane for itself; else the lanes of a warp together, those behind the end with nothing
    for (long long at = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; at - (VEC ? 0 : lane) < n; at += static_cast<long long>(gridDim.x) * 256) {
        const bool in = VEC || at < n;
        const long long i = in ? at : n - 1;
        const long long row = i < (1ll << 32) ? static_cast<long long>(udiv_magic(static_cast<uint32_t>(i), prm.magic)) : i / prm.units;
        const int c = static_cast<int>(i - row * prm.units) * 16, d = prm.d;
        const float scale = prm.scale[row];
        const bool whole = VEC && (EVEN || c + 16 <= d), qwhole = VEC ? whole : prm.qvec && c + 16 <= d;
        float v[16];
        if (IN == OUT_I8) {
            const uint8_t *q = prm.q + row * prm.ldq + c;
            uint32_t w[4] = {0, 0, 0, 0};
            if (qwhole) {
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
            if (qwhole) {
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
        if (whole) {
            ips::store16<T>(y, 0, prm.wide, v);
        } else if (VEC) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < d) y[j] = from_f32<T>(v[j]);
        } else {
            Turn<T> &own = turns[threadIdx.x >> 5];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) own.e[lane * Turn<T>::LD + j] = from_f32<T>(v[j]);
            __syncwarp();
            const int left = in ? d - c : 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {      // two lanes' elements at a time
                const int from = 2 * k + (lane >> 4), j = lane & 15;
                T *to = reinterpret_cast<T *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(y), from));
                if (j < __shfl_sync(0xffffffffu, left, from)) to[j] = own.e[from * Turn<T>::LD + j];
            }
        }
    }
}

}  // namespace ipw
