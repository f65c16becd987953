// Device code of the operators with run-time scales for sm_103a: rows quantised to
// int8 with one scale each, and the int8 matrix product with a scale per row of X
// (token) and per row of W (channel).  Floating point holds the scales and, in the
// tensor-core kernel, integers that it represents exactly.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "ip_ptx.cuh"
#include "ip_real.cuh"

namespace ips {

using namespace ipk;
using namespace ipr;

// ---- rows to int8 -------------------------------------------------------
//
// scale = amax / 127 rounded to f32 and q = the integer nearest to 127 x / amax, ties
// to even, for the row's largest magnitude amax.  The quotient is formed as x times
// the reciprocal rounded up (error below 127 2^-23 < 2^-16) and rounded by adding 1.5 2^23.
// That is right except near half integers n + 1/2, where 254 x = (2n + 1) amax is close:
//   16-bit x: with significands X of x and A of amax, integers below 2^11 (bf16: 2^8), a quotient
//     y = 127 x / amax that is no half integer is at least y / (254 X) from one, y 2^-19 (bf16
//     y 2^-16), and the error is below y 2^-23: safe.  Equality needs 2n + 1 = 127, x = amax / 2 (common: one element a row of 1024
//     bf16 values; the reciprocal rounded up takes it to the even 64), or an amax whose
//     significand 127 divides.  In bf16 that is 254 alone, where 127 / amax is a power of
//     two and all quotients are exact; fp16 rows with such an amax (8 of 1024) look at
//     every element: by the quotient of 127 x, which is exact at a half integer.
//   f32 x: units of eight elements with one near a half integer are looked at: within
//     2^-14 of one the exact sign of 254 |x| - (2n + 1) amax decides, both products as
//     unevaluated sums of two floats, whose leading parts differ by little there (an exact
//     subtraction) and whose errors have eight bits.
// An amax near the ends of the range is first brought to [1, 4) by a power of two, its
// row with it, so that nothing of this overflows or underflows.  amax = 0: scale and q
// are 0.  A NaN or an infinity in the row: the scale is NaN and q is 0, so that a product
// with the row is NaN and not a plausible number.
//
// What bounds it: DRAM.  A row stays in registers between the two passes up to
// 8 UNITS elements a thread; a longer one is read again (from L2).  12000 x 4096 bf16
// 26.5 us, 5.6 TB/s; a single row of 1024 1.6 us, a launch's latency.

constexpr int QUANT_THREADS = 256;
constexpr int QUANT_UNITS = 4;      // units of eight elements that a thread keeps

struct QuantParams {
    const void *x;
    long long rows, ldx, ldq;
    int d;
    int8_t *q;
    float *scale;
};

// The low bytes of eight words.
__device__ __forceinline__ uint2 low_bytes(const uint32_t (&k)[8]) {
    return make_uint2(
        __byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410),
        __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410));
}

// Eight elements, each looked at near half integers (out of line: rare, and the registers
// it takes would cost the others their occupancy).
template <typename T>
__device__ __noinline__ uint2 quant_look(Raw8<T> raw, float f, float inv, float top) {
    uint32_t k[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = raw.at(j) * f;
        if constexpr (sizeof(T) == 2) {
            k[j] = static_cast<uint32_t>(__float2int_rn(__fdiv_rn(127.0f * x, top)));
            continue;
        }
        const float y = x * inv, r = __fsub_rn(__fmaf_rn(x, inv, 12582912.0f), 12582912.0f);
        int q = __float2int_rn(r);
        if (fabsf(__fmaf_rn(x, inv, -r)) > 0.5f - 0x1p-14f) {
            const float n = rintf(fabsf(y) - 0.5f), ax = fabsf(x), odd = 2.0f * n + 1.0f;
            const float p1 = 254.0f * ax, e1 = __fmaf_rn(254.0f, ax, -p1);
            const float p2 = odd * top, e2 = __fmaf_rn(odd, top, -p2);
            const float diff = __fadd_rn(__fsub_rn(p1, p2), __fsub_rn(e1, e2));
            const int ni = static_cast<int>(n);
            q = diff > 0.0f ? ni + 1 : (diff < 0.0f ? ni : ni + (ni & 1));
            q = q < 0 ? 0 : q;
            q = x < 0.0f ? -q : q;
        }
        k[j] = static_cast<uint32_t>(q);
    }
    return low_bytes(k);
}

// TPR threads a row (32, 128 or 256).  VEC: x's rows start on 16 bytes, q's on 8 and d is a
// multiple of eight, so that a row's loads are in flight together.
template <typename T, int TPR, bool VEC>
__global__ void __launch_bounds__(QUANT_THREADS) quantize_rows_kernel(const QuantParams prm) {
    constexpr int RPC = QUANT_THREADS / TPR, UNITS = QUANT_UNITS;
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
    __shared__ float red[QUANT_THREADS / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int d = prm.d;
    for (long long r0 = static_cast<long long>(blockIdx.x) * RPC; r0 < prm.rows;
         r0 += static_cast<long long>(gridDim.x) * RPC) {
        const long long row = r0 + sub;
        const bool live = row < prm.rows;
        const T *x = static_cast<const T *>(prm.x) + (live ? row : 0) * prm.ldx;
        Raw8<T> v[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int c = (i * TPR + t) * 8;
            if (live && c < d) v[i].template load<VEC>(x + c, d - c);
            else v[i].zero();
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) v[i].largest(top);
        if (live)
            for (int c = (UNITS * TPR + t) * 8; c < d; c += TPR * 8) {
                Raw8<T> w;
                w.template load<VEC>(x + c, d - c);
                w.largest(top);
            }
        unsigned bits = __reduce_max_sync(0xffffffffu, Raw8<T>::value(top));
        if (TPR > 32) {
            __syncthreads();
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = __uint_as_float(bits);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TPR / 32; ++i) bits = max(bits, __float_as_uint(red[sub * (TPR / 32) + i]));
        }
        if (!live) continue;   // no thread of the row's group is live, all meet at the next row
        const bool finite = bits < 0x7f800000u;
        const float amax = __uint_as_float(bits);
        if (t == 0) prm.scale[row] = finite ? __fdiv_rn(amax, 127.0f) : __uint_as_float(0x7fc00000u);
        const bool zero = !finite || bits == 0;
        // 2^(127 - e) for an amax of exponent field e, kept a normal number; 1 in the middle
        const int e = static_cast<int>(bits >> 23);
        const bool far = e < 32 || e > 222;
        const int fe = 254 - e < 1 ? 1 : (254 - e > 253 ? 253 : 254 - e);
        const float f = far ? __uint_as_float(static_cast<unsigned>(fe) << 23) : 1.0f;
        const float ntop = amax * f, inv = zero ? 0.0f : __fdiv_ru(127.0f, ntop);
        // rows near the ends of the range go the same way
        const bool look = !zero && (far || (sizeof(T) == 2 && !BF16 && ((bits & 0x7fffffu) | 0x800000u) % 127u == 0));
        int8_t *q = prm.q + row * prm.ldq;
        auto put = [&](int c, const Raw8<T> &raw) {
            uint2 b = make_uint2(0u, 0u);
            if (look) {
                b = quant_look(raw, f, inv, ntop);
            } else if (!zero) {
                uint32_t k[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)      // the integer in two's complement below bit 22
                    k[j] = __float_as_uint(__fmaf_rn(raw.at(j), inv, 12582912.0f));
                b = low_bytes(k);
                if (sizeof(T) == 4) {
                    float off = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        off = fmaxf(off, fabsf(__fmaf_rn(raw.at(j), inv, -__fsub_rn(__uint_as_float(k[j]), 12582912.0f))));
                    if (off > 0.5f - 0x1p-14f) b = quant_look(raw, f, inv, ntop);
                }
            }
            if (VEC) {
                *reinterpret_cast<uint2 *>(q + c) = b;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < d) q[c + j] = static_cast<int8_t>((j < 4 ? b.x : b.y) >> (8 * (j & 3)));
            }
        };
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int c = (i * TPR + t) * 8;
            if (c < d) put(c, v[i]);
        }
        for (int c = (UNITS * TPR + t) * 8; c < d; c += TPR * 8) {
            Raw8<T> w;
            w.template load<VEC>(x + c, d - c);
            put(c, w);
        }
    }
}

// ---- the scaled product -------------------------------------------------
//
// y[m][n] = act(sx[m] sw[n] S + bias[n]), S = sum_k x[m][k] w[n][k] as an exact
// integer, act the identity or z / (1 + exp(-z)).

constexpr int ERR_TIMEOUT = 1;      // status word: a barrier wait ran out
// Bound of the waits for a CTA's own copies and MMAs in flight once it has given up, whatever the
// limit of the others: it must not end before them.
constexpr long long LAND_CYCLES = 4000000000ll;

struct ScaledParams {
    const int8_t *x, *w;            // the vector kernel's operands (the tiles come by TMA)
    const float *sx, *sw, *bias;
    void *y;
    long long M, ldx, ldw, ldy;
    int K, N, act;
    int splits;                     // CTAs that share a tile's K
    int tiles_n;
    long long tiles;
    int *err;
    long long timeout_cycles;
    int stall;                      // test hook: the output warps first wait on a barrier that nothing arrives on
};

// z / (1 + exp(-z)) is formed with t = exp(-|z|) <= 1, so that nothing overflows: z / (1 + t) or
// z t / (1 + t).  For 16-bit outputs t and the reciprocal of 1 + t, in [1, 2], come from the
// approximate units (2^-22 and less; the argument's rounding adds |z| 2^-24).
template <typename T>
__device__ __forceinline__ float swish(float z) {
    if (sizeof(T) == 4) {
        const float t = expf(-fabsf(z));
        return __fdiv_rn(z < 0.0f ? z * t : z, 1.0f + t);
    }
    float t, r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(t) : "f"(fabsf(z) * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + t));
    return (z < 0.0f ? z * t : z) * r;
}
template <typename T>
__device__ __forceinline__ float finish(float s, float scale, float bias, int act) {
    const float z = __fmaf_rn(s, scale, bias);
    return act ? swish<T>(z) : z;
}

// Few tokens: the weights are read once and the products formed by dp4a.  KT threads share
// a channel's K in chunks of 16 bytes (64 where K is short, all 256 of the CTA where it is
// long, so that a thread has one or two rounds of loads), a thread takes CPT channels, so
// that each chunk of x is loaded once for them, and 256 / KT x CPT channels are a CTA's.
// Bound by latency and the weights' bytes: 1 x 1024 -> 4096 2.0 us, 8 x 4096 -> 1024 3.2 us
// (4.2 MB of weights each, from L2).
constexpr int VEC_THREADS = 256;

__device__ __forceinline__ uint4 chunk16(const int8_t *p, int n) {
    if (n >= 16) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4] = {0, 0, 0, 0};
    for (int i = 0; i < n; ++i)
        w[i >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(p[i])) << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ONE: K fits one round of chunks, whose x a thread keeps for all its channels.
template <typename T, int MT, int CPT, int KT, bool ONE>
__global__ void __launch_bounds__(VEC_THREADS) scaled_vec_kernel(const ScaledParams prm) {
    constexpr int GROUPS = VEC_THREADS / KT, WARPS = KT / 32, BLOCK = GROUPS * CPT;
    __shared__ int part[2][GROUPS][WARPS][MT * CPT];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % KT, g = threadIdx.x / KT;
    const long long m0 = static_cast<long long>(blockIdx.y) * MT;
    const int mv = static_cast<int>(prm.M - m0 < MT ? prm.M - m0 : MT);
    auto load_x = [&](uint4 (&x)[MT], int k) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
            x[i] = i < mv && k < prm.K ? chunk16(prm.x + (m0 + i) * prm.ldx + k, prm.K - k) : make_uint4(0, 0, 0, 0);
    };
    uint4 x[MT];
    if (ONE) load_x(x, t * 16);
    int turn = 0;
    for (int c0 = static_cast<int>(blockIdx.x) * BLOCK; c0 < prm.N; c0 += static_cast<int>(gridDim.x) * BLOCK) {
        const int n0 = c0 + g * CPT;
        int acc[MT][CPT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < CPT; ++j) acc[i][j] = 0;
        for (int k = t * 16; k < (ONE ? t * 16 + 1 : prm.K); k += KT * 16) {
            uint4 w[CPT];
#pragma unroll
            for (int j = 0; j < CPT; ++j)
                w[j] = n0 + j < prm.N && k < prm.K ? chunk16(prm.w + (n0 + j) * prm.ldw + k, prm.K - k)
                                                   : make_uint4(0, 0, 0, 0);
            if (!ONE) load_x(x, k);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < CPT; ++j) {
                    int a = acc[i][j];
                    a = __dp4a(static_cast<int>(x[i].x), static_cast<int>(w[j].x), a);
                    a = __dp4a(static_cast<int>(x[i].y), static_cast<int>(w[j].y), a);
                    a = __dp4a(static_cast<int>(x[i].z), static_cast<int>(w[j].z), a);
                    acc[i][j] = __dp4a(static_cast<int>(x[i].w), static_cast<int>(w[j].w), a);
                }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < CPT; ++j) {
                const int s = __reduce_add_sync(0xffffffffu, acc[i][j]);
                if ((threadIdx.x & 31) == 0) part[turn][g][t >> 5][i * CPT + j] = s;
            }
        __syncthreads();       // the other half of `part` is read until the next one
        // consecutive threads finish consecutive channels of a token
        for (int e = threadIdx.x; e < MT * BLOCK; e += VEC_THREADS) {
            const int i = e / BLOCK, c = e % BLOCK, n = c0 + c;
            if (i >= mv || n >= prm.N) continue;
            int s = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += part[turn][c / CPT][w][i * CPT + c % CPT];
            const float z = finish<T>(static_cast<float>(s), prm.sx[m0 + i] * prm.sw[n],
                                      prm.bias ? prm.bias[n] : 0.0f, prm.act);
            static_cast<T *>(prm.y)[(m0 + i) * prm.ldy + n] = from_f32<T>(z);
        }
        turn ^= 1;
    }
}

// Many tokens: tiles of 128 tokens x BN channels on the fp16 tensor cores, or of 256 x 256 by
// two CTAs (PAIR).
//
// sm_103a has no integer tcgen05 kind, and its integer warp MMA and dp4a together
// reach 289 TOPS; but fp16 holds every int8 value, the product of two is exact in the
// fp32 accumulator, and so is every partial sum up to 2^24: at most 1024 products of
// magnitude 2^14.  So the K axis runs in segments of 1024, each summed exactly in
// TMEM, and the segments are added as int32 in registers.
//
// Roles of a persistent CTA (one per SM): warp 16 fetches raw stages of 64 K bytes of
// both operands by TMA, warps 8-15 convert them to fp16 in the 128-byte swizzled
// K-major layout of the MMA, one thread of warp 17 issues tcgen05.mma, warps 0-7
// drain one of two TMEM accumulators and write the output while the other fills.
//
// What bounds it: the conversion's shared-memory accesses (a read and two writes per operand
// byte), which the MMA's own operand reads share the pipe with, and the epilogue's time
// where K is short.  So the CTAs of a pair share their channels: each converts its 128
// tokens and half of the 256 channels for an MMA of 256 x 256 (cta_group::2), a third
// less for the same products (a CTA alone on 128 x 256: 80 % of that pipe, the tensor pipe
// at 36 %).  12000 x 1024 -> 4096 97 us (without the epilogue's arithmetic and stores some
// 20 less, without the conversion as well some 35), 12000 x 4096 -> 1024 100 us (188 pair
// tiles for 76 pairs: the third round is half empty; its tiles cut in halves of 128
// channels gave 5 us there and cost up to 2 elsewhere), 4096 x 8192 -> 8192 431 us,
// 1275 TFLOP/s.

constexpr int TILE_M = 128;
constexpr int BK = 64;              // K elements of a stage (rows of 64 bytes raw, of 128 in fp16)
constexpr int SEG = 1024 / BK;      // stages of an exact segment
constexpr int TC_THREADS = 640;     // five warpgroups (registers are dealt by warpgroup)
constexpr int TC_REGS = 96;         // registers a thread at launch
constexpr int EPI_WARPS = 8, CONV_WARPS = 8, CONV_GROUPS = 4;
constexpr int TMA_WARP = 16, MMA_WARP = 17;

constexpr int TURN_LD = 17, TURN_BYTES = 16 * TURN_LD * 4;

template <int BN_, bool PAIR_>
struct Tile {
    static constexpr int BN = BN_;
    static constexpr int CTAS = PAIR_ ? 2 : 1;
    static constexpr int BR = BN / CTAS;              // channels that a CTA converts
    static constexpr int RAW = (TILE_M + BR) * BK;
    static constexpr int F16 = (TILE_M + BR) * BK * 2;
    static constexpr int RS = BN == 32 ? 8 : 5;       // raw stages (as many bytes in two stages of 128: 20 % slower)
    static constexpr int FS = 4;                      // fp16 stages
    // A parity is also that of the phase two before, and a group of warps sees every CONV_GROUPS-th
    // stage only.  The slot of its next fp16 stage was its own before, so that wait is unambiguous; it
    // says that the MMA is done with all stages up to FS back, so the raw slot's stage before, RS
    // back, has landed too: the raw barrier may be asked after the fp16 one, not before it.
    static_assert(FS % CONV_GROUPS == 0 && RS >= FS, "phases");
    static constexpr int BARS = 0;                    // 2 RS + 2 FS + 6 barriers
    static constexpr int TMEM_PTR = 256, DEAD = 260;
    static constexpr int CONSTS = 512;                // per epilogue warp: sw and bias of its columns
    // the sums of a tile, where the CTAs of a cluster share its K
    static constexpr int TURN = CONSTS + EPI_WARPS * 2 * 4 * (BN / 2);      // per epilogue warp: store_odd's block
    static constexpr int SUMS_AT = (TURN + EPI_WARPS * TURN_BYTES + 1023) & ~1023;
    static constexpr int F16_AT = SUMS_AT + (BN == 32 ? 4 * TILE_M * BN : 0);
    static constexpr int RAW_AT = F16_AT + FS * F16;
    static constexpr int SMEM = RAW_AT + RS * RAW + 1024;
    static constexpr int COLS = 2 * BN;               // TMEM columns
    static_assert(8 * (2 * RS + 2 * FS + 6) <= 256, "barriers");
    static_assert(SMEM <= 232448, "shared memory");
    static_assert((COLS & (COLS - 1)) == 0 && COLS <= 512, "TMEM columns");
};

// Four int8 values to fp16 pairs, exactly: with its sign bit flipped a byte is u = b +
// 128, and 0x6400 | u is the fp16 number 1024 + u.
__device__ __forceinline__ void cvt4(uint32_t w, uint32_t &lo, uint32_t &hi) {
    const uint32_t u = w ^ 0x80808080u;
    uint32_t a, b;
    asm("prmt.b32 %0, %1, %2, 0x4140;" : "=r"(a) : "r"(u), "r"(0x64646464u));
    asm("prmt.b32 %0, %1, %2, 0x4342;" : "=r"(b) : "r"(u), "r"(0x64646464u));
    const uint32_t c = 0xe480e480u;   // -1152
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(c));
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(c));
}

// One poll of a barrier that threads of the other CTA of a pair arrive on as well.
template <bool PAIR>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    if (!PAIR) return mbar_try_wait(bar, parity);
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait that also ends when another role of the CTA has given up.
template <bool PAIR>
__device__ __forceinline__ bool wait_or_dead(uint32_t bar, uint32_t parity, volatile int *dead,
                                             long long limit) {
    if (try_wait<PAIR>(bar, parity)) return true;
    const long long t0 = clock64();
    while (!try_wait<PAIR>(bar, parity)) {
        if (*dead) return false;
        if (clock64() - t0 > limit) {
            *dead = 1;
            return false;
        }
    }
    return true;
}
template <bool PAIR>
__device__ __forceinline__ bool warp_wait_or_dead(uint32_t bar, uint32_t parity, volatile int *dead,
                                                  long long limit) {
    return __all_sync(0xffffffffu, wait_or_dead<PAIR>(bar, parity, dead, limit)) != 0;
}
// Arrives on the barrier at this shared-memory offset of the pair's first CTA.
template <bool PAIR>
__device__ __forceinline__ void arrive_first(uint32_t bar) {
    if (!PAIR) {
        mbar_arrive(bar);
        return;
    }
    asm volatile(
        "{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, 0;\n"
        " mbarrier.arrive.release.cluster.shared::cluster.b64 _, [r];\n}\n" ::"r"(bar)
        : "memory");
}
// Word at this shared-memory offset of the cluster's CTA `rank`.
__device__ __forceinline__ int ld_cluster(uint32_t addr, int rank) {
    int v;
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %1, %2;\n ld.shared::cluster.s32 %0, [r];\n}\n"
                 : "=r"(v)
                 : "r"(addr), "r"(rank)
                 : "memory");
    return v;
}
// True in one lane of a converged warp, always the same.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared-memory descriptor of a K-major operand with 128-byte swizzle: rows of 128
// bytes, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3ffff) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) |
           (2ull << 61);
}

template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                        uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// Arrives on the barrier (of both CTAs of a pair) when the MMAs so far have completed.
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if (PAIR)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                bar),
            "h"(static_cast<uint16_t>(3))
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
                     : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t at, int cols) {
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t tmem, int cols) {
    if (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15},"
        " [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// 16 outputs of one token from column n on, in stores of 32 bytes (WIDE) or 8, as all rows are
// aligned.  Whole sectors straight from the registers: the blocks that TMA stores need take the room of a raw stage (12000 x 1024
// -> 4096 3 us less, but 12000 x 4096 -> 1024 11 us more), and a tensor store writes behind
// column N up to the next 16 bytes.
template <typename T>
__device__ __forceinline__ void store16(T *row, int n, bool wide, const float (&z)[16]) {
    constexpr int WORDS = 4 * sizeof(T);
    union { T e[16]; uint32_t w[WORDS]; } v;
#pragma unroll
    for (int j = 0; j < 16; ++j) v.e[j] = from_f32<T>(z[j]);
    const uint32_t (&w)[WORDS] = v.w;
    uint32_t *p = reinterpret_cast<uint32_t *>(row + n);
    if (wide) {
#pragma unroll
        for (int i = 0; i < WORDS; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p + i), "r"(w[i]), "r"(w[i + 1]),
                         "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < WORDS; i += 2) *reinterpret_cast<uint2 *>(p + i) = make_uint2(w[i], w[i + 1]);
    }
}
// 16 columns of the tokens of a warp's lanes for rows of any alignment, `rows` and `cols` of them (y: the
// first token's first): turned in shared memory, 16 tokens at a time, so that half a warp writes
// consecutive columns (12000 x 1024 -> 4097 in bf16: 164 us, a lane a row 476).
template <typename T>
__device__ __forceinline__ void store_odd(T *y, long long ldy, int rows, int cols, uint32_t turn, const float (&z)[16]) {
    const int lane = threadIdx.x & 31, half = lane >> 4, col = lane & 15;
    y += half * ldy + col;
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
        __syncwarp();
        if (half == h)
#pragma unroll
            for (int j = 0; j < 16; ++j) sts32(turn + 4 * (col * TURN_LD + j), __float_as_uint(z[j]));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float x = __uint_as_float(lds32(turn + 4 * ((i + half) * TURN_LD + col)));
            if (16 * h + i + half < rows && col < cols) y[(16 * h + i) * ldy] = from_f32<T>(x);
        }
    }
}

// LONG: a CTA's K is longer than 1024, several segments per tile.  KSPLIT: the CTAs of a cluster
// share one tile's K and add their sums through each other's shared memory, a part of the
// rows each (few tiles: 64 x 4096 -> 1024 in 32 tiles 20 us, by clusters of four 10).
// ODD: output rows that are not aligned to 8 bytes, or an N that 16 does not divide (for the others the
// registers of store_odd would cost 12000 x 4096 -> 1024 104 us for 98).
template <typename T, int BN, bool LONG, bool PAIR, bool KSPLIT, bool ODD>
__global__ void __launch_bounds__(TC_THREADS, 1)
    scaled_tc_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w,
                     const ScaledParams prm) {
    using C = Tile<BN, PAIR>;
    // The sums of a long K take 128 registers of an epilogue thread (BN = 256): its warpgroups
    // take over what the others can spare, 2 x 168 + 2 x 56 + 32 = 5 x 96.
    constexpr bool DEAL = LONG && BN == 256;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    auto raw_full = [&](int s) { return base + C::BARS + 8u * s; };
    auto raw_empty = [&](int s) { return base + C::BARS + 8u * (C::RS + s); };
    auto f16_full = [&](int s) { return base + C::BARS + 8u * (2 * C::RS + s); };
    auto f16_empty = [&](int s) { return base + C::BARS + 8u * (2 * C::RS + C::FS + s); };
    auto acc_full = [&](int s) { return base + C::BARS + 8u * (2 * C::RS + 2 * C::FS + s); };
    auto acc_empty = [&](int s) { return base + C::BARS + 8u * (2 * C::RS + 2 * C::FS + 2 + s); };
    const uint32_t drained = base + C::BARS + 8u * (2 * C::RS + 2 * C::FS + 4), never = drained + 8u;
    volatile int *dead = reinterpret_cast<volatile int *>(smem + C::DEAD);
    const int rank = PAIR ? static_cast<int>(blockIdx.x & 1u) : 0;      // clusters are (2, 1, 1)
    static_assert(!KSPLIT || (BN == 32 && !PAIR), "room for the sums");
    const int splits = KSPLIT ? prm.splits : 1;                         // else clusters are (splits, 1, 1)
    const int part = KSPLIT ? static_cast<int>(blockIdx.x) % splits : 0;
    const long long worker = blockIdx.x / (KSPLIT ? splits : C::CTAS), workers = gridDim.x / (KSPLIT ? splits : C::CTAS);

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::RS; ++s) {
            mbar_init(raw_full(s), 1);
            mbar_init(raw_empty(s), CONV_WARPS / CONV_GROUPS);
        }
        for (int s = 0; s < C::FS; ++s) {
            mbar_init(f16_full(s), CONV_WARPS / CONV_GROUPS * C::CTAS);
            mbar_init(f16_empty(s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full(s), 1);
            mbar_init(acc_empty(s), EPI_WARPS * C::CTAS);
        }
        mbar_init(drained, 1);
        mbar_init(never, 1);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    if (PAIR) cluster_sync();
    if (warp == MMA_WARP) tmem_alloc<PAIR>(base + C::TMEM_PTR, C::COLS);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (PAIR) cluster_sync();
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // only now: a CTA of the next launch that took this SM's TMEM first would wait for
    // this grid with it
    pdl_launch_dependents();
    const uint32_t tmem = lds32(base + C::TMEM_PTR);
    pdl_wait();

    // stages of this CTA: st0 .. st1 - 1 of all (K behind the end reads as 0)
    const int all = (prm.K + BK - 1) / BK;
    const int st0 = KSPLIT ? all * part / splits : 0, st1 = KSPLIT ? all * (part + 1) / splits : all;
    const int stages = st1 - st0;
    const long long limit = prm.timeout_cycles;

    if (warp >= EPI_WARPS + CONV_WARPS) {
        if (DEAL) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        if (warp == TMA_WARP && lane == 0) {
            int s = 0, ph = 0;
            long long issued = 0;
            bool ok = true;
            for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
                const int m0 = static_cast<int>(tile / prm.tiles_n) * (TILE_M * C::CTAS) + rank * TILE_M;
                const int n0 = static_cast<int>(tile % prm.tiles_n) * BN + rank * C::BR;
                for (int k = st0 * BK; k < st1 * BK; k += BK) {
                    ok = wait_or_dead<false>(raw_empty(s), ph ^ 1, dead, limit);
                    if (!ok) break;
                    const uint32_t st = base + C::RAW_AT + s * C::RAW;
                    mbar_expect_tx(raw_full(s), C::RAW);
                    tma_load_2d(st, &tm_x, k, m0, raw_full(s));
                    tma_load_2d(st + TILE_M * BK, &tm_w, k, n0, raw_full(s));
                    ++issued;
                    if (++s == C::RS) s = 0, ph ^= 1;
                }
            }
            // after a wait that ran out: the copies in flight land before the CTA ends
            if (!ok)
                for (long long i = issued > C::RS ? issued - C::RS : 0; i < issued; ++i)
                    mbar_wait(raw_full(static_cast<int>(i % C::RS)),
                              static_cast<uint32_t>((i / C::RS) & 1), LAND_CYCLES);
        } else if (warp == MMA_WARP && rank == 0) {
            // the whole warp runs the loop, so that the descriptors stay uniform; one lane issues
            constexpr uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(BN / 8) << 17) |
                                       (static_cast<uint32_t>(TILE_M * C::CTAS / 16) << 24);
            int s = 0, ph = 0, a = 0, aph = 0;
            bool ok = true;
            for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
                for (int it = 0; ok && it < stages;) {
                    ok = warp_wait_or_dead<PAIR>(acc_empty(a), aph ^ 1, dead, limit);
                    if (!ok) break;
                    const int end = it + SEG < stages ? it + SEG : stages;
                    for (int first = it; it < end; ++it) {
                        ok = warp_wait_or_dead<PAIR>(f16_full(s), ph, dead, limit);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t st = base + C::F16_AT + s * C::F16;
                        const uint64_t da = smem_desc(st), db = smem_desc(st + TILE_M * BK * 2);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k)
                                mma_f16<PAIR>(tmem + a * BN, da + 2 * k, db + 2 * k, idesc, it > first || k > 0);
                            mma_commit<PAIR>(f16_empty(s));
                        }
                        __syncwarp();
                        if (++s == C::FS) s = 0, ph ^= 1;
                    }
                    if (!ok) break;
                    if (elect_one()) mma_commit<PAIR>(acc_full(a));
                    __syncwarp();
                    a ^= 1;
                    aph ^= a == 0;
                }
            }
            if (!ok) {   // the MMAs in flight end before their TMEM is freed
                if (elect_one()) mma_commit<PAIR>(drained);
                __syncwarp();
                mbar_wait(drained, 0, LAND_CYCLES);
            }
        }
    } else if (warp >= EPI_WARPS) {
        if (DEAL) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // The warps form CONV_GROUPS groups that take the stages in turn, so that one group's
        // loads and fence overlap the others' arithmetic.
        constexpr int UNITS = (TILE_M + C::BR) / 8;   // of eight rows
        constexpr int GW = CONV_WARPS / CONV_GROUPS, PER = (UNITS + GW - 1) / GW;
        const int cw = (warp - EPI_WARPS) % GW, grp = (warp - EPI_WARPS) / GW;
        // A unit is eight rows (past the end of X or W zeros, converted like the others: a second loop
        // that leaves them out costs registers, 12000 x 4096 -> 1024 107 us for 98).  A lane takes 16 bytes of row r8: a quarter-warp reads 128 consecutive
        // bytes, two rows, whose fp16 chunks of one parity fall on different banks under the swizzle.
        const int r8 = lane >> 2, j = lane & 3;
        const uint32_t d0 = swz(r8, 2 * j), d1 = swz(r8, 2 * j + 1);
        int rs = 0, rph = 0, fs = 0, fph = 0, turn = 0;
        bool ok = true;
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
            for (int it = 0; it < stages; ++it) {
                if (turn == grp) {
                    // in this order (Tile's phases); a wait that ran out shows after both
                    ok = wait_or_dead<PAIR>(f16_empty(fs), fph ^ 1, dead, limit);
                    ok = wait_or_dead<false>(raw_full(rs), rph, dead, limit) && ok;
                    if (!__all_sync(0xffffffffu, ok)) {
                        ok = false;
                        break;
                    }
                    const uint32_t src = base + C::RAW_AT + rs * C::RAW + lane * 16;
                    const uint32_t dst = base + C::F16_AT + fs * C::F16;
                    static_assert(UNITS % GW == 0, "units");
                    constexpr int AHEAD = PER < 4 ? PER : 4;
                    uint4 v[AHEAD];
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) v[i] = lds128(src + (i * GW + cw) * 512);
                    auto one = [&](int u, const uint4 &v) {
                        uint32_t h[8];
                        cvt4(v.x, h[0], h[1]);
                        cvt4(v.y, h[2], h[3]);
                        cvt4(v.z, h[4], h[5]);
                        cvt4(v.w, h[6], h[7]);
                        sts128(dst + u * 1024 + d0, h[0], h[1], h[2], h[3]);
                        sts128(dst + u * 1024 + d1, h[4], h[5], h[6], h[7]);
                    };
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        one(i * GW + cw, v[i % AHEAD]);
                        if (i + AHEAD < PER) v[i % AHEAD] = lds128(src + ((i + AHEAD) * GW + cw) * 512);
                    }
                    // the fp16 stage to the MMA, the raw stage to the next TMA copy
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        arrive_first<PAIR>(f16_full(fs));
                        mbar_arrive(raw_empty(rs));
                    }
                }
                if (++rs == C::RS) rs = 0, rph ^= 1;
                if (++fs == C::FS) fs = 0, fph ^= 1;
                if (++turn == CONV_GROUPS) turn = 0;
            }
        }
    } else {
        if (DEAL) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        const int quarter = warp & 3, half = warp >> 2;
        constexpr int CW = BN / 2;            // columns of a warp
        constexpr int CH = CW < 16 ? 1 : CW / 16;
        const int col0 = half * CW;
        const unsigned low = static_cast<unsigned>(reinterpret_cast<uintptr_t>(prm.y) | (prm.ldy * sizeof(T))) & 31u;
        const bool wide = low == 0, even = (low & 7u) == 0;
        const uint32_t cst = base + C::CONSTS + warp * (8 * CW);
        int a = 0, aph = 0;
        bool ok = true;
        if (prm.stall) ok = warp_wait_or_dead<false>(never, 0, dead, limit);
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
            const long long mq = tile / prm.tiles_n * (TILE_M * C::CTAS) + rank * TILE_M + quarter * 32, m = mq + lane;
            const int n0 = static_cast<int>(tile % prm.tiles_n) * BN + col0;
            __syncwarp();
            for (int c = lane; c < CW; c += 32) {
                const int n = n0 + c;
                sts32(cst + 4 * c, __float_as_uint(n < prm.N ? prm.sw[n] : 0.0f));
                sts32(cst + 4 * (CW + c), __float_as_uint(n < prm.N && prm.bias ? prm.bias[n] : 0.0f));
            }
            __syncwarp();
            const float sx = m < prm.M ? prm.sx[m] : 0.0f;
            T *row = static_cast<T *>(prm.y) + (m < prm.M ? m : 0) * prm.ldy;
            auto write = [&](int ch, const float (&s)[16]) {
                const int c = 16 * ch;
                float z[16];
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint4 w4 = lds128(cst + 4 * (c + i));
                    const uint4 b4 = lds128(cst + 4 * (CW + c + i));
                    z[i] = __fmaf_rn(s[i], sx * __uint_as_float(w4.x), __uint_as_float(b4.x));
                    z[i + 1] = __fmaf_rn(s[i + 1], sx * __uint_as_float(w4.y), __uint_as_float(b4.y));
                    z[i + 2] = __fmaf_rn(s[i + 2], sx * __uint_as_float(w4.z), __uint_as_float(b4.z));
                    z[i + 3] = __fmaf_rn(s[i + 3], sx * __uint_as_float(w4.w), __uint_as_float(b4.w));
                }
                if (prm.act)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = swish<T>(z[i]);
                if (ODD && (!even || n0 + c + 16 > prm.N)) {
                    const long long first = m - lane, left = prm.M - first;
                    if (n0 + c < prm.N)
                        store_odd<T>(static_cast<T *>(prm.y) + first * prm.ldy + n0 + c, prm.ldy,
                                     left < 32 ? static_cast<int>(left) : 32, prm.N - n0 - c,
                                     base + C::TURN + warp * TURN_BYTES, z);
                } else if (m < prm.M && n0 + c < prm.N) {
                    store16<T>(row, n0 + c, wide, z);
                }
            };
            int sum[LONG || KSPLIT ? CH : 1][16];
            if (LONG || KSPLIT)
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[c][i] = 0;
            for (int it = 0; it < stages; it += SEG) {
                ok = warp_wait_or_dead<PAIR>(acc_full(a), aph, dead, limit);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = tmem + a * BN + col0 + (static_cast<uint32_t>(quarter * 32) << 16);
                uint32_t r[2][16];      // the next columns are fetched while these are worked on
                tmem_ld16(at, r[0]);
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    tmem_wait_ld();
                    if (c + 1 < CH) tmem_ld16(at + 16 * (c + 1), r[(c + 1) & 1]);
                    const uint32_t (&v)[16] = r[c & 1];
                    if (LONG || KSPLIT) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c][i] += __float2int_rn(__uint_as_float(v[i]));
                    } else {
                        float s[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __uint_as_float(v[i]);
                        write(c, s);
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_first<PAIR>(acc_empty(a));
                a ^= 1;
                aph ^= a == 0;
            }
            if (KSPLIT && ok) {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    sts128(base + C::SUMS_AT + 4u * ((quarter * 32 + lane) * BN + col0 + i), sum[0][i], sum[0][i + 1],
                           sum[0][i + 2], sum[0][i + 3]);
            } else if (LONG && ok) {
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    float s[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = static_cast<float>(sum[c][i]);
                    write(c, s);
                }
            }
        }
    }
    __syncwarp();
    if (KSPLIT) {
        cluster_sync();           // every part's sums are in place
        const int row0 = TILE_M * part / splits, rows = TILE_M * (part + 1) / splits - row0;
        const long long m0 = worker / prm.tiles_n * TILE_M;
        const int n0 = static_cast<int>(worker % prm.tiles_n) * BN;
        for (int e = threadIdx.x; e < rows * BN; e += TC_THREADS) {
            const int r = row0 + e / BN, c = e % BN, n = n0 + c;
            if (m0 + r >= prm.M || n >= prm.N) continue;
            int sum = 0;
            for (int i = 0; i < splits; ++i) sum += ld_cluster(base + C::SUMS_AT + 4u * (r * BN + c), i);
            static_cast<T *>(prm.y)[(m0 + r) * prm.ldy + n] =
                from_f32<T>(finish<T>(static_cast<float>(sum), prm.sx[m0 + r] * prm.sw[n],
                                      prm.bias ? prm.bias[n] : 0.0f, prm.act));
        }
        cluster_sync();           // no part ends while another reads its sums
    }
    if (PAIR) cluster_sync();     // neither CTA ends while the other may still arrive on its barriers
    else __syncthreads();
    if (warp == MMA_WARP) tmem_free<PAIR>(tmem, C::COLS);
    if (threadIdx.x == 0 && *dead) atomicOr(prm.err, ERR_TIMEOUT);
}

}  // namespace ips
