// Device code of the product of 4-bit rows for sm_103a (e2m1 codes, e4m3 scales of 16, an f32 scale a
// row) on the block-scaled tensor cores.
#pragma once

#include <stdint.h>

#include "ip_scaled_kernels.cuh"

namespace ip4 {

using namespace ipk;
using namespace ipr;
using ips::elect_one, ips::cluster_sync, ips::mma_commit, ips::tmem_alloc, ips::tmem_free, ips::tmem_wait_ld, ips::smem_desc;

// y[m][n] = act(sx[m] sw[n] S + bias[n]), S = sum over blocks of s_x s_w sum of 16 code products, by
// tcgen05.mma kind::mxf4nvf4 with a scale for each 16 elements: products and scales are exact there, sums
// in f32.
//
// Roles of a persistent CTA (one an SM): warps 20, 22 and 23 fetch stages of 256 elements of K by TMA (128 rows of
// x and BN channels of w, 128 bytes each in the 128-byte swizzled layout, and their scales as they
// lie in memory, 512 bytes for 128 rows x 64 elements), warps 16-19 copy the scales to TMEM, one
// thread of warp 21 issues the MMAs of 64 elements each, warps 0-15 take the sums to registers, release
// the accumulator and write the output while the next tile is summed.
// PAIR: two CTAs share a tile of 256 rows x BN channels (cta_group::2), each fetching its 128 rows and half of
// the channels; the scales of all channels go to both.  Both CTAs' copies report to the first one's
// barriers, whose warp 21 issues for both.

constexpr int TILE_M = 128;
constexpr int BKB = 128;                 // bytes of a row in a stage
constexpr int BK = 256;                  // elements
constexpr int THREADS = 768;             // six warpgroups (registers are dealt by warpgroup)
constexpr int REGS = 80;                 // registers a thread at launch
constexpr int EPI_WARPS = 16, SCALE_WARP = 16, X_WARP = 20, MMA_WARP = 21, W_WARP = 22, SCALES_WARP = 23;

struct Params {
    const float *sx, *sw, *bias;
    void *y;
    long long M, ldy;
    int N, act;
    int steps;                           // of 64 elements
    int tiles_n;
    long long tiles;
    int *err;
    long long timeout_cycles;
    int stall;
};

template <int BN_, bool PAIR_>
struct Tile {
    static constexpr int BN = BN_;
    static constexpr int CTAS = PAIR_ ? 2 : 1;
    static constexpr int BR = BN / CTAS;              // channels that a CTA fetches
    static constexpr int WT = BN <= 128 ? 1 : BN / 128;      // tiles of scales of w
    static constexpr int A = TILE_M * BKB, B = BR * BKB, SA = 2048, SB = 2048 * WT;
    static constexpr int STAGE = A + B + SA + SB;
    static constexpr int ST = BN == 64 ? 6 : 5;
    static constexpr int ACCS = BN == 256 ? 1 : 2;    // accumulators
    static constexpr int SF = ACCS * BN;              // first column of the scales
    static constexpr int SF_COLS = 16 + 16 * WT;      // of a stage
    static constexpr int COLS = 512;
    static constexpr int TMEM_PTR = 256, DEAD = 260;
    static constexpr int FETCHED = 272;               // stages, of x, of w and of scales
    static constexpr int OTHER = 288;                 // of the other CTA of a pair: given up, -, stages fetched
    static constexpr int CONSTS = 512;                // sw and bias of a tile's columns
    // per output warp: a block of 32 rows x 64 bytes on its way out
    static constexpr int OUT_AT = (CONSTS + 8 * BN + 1023) & ~1023, OUT = 2048;
    static constexpr int STAGES_AT = OUT_AT + EPI_WARPS * OUT;
    static constexpr int SMEM = STAGES_AT + ST * STAGE + 1024;
    static_assert(8 * (4 * ST + 6) <= 256, "barriers");
    static_assert(SMEM <= 232448, "shared memory");
    static_assert(SF + ST * SF_COLS <= COLS, "TMEM columns");
    static_assert(STAGE % 1024 == 0 && B % 1024 == 0 , "alignment");
};

// Waits acquire, within the CTA: the scale warps read with ordinary loads what the copies left (volatile, as the waits are, so
// that the compiler keeps their order).  A pair's arrivals on the first CTA's
// barriers release nothing: what they report are TMEM and tiles, which only asynchronous units touch and the
// tcgen05 fences order, and with the release of the cluster they take 0.7 us each (12000 x 16384 -> 1024: 164 us, relaxed 87).
// Bounded wait that also ends when another role of the CTA has given up.
__device__ __forceinline__ bool wait_or_dead(uint32_t bar, uint32_t parity, volatile int *dead, long long limit) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity)) {
        if (*dead) return false;
        if (clock64() - t0 > limit) {
            *dead = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool warp_wait_or_dead(uint32_t bar, uint32_t parity, volatile int *dead, long long limit) {
    return __all_sync(0xffffffffu, wait_or_dead(bar, parity, dead, limit)) != 0;
}

template <bool PAIR>
__device__ __forceinline__ void arrive_first(uint32_t bar) {
    if (PAIR)
        asm volatile(
            "{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, 0;\n"
            " mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [r];\n}\n" ::"r"(bar)
            : "memory");
    else
        mbar_arrive(bar);
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint4 (&v)[4]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(v[0].x), "r"(v[0].y), "r"(v[0].z), "r"(v[0].w), "r"(v[1].x), "r"(v[1].y), "r"(v[1].z), "r"(v[1].w),
        "r"(v[2].x), "r"(v[2].y), "r"(v[2].z), "r"(v[2].w), "r"(v[3].x), "r"(v[3].y), "r"(v[3].z), "r"(v[3].w)
        : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                        uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
}
// This shared-memory offset in the pair's first CTA, as an address of the cluster.
__device__ __forceinline__ uint32_t of_first(uint32_t addr) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ uint32_t of_other(uint32_t addr, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank ^ 1));
    return r;
}
// Tile loads that report to a barrier of the pair's first CTA (`bar`: of_first).
template <bool PAIR>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
    if (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
            : "memory");
    else
        tma_load_2d(dst, map, c0, c1, bar);
}
template <bool PAIR>
__device__ __forceinline__ void expect_first(uint32_t bar, uint32_t bytes) {      // bar: of_first
    if (PAIR)
        asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                     : "memory");
    else
        mbar_expect_tx(bar, bytes);
}

// Whether all 128 threads that meet at this barrier say so.
__device__ __forceinline__ bool all_of_group(bool ok, int bar) {
    uint32_t r;
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.and.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(ok)), "r"(bar)
        : "memory");
    return r != 0;
}
// Two f32 numbers in one register pair: one instruction for both.
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(Two v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// z / (1 + exp(-z)) as max(z, 0) - a t / (1 + t), a = |z|, t = exp(-a) <= 1: nothing overflows, a negative
// z's value is the product alone and a positive one's at least half its first term.  An infinite a is
// taken as 3e38, so that -inf gives its limit 0; NaN stays NaN.  For 16-bit outputs t and the
// reciprocals come from the special unit, one reciprocal for the product of two or four denominators of [1, 2]
// (four: 12000 x 1024 -> 4096 38.9 us, two: 39.7).
template <typename T>
__device__ __forceinline__ void swish2(float &z0, float &z1) {
    const float a0 = fminf(fabsf(z0), 3e38f), a1 = fminf(fabsf(z1), 3e38f);      // NaN: 3e38, so that the other's value stands
    float m0, m1, q0, q1;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(m0) : "f"(z0));
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(m1) : "f"(z1));
    if (sizeof(T) == 4) {
        const float t0 = expf(-a0), t1 = expf(-a1);
        q0 = __fdiv_rn(t0, 1.0f + t0), q1 = __fdiv_rn(t1, 1.0f + t1);
    } else {
        const float t0 = ex2(a0 * -1.44269504f), t1 = ex2(a1 * -1.44269504f);
        const float d0 = 1.0f + t0, d1 = 1.0f + t1;
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d0 * d1));
        q0 = t0 * (r * d1), q1 = t1 * (r * d0);
    }
    z0 = __fmaf_rn(-a0, q0, m0);
    z1 = __fmaf_rn(-a1, q1, m1);
}
// Four elements for 16-bit outputs: one reciprocal, of the product of the denominators, in [1, 16].
__device__ __forceinline__ void swish4(float *z) {
    float n[4], m[4], t[4], d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        n[j] = fmaxf(-fabsf(z[j]), -3e38f);
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(m[j]) : "f"(z[j]));
    }
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        float p0, p1;
        split(mul2(two(n[j], n[j + 1]), two(1.44269504f, 1.44269504f)), p0, p1);
        t[j] = ex2(p0), t[j + 1] = ex2(p1);
        split(add2(two(t[j], t[j + 1]), two(1.0f, 1.0f)), d[j], d[j + 1]);
    }
    const float d01 = d[0] * d[1], d23 = d[2] * d[3];
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d01 * d23));
    const float r01 = r * d23, r23 = r * d01;
    split(fma2(two(n[0], n[1]), two(t[0] * (r01 * d[1]), t[1] * (r01 * d[0])), two(m[0], m[1])), z[0], z[1]);
    split(fma2(two(n[2], n[3]), two(t[2] * (r23 * d[3]), t[3] * (r23 * d[2])), two(m[2], m[3])), z[2], z[3]);
}

// Two outputs of a 16-bit type in a word, the first low.
template <typename T>
__device__ __forceinline__ uint32_t word_of(float a, float b) {
    uint32_t w;
    if (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}
// 16 lanes x 16 columns of sums: lane l receives of each 8 columns the two from 2 (l mod 4) on, in row l / 4
// (v[0], v[1]) and in row l / 4 + 8.
__device__ __forceinline__ void tmem_ld_rows(uint32_t addr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(addr)
                 : "memory");
}
// Columns of an output block: rows of 64 bytes, or what a warp has of a tile's columns.
template <typename T, int BN>
__host__ __device__ constexpr int block_columns() {
    return BN / 4 < 64 / static_cast<int>(sizeof(T)) ? BN / 4 : 64 / static_cast<int>(sizeof(T));
}
// An output from shared memory.
__device__ __forceinline__ void copy_out(float *y, uint32_t at) { *y = __uint_as_float(lds32(at)); }
template <typename T>
__device__ __forceinline__ void copy_out(T *y, uint32_t at) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
    *reinterpret_cast<uint16_t *>(y) = v;
}
// Block of 32 rows to the output, from shared memory in the swizzled layout.
__device__ __forceinline__ void store_block(const CUtensorMap *map, uint32_t src, int n, int m) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(n), "r"(m), "r"(src)
                 : "memory");
}
// Byte offset of a part's sum: rows of BN, groups of eight columns moved by the row so that a warp's stores fall on different banks.
template <int BN>
__device__ __forceinline__ uint32_t sum_at(int row, int col) {
    static_assert(BN >= 64, "groups of eight columns");
    return 4u * static_cast<uint32_t>(row * BN + (col ^ (row & 7) << 3));
}
// ODD: output rows that are not on 16 bytes or whose N columns do not end there: written element by element, others
// by TMA.  PARTS: CTAs of a cluster that share a tile's K, one tile a cluster; each then adds up 128 / PARTS rows.
template <typename T, int BN, bool PAIR, bool ODD, int PARTS = 1>
__global__ void __launch_bounds__(THREADS, 1)
    fp4_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w,
               const __grid_constant__ CUtensorMap tm_xb, const __grid_constant__ CUtensorMap tm_wb,
               const __grid_constant__ CUtensorMap tm_y, const Params prm) {
    using C = Tile<BN, PAIR>;
    static_assert(PARTS == 1 || (!PAIR && ODD), "forms");
    // 256 columns are 64 registers of an output thread: its warpgroups take over what the others can
    // spare, 4 x 96 + 2 x 48 = 6 x 80 (ptxas, which allows for the 80, spills 44 bytes a thread)
    constexpr bool DEAL = BN == 256;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    auto full = [&](int s) { return base + 8u * s; };
    auto empty = [&](int s) { return base + 8u * (C::ST + s); };
    auto scales = [&](int s) { return base + 8u * (2 * C::ST + s); };      // have landed, in each CTA
    auto ready = [&](int s) { return base + 8u * (3 * C::ST + s); };       // are in TMEM
    auto acc_full = [&](int s) { return base + 8u * (4 * C::ST + s); };
    auto acc_empty = [&](int s) { return base + 8u * (4 * C::ST + 2 + s); };
    const uint32_t drained = base + 8u * (4 * C::ST + 4), never = drained + 8u;
    volatile int *dead = reinterpret_cast<volatile int *>(smem + C::DEAD);
    const int rank = PAIR ? static_cast<int>(blockIdx.x & 1u) : 0;      // clusters are (2, 1, 1)
    const int part = PARTS > 1 ? static_cast<int>(blockIdx.x % PARTS) : 0;      // clusters are (PARTS, 1, 1)
    const long long worker = blockIdx.x / (C::CTAS * PARTS), workers = gridDim.x / (C::CTAS * PARTS);

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::ST; ++s) {
            mbar_init(full(s), 2 * C::CTAS);
            mbar_init(empty(s), 1);
            mbar_init(scales(s), 1);
            mbar_init(ready(s), 4 * C::CTAS);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full(s), 1);
            mbar_init(acc_empty(s), EPI_WARPS / 4 * C::CTAS);
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

    const int stages = (prm.steps + 3) / 4, share = (stages + PARTS - 1) / PARTS;
    const int from = part * share, to = PARTS > 1 ? min(stages, from + share) : stages;
    const long long limit = prm.timeout_cycles;

    if (DEAL && warp >= SCALE_WARP) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    volatile int *fetched = reinterpret_cast<volatile int *>(smem + C::FETCHED);
    if (warp == X_WARP || warp == W_WARP || warp == SCALES_WARP) {
        // a thread each for the rows, the channels and the scales: one for all four copies of a stage
        // takes 0.34 us a stage, whatever their size
        if (lane == 0) {
            int s = 0, ph = 0, issued = 0;
            bool ok = true;
            for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
                const int mt = static_cast<int>(tile / prm.tiles_n) * C::CTAS + rank;
                const int n0 = static_cast<int>(tile % prm.tiles_n) * BN;
                for (int it = from; it < to; ++it) {
                    ok = wait_or_dead(empty(s), ph ^ 1, dead, limit);
                    if (!ok) break;
                    const uint32_t st = base + C::STAGES_AT + s * C::STAGE;
                    if (warp == SCALES_WARP) {
                        mbar_expect_tx(scales(s), C::SA + C::SB);
                        tma_load_3d(st + C::A + C::B, &tm_xb, 0, 4 * it, mt, scales(s));
                        tma_load_3d(st + C::A + C::B + C::SA, &tm_wb, 0, 4 * it, n0 / 128, scales(s));
                    } else {
                        const uint32_t bar = PAIR ? of_first(full(s)) : full(s);
                        if (warp == X_WARP) {
                            expect_first<PAIR>(bar, C::A);
                            load_2d<PAIR>(st, &tm_x, it * BKB, mt * TILE_M, bar);
                        } else {
                            expect_first<PAIR>(bar, C::B);
                            load_2d<PAIR>(st + C::A, &tm_w, it * BKB, n0 + rank * C::BR, bar);
                        }
                    }
                    ++issued;
                    if (++s == C::ST) s = 0, ph ^= 1;
                }
            }
            fetched[warp == X_WARP ? 0 : (warp == W_WARP ? 1 : 2)] = issued;
        }
    } else if (warp == MMA_WARP) {
        if (rank == 0 && worker < prm.tiles) {
            // the whole warp runs the loop, so that the descriptors stay uniform; one lane issues.
            // e2m1 x e2m1, e4m3 scales
            constexpr uint32_t idesc = (1u << 7) | (1u << 10) | (static_cast<uint32_t>(BN / 8) << 17) |
                                       (static_cast<uint32_t>(TILE_M * C::CTAS / 16) << 24);
            int s = 0, ph = 0, a = 0, aph = 0;
            bool ok = true;
            for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
                ok = warp_wait_or_dead(acc_empty(a), aph ^ 1, dead, limit);
                if (!ok) break;
                const int n0 = static_cast<int>(tile % prm.tiles_n) * BN;
                for (int it = from; it < to; ++it) {
                    ok = warp_wait_or_dead(ready(s), ph, dead, limit) && warp_wait_or_dead(full(s), ph, dead, limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t st = base + C::STAGES_AT + s * C::STAGE;
                    const uint64_t da = smem_desc(st), db = smem_desc(st + C::A);
                    const uint32_t sa = tmem + C::SF + s * C::SF_COLS, sb = sa + 16 + (n0 % 128) / 32;
                    const int nk = prm.steps - 4 * it < 4 ? prm.steps - 4 * it : 4;
                    if (elect_one()) {
                        for (int k = 0; k < nk; ++k)
                            mma_fp4<PAIR>(tmem + a * BN, da + 2 * k, db + 2 * k, idesc, sa + 4 * k, sb + 4 * C::WT * k, it > from || k > 0);
                        mma_commit<PAIR>(empty(s));
                    }
                    __syncwarp();
                    if (++s == C::ST) s = 0, ph ^= 1;
                }
                if (!ok) break;
                if (elect_one()) mma_commit<PAIR>(acc_full(a));
                __syncwarp();
                if (++a == C::ACCS) a = 0, aph ^= 1;
            }
            if (!ok) {   // the MMAs in flight end before their TMEM is freed
                if (elect_one()) mma_commit<PAIR>(drained);
                __syncwarp();
                mbar_wait(drained, 0, ips::LAND_CYCLES);
            }
        }
    } else if (warp >= SCALE_WARP) {
        // Scales to TMEM, byte by byte as they are (a sign bit, which the contract excludes, would have to be cleared
        // here: 1 to 3 % of the large products' time): lane l of every quarter holds those of the rows l, l + 32, l + 64, l + 96, four columns
        // for each 64 elements.  A stage's slot there is free when its shared memory is: its scales
        // are fetched after the MMAs that read the ones before.
        const uint32_t at = tmem + C::SF + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        int s = 0, ph = 0;
        bool ok = true;
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers)
            for (int it = from; it < to; ++it) {
                ok = warp_wait_or_dead(scales(s), ph, dead, limit);
                if (!ok) break;
                const uint32_t src = base + C::STAGES_AT + s * C::STAGE + C::A + C::B + 16 * lane;
                uint4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = lds128(src + 512 * k);
                tmem_st16(at + s * C::SF_COLS, v);
#pragma unroll
                for (int h = 0; h < C::WT; ++h) {
                    // of x then w: columns 4 (WT k + j) for step k and tile j
                    uint4 u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int c = 4 * h + i, k = c / C::WT, j = c % C::WT;
                        u[i] = lds128(src + C::SA + 2048 * j + 512 * k);
                    }
                    tmem_st16(at + s * C::SF_COLS + 16 + 16 * h, u);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                // these reads come before the copy that refills the stage (release_stage has the same fence)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_first<PAIR>(ready(s));
                if (++s == C::ST) s = 0, ph ^= 1;
            }
    } else {
        if (DEAL) asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
        const int quarter = warp & 3, group = warp >> 2;
        constexpr int CW = BN / 4;            // columns of a warp
        const int col0 = group * CW;
        constexpr int BC = block_columns<T, BN>(), CHUNKS = BC * static_cast<int>(sizeof(T)) / 16;      // columns and 16-byte chunks of a block's row
        const uint32_t cst = base + C::CONSTS + group * (8 * CW), out = base + C::OUT_AT + warp * C::OUT;
        // where a block's row and chunk lie: rows of 64 or 32 bytes in the swizzled layout of that width
        auto place = [&](int row, int chunk) {
            return out + row * (CHUNKS * 16) + ((CHUNKS == 4 ? chunk ^ (row >> 1 & 3) : chunk ^ (row >> 2 & 1)) << 4);
        };
        int a = 0, aph = 0;
        bool ok = true;
        if (prm.stall) ok = warp_wait_or_dead(never, 0, dead, limit);
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
            const long long first = (tile / prm.tiles_n * C::CTAS + rank) * TILE_M + quarter * 32;
            const int n0 = static_cast<int>(tile % prm.tiles_n) * BN + col0;
            // each thread has the constants of one of the columns
            const int cc = quarter * 32 + lane, cn = n0 + cc;
            const bool in = cc < CW && cn < prm.N;
            const float csw = in ? prm.sw[cn] : 0.0f, cb = in && prm.bias ? prm.bias[cn] : 0.0f;
            // a lane has the rows lane / 4 + 8 i, in each 8 columns two from 2 (lane mod 4) on: so the
            // constants of a column are read for four rows at once, and blocks leave by stmatrix
            float sx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long long m = first + lane / 4 + 8 * i;
                sx[i] = m < prm.M ? prm.sx[m] : 0.0f;
            }
            // the four warps of these columns go on together, or none does
            ok = all_of_group(warp_wait_or_dead(acc_full(a), aph, dead, limit), 1 + group);
            if (!ok) break;
            if (cc < CW) {
                sts32(cst + 4 * cc, __float_as_uint(csw));
                sts32(cst + 4 * (CW + cc), __float_as_uint(cb));
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t r[CW / 16][2][8];      // [..][rows 0-15, 16-31][8 columns, 8 columns: rows + 0, + 8, of two columns]
#pragma unroll
            for (int c = 0; c < CW / 16; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    tmem_ld_rows(tmem + a * BN + col0 + 16 * c + (static_cast<uint32_t>(quarter * 32 + 16 * h) << 16), r[c][h]);
            tmem_wait_ld();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");      // the sums are in registers, the constants there
            if (quarter == 0 && lane == 0) arrive_first<PAIR>(acc_empty(a));
            if (++a == C::ACCS) a = 0, aph ^= 1;
            if constexpr (PARTS > 1) {
                // where blocks on their way out would be, none of which this form has
                static_assert(4 * TILE_M * BN <= EPI_WARPS * C::OUT, "room for a part's sums");
#pragma unroll
                for (int c = 0; c < CW / 8; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t *v = &r[c / 2][i / 2][4 * (c & 1) + 2 * (i & 1)];
                        sts64(base + C::OUT_AT + sum_at<BN>(quarter * 32 + lane / 4 + 8 * i, col0 + 8 * c + 2 * (lane & 3)),
                              static_cast<int>(v[0]), static_cast<int>(v[1]));
                    }
            } else {
#pragma unroll
            for (int c = 0; c < CW; c += BC) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the last block has been read
                __syncwarp();
#pragma unroll
                for (int g = 0; g < BC / 8; ++g) {
                    const int2 w2 = lds64(cst + 4 * (c + 8 * g + 2 * (lane & 3))), b2 = lds64(cst + 4 * (CW + c + 8 * g + 2 * (lane & 3)));
                    const Two w = two(__int_as_float(w2.x), __int_as_float(w2.y)), b = two(__int_as_float(b2.x), __int_as_float(b2.y));
                    float z[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t *v = &r[(c + 8 * g) / 16][i / 2][4 * (g & 1) + 2 * (i & 1)];
                        split(fma2(two(__uint_as_float(v[0]), __uint_as_float(v[1])), mul2(w, two(sx[i], sx[i])), b), z[2 * i], z[2 * i + 1]);
                    }
                    if (prm.act) {
                        if constexpr (sizeof(T) == 2) {
                            swish4(z), swish4(z + 4);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; i += 2) swish2<T>(z[i], z[i + 1]);
                        }
                    }
                    uint32_t q[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (sizeof(T) == 4)
                            sts64(place(lane / 4 + 8 * i, 2 * g + (lane >> 1 & 1)) + 8 * (lane & 1), __float_as_int(z[2 * i]), __float_as_int(z[2 * i + 1]));
                        else
                            q[i] = word_of<T>(z[2 * i], z[2 * i + 1]);
                    }
                    if constexpr (sizeof(T) == 2)
                        asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(place(lane, g)),
                                     "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3])
                                     : "memory");
                }
                if constexpr (ODD) {
                    __syncwarp();
                    for (int e = lane; e < 32 * BC; e += 32) {
                        const int row = e / BC, col = e % BC;
                        const uint32_t at = place(row, col * static_cast<int>(sizeof(T)) / 16) + col * static_cast<int>(sizeof(T)) % 16;
                        if (first + row < prm.M && n0 + c + col < prm.N)
                            copy_out(static_cast<T *>(prm.y) + (first + row) * prm.ldy + n0 + c + col, at);
                    }
                    __syncwarp();
                } else {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (first < prm.M && n0 + c < prm.N) store_block(&tm_y, out, n0 + c, static_cast<int>(first));
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            }
            }
        }
        if (!ODD && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");      // no block is still on its way
    }
    if constexpr (PARTS > 1) {
        __syncthreads();
        cluster_sync();
        constexpr int ROWS = TILE_M / PARTS;
        for (int e = threadIdx.x; e < ROWS * BN / 2; e += THREADS) {
            const int row = part * ROWS + e / (BN / 2), col = e % (BN / 2) * 2;
            const long long m = worker / prm.tiles_n * TILE_M + row;
            const int n = static_cast<int>(worker % prm.tiles_n) * BN + col;
            if (m >= prm.M || n >= prm.N) continue;
            const uint32_t at = base + C::OUT_AT + sum_at<BN>(row, col);
            float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                uint32_t there;
                float u0, u1;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(p));
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(u0), "=f"(u1) : "r"(there) : "memory");
                v0 += u0, v1 += u1;
            }
            const bool both = n + 1 < prm.N;
            const float sx = prm.sx[m];
            float z0 = __fmaf_rn(v0, __fmul_rn(prm.sw[n], sx), prm.bias ? prm.bias[n] : 0.0f);
            float z1 = both ? __fmaf_rn(v1, __fmul_rn(prm.sw[n + 1], sx), prm.bias ? prm.bias[n + 1] : 0.0f) : 0.0f;
            if (prm.act) swish2<T>(z0, z1);
            T *y = static_cast<T *>(prm.y) + m * prm.ldy + n;
            y[0] = from_f32<T>(z0);
            if (both) y[1] = from_f32<T>(z1);
        }
        __syncthreads();
        cluster_sync();      // no CTA ends while another one reads its sums
    }
    // After a wait that ran out the copies in flight land before a CTA ends.  The scales' report to their own CTA's
    // barriers; a pair's others to the first CTA's, where a stage that not all of its fetching
    // threads came to lacks their arrivals.
    volatile int *other = reinterpret_cast<volatile int *>(smem + C::OTHER);
    __syncthreads();
    if (PAIR) {
        if (threadIdx.x == 0) {
            const uint32_t at = of_other(base + C::OTHER, rank);
            asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at), "r"(*dead) : "memory");
            asm volatile("st.shared::cluster.v2.s32 [%0], {%1, %2};" ::"r"(at + 8), "r"(fetched[0]), "r"(fetched[1]) : "memory");
        }
        cluster_sync();
    }
    if (threadIdx.x == 0 && (*dead || (PAIR && other[0])))
        for (int n = fetched[2], i = n > C::ST ? n - C::ST : 0; i < n; ++i)
            mbar_wait(scales(i % C::ST), static_cast<uint32_t>((i / C::ST) & 1), ips::LAND_CYCLES);
    if (threadIdx.x == 0 && rank == 0 && (*dead || (PAIR && other[0]))) {
        const int n[4] = {fetched[0], fetched[1], PAIR ? other[2] : fetched[0], PAIR ? other[3] : fetched[1]};
        const int last = max(max(n[0], n[1]), max(n[2], n[3]));
        for (int i = last > C::ST ? last - C::ST : 0; i < last; ++i) {
            for (int k = 0; k < 2 * C::CTAS; ++k)
                if (i >= n[k]) mbar_arrive(full(i % C::ST));
            mbar_wait(full(i % C::ST), static_cast<uint32_t>((i / C::ST) & 1), ips::LAND_CYCLES);
        }
    }
    if (PAIR && (*dead || other[0])) cluster_sync();      // the same in both CTAs
    if (!PAIR) __syncthreads();
    if (warp == MMA_WARP) tmem_free<PAIR>(tmem, C::COLS);
    if (threadIdx.x == 0 && *dead) atomicOr(prm.err, ips::ERR_TIMEOUT);
}

// ---- few rows ------------------------------------------------------------
//
// Up to eight rows, where that is sooner than tiles (few_time in ip_fp4.cu): ordinary lanes read the weights once, a warp has the four channels n, n + 32, n + 64, n + 96 of
// 128, whose scales lie side by side, a lane 32 elements of them (16 bytes) at a time.  Products of codes are multiples
// of 1/4 up to 36, so f16 holds the sums of eight exactly; a block's two sums and its scales' product go to f32.
// PARTS warps of a CTA share a row's elements and add up in a fixed order.  What bounds it: latency (launch, loads,
// join) with one or two rows, their products with more: 1 x 1024 -> 4096 2.7 us (2.4 MB), by tiles 4.3.

struct FewParams {
    const uint8_t *x, *xb, *w, *wb;
    const float *sx, *sw, *bias;
    void *y;
    long long ldx, ldw, ldy;
    int M, N, act, bytes, steps;
};

// The 16 bytes of a row's codes from c on, zeros behind its last.
__device__ __forceinline__ uint4 codes16(const uint8_t *row, int c, int bytes) {
    if (c + 16 <= bytes) return *reinterpret_cast<const uint4 *>(row + c);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll 1
    for (int i = 0; c + i < bytes; ++i) {
        const uint32_t v = static_cast<uint32_t>(row[c + i]) << (8 * (i & 3));
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] |= i >> 2 == k ? v : 0u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight codes as f16 pairs.
__device__ __forceinline__ void halves8(uint32_t w, __half2 *v) {
    uint32_t h[4];
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const __half2 *>(&h[i]);
}
__device__ __forceinline__ void halves32(uint4 c, __half2 (&v)[16]) {
    halves8(c.x, v), halves8(c.y, v + 4), halves8(c.z, v + 8), halves8(c.w, v + 12);
}
// The two scales of one half of a word.
__device__ __forceinline__ float2 scales2(uint32_t word, int half) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(half ? word >> 16 : word)));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

template <typename T, int MR, int PARTS>
__global__ void __launch_bounds__(128) few_rows_kernel(const FewParams prm) {
    constexpr int SETS = 4 / PARTS;            // of four channels, a CTA
    __shared__ float sums[PARTS][SETS][4 * MR];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % PARTS, set = warp / PARTS;
    const int at = static_cast<int>(blockIdx.x) * SETS + set, group = at >> 5, r = at & 31, n0 = group * 128 + r;
    const int chunks = (prm.bytes + 15) / 16;
    float acc[4][MR];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int m = 0; m < MR; ++m) acc[j][m] = 0.0f;
    if (n0 < prm.N) {
        for (int c = part * 32 + lane; c < chunks; c += 32 * PARTS) {
            uint4 wc[4], xc[MR];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                wc[j] = n0 + 32 * j < prm.N ? codes16(prm.w + (n0 + 32 * j) * prm.ldw, 16 * c, prm.bytes) : make_uint4(0, 0, 0, 0);
            const uint4 ws = *reinterpret_cast<const uint4 *>(prm.wb + (static_cast<long long>(group) * prm.steps + (c >> 1)) * 512 + 16 * r);
            uint32_t xs[MR];
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                const bool in = m < prm.M;
                xc[m] = in ? codes16(prm.x + m * prm.ldx, 16 * c, prm.bytes) : make_uint4(0, 0, 0, 0);
                xs[m] = in ? *reinterpret_cast<const uint32_t *>(prm.xb + static_cast<long long>(c >> 1) * 512 + 16 * m) : 0;
            }
            const uint32_t wsj[4] = {ws.x, ws.y, ws.z, ws.w};
            __half2 w[4][16];
            float2 s[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                halves32(wc[j], w[j]);
                s[j] = scales2(wsj[j], c & 1);
            }
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                __half2 x[16];
                halves32(xc[m], x);
                const float2 sx = scales2(xs[m], c & 1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    __half2 a = __hmul2(w[j][0], x[0]), b = __hmul2(w[j][8], x[8]);
#pragma unroll
                    for (int i = 1; i < 8; ++i) {
                        a = __hfma2(w[j][i], x[i], a);
                        b = __hfma2(w[j][8 + i], x[8 + i], b);
                    }
                    acc[j][m] = __fmaf_rn(__low2float(a) + __high2float(a), s[j].x * sx.x, acc[j][m]);
                    acc[j][m] = __fmaf_rn(__low2float(b) + __high2float(b), s[j].y * sx.y, acc[j][m]);
                }
            }
        }
    }
    // the lanes' sums: at each step a lane hands half of its values over and keeps the others, until value `lane` is left
    constexpr int V = 4 * MR;
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = acc[i & 3][i >> 2];
#pragma unroll
    for (int h = V / 2; h; h >>= 1)
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const bool up = lane & h;
            const float give = up ? a[i] : a[i + h];
            a[i] = (up ? a[i + h] : a[i]) + __shfl_xor_sync(0xffffffffu, give, h);
        }
#pragma unroll
    for (int o = V; o < 32; o <<= 1) a[0] += __shfl_xor_sync(0xffffffffu, a[0], o);
    if (lane < V) sums[part][set][lane] = a[0];
    if (PARTS > 1) __syncthreads();
    else __syncwarp();
    const int j = lane & 3, m = lane >> 2, n = n0 + 32 * j;
    if (part != 0 || lane >= 4 * MR || m >= prm.M || n >= prm.N) return;
    float v = sums[0][set][lane];
#pragma unroll
    for (int i = 1; i < PARTS; ++i) v += sums[i][set][lane];
    float z = __fmaf_rn(v, __fmul_rn(prm.sw[n], prm.sx[m]), prm.bias ? prm.bias[n] : 0.0f), other = 0.0f;
    if (prm.act) swish2<T>(z, other);
    static_cast<T *>(prm.y)[m * prm.ldy + n] = from_f32<T>(z);
}

}  // namespace ip4
