// Device code of the product of 4-bit rows for sm_103a (e2m1 codes, e4m3 scales of 16, an f32 scale a
// row) on the block-scaled tensor cores.
#pragma once

#include <stdint.h>

#include "ip_scaled_kernels.cuh"

namespace ip4 {

using namespace ipk;
using namespace ipr;
using ips::elect_one, ips::cluster_sync, ips::mma_commit, ips::tmem_alloc, ips::tmem_free, ips::tmem_ld16,
    ips::tmem_wait_ld, ips::wait_or_dead, ips::warp_wait_or_dead, ips::arrive_first, ips::smem_desc;

// y[m][n] = act(sx[m] sw[n] S + bias[n]), S = sum over blocks of s_x s_w sum of 16 code products, by
// tcgen05.mma kind::mxf4nvf4 with a scale for each 16 elements: products and scales are exact there, sums
// in f32.
//
// Roles of a persistent CTA (one an SM): warp 8 fetches stages of 256 elements of K by TMA (128 rows of
// x and BN channels of w, 128 bytes each in the 128-byte swizzled layout, and their scales as they
// lie in memory, 512 bytes for 128 rows x 64 elements), one thread of warp 9 copies the scales to TMEM
// (tcgen05.cp) and issues the MMAs of 64 elements each, warps 0-7 take the sums to registers, release
// the accumulator and write the output while the next tile is summed.
// PAIR: two CTAs share a tile of 256 rows x BN channels (cta_group::2), each fetching its 128 rows and half of
// the channels; the scales of all channels go to both.  The second CTA's warp 9 tells the first one's
// of stages that have landed.

constexpr int TILE_M = 128;
constexpr int BKB = 128;                 // bytes of a row in a stage
constexpr int BK = 256;                  // elements
constexpr int THREADS = 320;
constexpr int EPI_WARPS = 8, TMA_WARP = 8, MMA_WARP = 9;

struct Params {
    const float *sx, *sw, *bias;
    const uint8_t *xb, *wb;              // e4m3 scales
    void *y;
    long long M, ldy;
    int N, act;
    int steps;                           // of 64 elements
    int xtiles, wtiles;                  // of 128 rows in xb and wb
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
    static constexpr int CONSTS = 512;                // per output warp: sw and bias of its columns
    static constexpr int TURN = CONSTS + EPI_WARPS * 2 * 4 * (BN / 2);
    static constexpr int STAGES_AT = (TURN + EPI_WARPS * ips::TURN_BYTES + 1023) & ~1023;
    static constexpr int SMEM = STAGES_AT + ST * STAGE + 1024;
    static_assert(8 * (3 * ST + 6) <= 256, "barriers");
    static_assert(SMEM <= 232448, "shared memory");
    static_assert(SF + ST * SF_COLS <= COLS, "TMEM columns");
    static_assert(STAGE % 1024 == 0 && B % 1024 == 0, "alignment");
};

// Scales of 128 rows x 64 elements to four TMEM columns, in all four quarters of the lanes.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem) {
    // rows of 16 bytes without swizzle, groups of eight rows 128 bytes apart
    const uint64_t desc = static_cast<uint64_t>((smem & 0x3ffff) >> 4) | (8ull << 16) | (8ull << 32) | (1ull << 46);
    if (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, int bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// ODD: output rows that are not aligned to 8 bytes, or an N that 16 does not divide.
template <typename T, int BN, bool PAIR, bool ODD>
__global__ void __launch_bounds__(THREADS, 1)
    fp4_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const Params prm) {
    using C = Tile<BN, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    auto full = [&](int s) { return base + 8u * s; };
    auto peer = [&](int s) { return base + 8u * (C::ST + s); };      // the second CTA's stages, told to the first
    auto empty = [&](int s) { return base + 8u * (2 * C::ST + s); };
    auto acc_full = [&](int s) { return base + 8u * (3 * C::ST + s); };
    auto acc_empty = [&](int s) { return base + 8u * (3 * C::ST + 2 + s); };
    const uint32_t drained = base + 8u * (3 * C::ST + 4), never = drained + 8u;
    volatile int *dead = reinterpret_cast<volatile int *>(smem + C::DEAD);
    const int rank = PAIR ? static_cast<int>(blockIdx.x & 1u) : 0;      // clusters are (2, 1, 1)
    const long long worker = blockIdx.x / C::CTAS, workers = gridDim.x / C::CTAS;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::ST; ++s) {
            mbar_init(full(s), 1);
            mbar_init(peer(s), 1);
            mbar_init(empty(s), 1);
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

    const int stages = (prm.steps + 3) / 4;
    const long long limit = prm.timeout_cycles;

    if (warp == TMA_WARP) {
        if (lane == 0) {
            int s = 0, ph = 0;
            long long issued = 0;
            bool ok = true;
            for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
                const int mt = static_cast<int>(tile / prm.tiles_n) * C::CTAS + rank;
                const int n0 = static_cast<int>(tile % prm.tiles_n) * BN;
                // scales of tiles behind the last (rows and channels that are not written): the last's
                const uint8_t *xb = prm.xb + static_cast<long long>(mt < prm.xtiles ? mt : prm.xtiles - 1) * prm.steps * 512;
                for (int it = 0; it < stages; ++it) {
                    ok = wait_or_dead<false>(empty(s), ph ^ 1, dead, limit);
                    if (!ok) break;
                    const uint32_t st = base + C::STAGES_AT + s * C::STAGE;
                    const int left = prm.steps - 4 * it, sc = (left < 4 ? left : 4) * 512;
                    mbar_expect_tx(full(s), C::A + C::B + (1 + C::WT) * sc);
                    tma_load_2d(st, &tm_x, it * BKB, mt * TILE_M, full(s));
                    tma_load_2d(st + C::A, &tm_w, it * BKB, n0 + rank * C::BR, full(s));
                    bulk_load(st + C::A + C::B, xb + it * 2048, sc, full(s));
#pragma unroll
                    for (int j = 0; j < C::WT; ++j) {
                        const int wt = n0 / 128 + j;
                        bulk_load(st + C::A + C::B + C::SA + 2048 * j,
                                  prm.wb + static_cast<long long>(wt < prm.wtiles ? wt : prm.wtiles - 1) * prm.steps * 512 + it * 2048,
                                  sc, full(s));
                    }
                    ++issued;
                    if (++s == C::ST) s = 0, ph ^= 1;
                }
            }
            // after a wait that ran out: the copies in flight land before the CTA ends
            if (!ok)
                for (long long i = issued > C::ST ? issued - C::ST : 0; i < issued; ++i)
                    mbar_wait(full(static_cast<int>(i % C::ST)), static_cast<uint32_t>((i / C::ST) & 1), ips::LAND_CYCLES);
        }
    } else if (warp == MMA_WARP) {
        // the whole warp runs the loop, so that the descriptors stay uniform; one lane issues
        // e2m1 x e2m1, e4m3 scales
        constexpr uint32_t idesc = (1u << 7) | (1u << 10) | (static_cast<uint32_t>(BN / 8) << 17) |
                                   (static_cast<uint32_t>(TILE_M * C::CTAS / 16) << 24);
        int s = 0, ph = 0, a = 0, aph = 0;
        bool ok = true;
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
            if (rank == 0) ok = warp_wait_or_dead<PAIR>(acc_empty(a), aph ^ 1, dead, limit);
            if (!ok) break;
            const int n0 = static_cast<int>(tile % prm.tiles_n) * BN;
            for (int it = 0; it < stages; ++it) {
                ok = warp_wait_or_dead<false>(full(s), ph, dead, limit);
                if (!ok) break;
                if (PAIR && rank == 1) {
                    if (lane == 0) arrive_first<PAIR>(peer(s));
                } else {
                    if (PAIR) ok = warp_wait_or_dead<PAIR>(peer(s), ph, dead, limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t st = base + C::STAGES_AT + s * C::STAGE;
                    const uint64_t da = smem_desc(st), db = smem_desc(st + C::A);
                    const uint32_t sa = tmem + C::SF + s * C::SF_COLS, sb = sa + 16;
                    const int nk = prm.steps - 4 * it < 4 ? prm.steps - 4 * it : 4;
                    if (elect_one()) {
                        for (int k = 0; k < nk; ++k) {
                            copy_scales<PAIR>(sa + 4 * k, st + C::A + C::B + 512 * k);
#pragma unroll
                            for (int j = 0; j < C::WT; ++j)
                                copy_scales<PAIR>(sb + 4 * (k * C::WT + j), st + C::A + C::B + C::SA + 2048 * j + 512 * k);
                        }
                        for (int k = 0; k < nk; ++k)
                            mma_fp4<PAIR>(tmem + a * BN, da + 2 * k, db + 2 * k, idesc, sa + 4 * k,
                                          sb + 4 * C::WT * k + (n0 % 128) / 32, it > 0 || k > 0);
                        mma_commit<PAIR>(empty(s));
                    }
                    __syncwarp();
                }
                if (++s == C::ST) s = 0, ph ^= 1;
            }
            if (!ok) break;
            if (rank == 0) {
                if (elect_one()) mma_commit<PAIR>(acc_full(a));
                __syncwarp();
            }
            if (++a == C::ACCS) a = 0, aph ^= 1;
        }
        if (!ok && rank == 0) {   // the MMAs in flight end before their TMEM is freed
            if (elect_one()) mma_commit<PAIR>(drained);
            __syncwarp();
            mbar_wait(drained, 0, ips::LAND_CYCLES);
        }
    } else {
        const int quarter = warp & 3, half = warp >> 2;
        constexpr int CW = BN / 2;            // columns of a warp
        const int col0 = half * CW;
        const unsigned low = static_cast<unsigned>(reinterpret_cast<uintptr_t>(prm.y) | (prm.ldy * sizeof(T))) & 31u;
        const bool wide = low == 0, even = (low & 7u) == 0;
        const uint32_t cst = base + C::CONSTS + warp * (8 * CW);
        int a = 0, aph = 0;
        bool ok = true;
        if (prm.stall) ok = warp_wait_or_dead<false>(never, 0, dead, limit);
        for (long long tile = worker; ok && tile < prm.tiles; tile += workers) {
            const long long m = (tile / prm.tiles_n * C::CTAS + rank) * TILE_M + quarter * 32 + lane;
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
            ok = warp_wait_or_dead<PAIR>(acc_full(a), aph, dead, limit);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t r[CW / 16][16];
#pragma unroll
            for (int c = 0; c < CW / 16; ++c)
                tmem_ld16(tmem + a * BN + col0 + 16 * c + (static_cast<uint32_t>(quarter * 32) << 16), r[c]);
            tmem_wait_ld();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive_first<PAIR>(acc_empty(a));
            if (++a == C::ACCS) a = 0, aph ^= 1;
#pragma unroll
            for (int ch = 0; ch < CW / 16; ++ch) {
                const int c = 16 * ch;
                float z[16];
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint4 w4 = lds128(cst + 4 * (c + i));
                    const uint4 b4 = lds128(cst + 4 * (CW + c + i));
                    z[i] = __fmaf_rn(__uint_as_float(r[ch][i]), sx * __uint_as_float(w4.x), __uint_as_float(b4.x));
                    z[i + 1] = __fmaf_rn(__uint_as_float(r[ch][i + 1]), sx * __uint_as_float(w4.y), __uint_as_float(b4.y));
                    z[i + 2] = __fmaf_rn(__uint_as_float(r[ch][i + 2]), sx * __uint_as_float(w4.z), __uint_as_float(b4.z));
                    z[i + 3] = __fmaf_rn(__uint_as_float(r[ch][i + 3]), sx * __uint_as_float(w4.w), __uint_as_float(b4.w));
                }
                if (prm.act)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = ips::swish<T>(z[i]);
                if (ODD && (!even || n0 + c + 16 > prm.N)) {
                    const long long first = m - lane, left = prm.M - first;
                    if (n0 + c < prm.N)
                        ips::store_odd<T>(static_cast<T *>(prm.y) + first * prm.ldy + n0 + c, prm.ldy,
                                          left < 32 ? static_cast<int>(left) : 32, prm.N - n0 - c,
                                          base + C::TURN + warp * ips::TURN_BYTES, z);
                } else if (m < prm.M && n0 + c < prm.N) {
                    ips::store16<T>(row, n0 + c, wide, z);
                }
            }
        }
    }
    __syncwarp();
    if (PAIR) cluster_sync();     // neither CTA ends while the other may still arrive on its barriers
    else __syncthreads();
    if (warp == MMA_WARP) tmem_free<PAIR>(tmem, C::COLS);
    if (threadIdx.x == 0 && *dead) atomicOr(prm.err, ips::ERR_TIMEOUT);
}

}  // namespace ip4
