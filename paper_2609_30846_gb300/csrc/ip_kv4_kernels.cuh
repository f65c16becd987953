// Device code of the 4-bit key/value cache for sm_103a: rows quantised into pages,
// read back, and the attention that reads the pages.
//
// A row of 128 channels of K or V is four groups of 32 with one bf16 scale each and
// codes c in -7 .. 7, stored as the nibble c + 8.  bf16 has the range of f32, and
// since the codes are taken against the rounded scale, its eight bits only move the
// step by at most 0.4 %.
//
// A page of one head is one block of 144 P bytes for its P tokens: P x 64 bytes of K
// codes, P x 4 K scales, P x 64 bytes of V codes, P x 4 V scales.  Within the 64 bytes
// of a row (low nibble first) channel d = 32 g + r sits, for K, in byte 16 (r / 8) + 4 g +
// (r mod 8) / 2, so that one 16-byte load gives a lane of the score product its eight
// channels of all four groups; for V, in byte 8 (r / 4) + 2 g + (r mod 4) / 2, so
// that one 8-byte load gives a lane of the output product its four channels of each.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ip_ptx.cuh"
#include "ip_real.cuh"

namespace ipv {

using namespace ipk;
using namespace ipr;

constexpr int DH = 128;
constexpr int ROW_BYTES = 144;      // of a token and head
constexpr int ERR_PARAM = 16;       // a length, position or page out of its domain

__host__ __device__ constexpr int k_scales(int page) { return 64 * page; }
__host__ __device__ constexpr int v_codes(int page) { return 72 * page; }
__host__ __device__ constexpr int v_scales(int page) { return 136 * page; }

struct Pages {
    uint8_t *cache;
    const int32_t *table;
    int max_pages, n_pages, shift, heads;    // page size 1 << shift
};

// ---- rows into pages and back -------------------------------------------

struct RowParams {
    const void *k, *v;                       // append: [B][T][H][128] by strides
    void *ko, *vo;                           // read: [B][T][H][128], contiguous
    long long ks[3], vs[3];                  // strides of batch, token, head (elements)
    const int32_t *start, *count;
    int B, T, H;
    Pages pages;
    int *err;
};

// A row (token and head) is a warp's: half of it for K, half for V, eight channels to a lane, so
// that a group of 32 is four lanes'.  Bound by the instructions of the conversion and the latency
// of the page table, so a warp takes two rows where there are many: 6000 tokens of 8 heads,
// 16 bits, 31 MB: append 13.5 us, read back 11 us (one row a warp: 15.1 and 12.2).
constexpr int ROW_THREADS = 256;

// The bf16 value nearest to amax / 7, ties to even (its bits).  The approximate quotient gives the
// value below, or a neighbour of it where it lies next to one; the middle of the next interval
// decides: seven times that (twelve bits) is exact.
__device__ __forceinline__ uint32_t scale4(float amax) {
    const uint32_t lo = __float_as_uint(amax * (1.0f / 7.0f)) >> 16;
    const float t = 7.0f * __uint_as_float(lo << 16 | 0x8000u);
    return lo + (amax > t || (amax == t && (lo & 1u)) ? 1u : 0u);
}

// Eight channels of a group, which the lanes l ^ 1, l ^ 2 and l ^ 3 hold the rest of: their
// nibbles, the integer n nearest to x / s, ties to even, within -7 .. 7, plus 8, and the group's
// scale s (bf16 bits).
//   16-bit x: the quotient by an approximate reciprocal, once corrected by its residue (the
//     Newton step of Markstein's division): exact at a half integer, where the residue of the
//     first quotient is exact too, and within 2^-20 elsewhere, where a half integer is 2^-13
//     away at least.
//   f32 x: n by the reciprocal, right but next to a half integer.  x - n s is exact (n s has
//     twelve bits, and the difference is about half of s at most), so comparing it with s / 2
//     shows what is left to do.
template <typename T>
__device__ __forceinline__ uint32_t quant8(const Raw8<T> &raw, uint32_t &scale) {
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr float ROUND = 12582912.0f;      // 1.5 2^23, bits 0x4b400000
    uint32_t top = 0;
    raw.largest(top);
    top = Raw8<T>::value(top);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (top >= 0x7f800000u) {      // a NaN or an infinity: the group reads back as NaN
        scale = 0x7fc0u;
        return 0x88888888u;
    }
    scale = scale4(__uint_as_float(top));
    if (scale == 0) return 0x88888888u;
    // a scale near the ends of the range and its row brought inside by 2^+-100; exactly but for
    // elements that are 0 either way
    const bool tiny = scale < (27u << 7), far = tiny || scale > (250u << 7);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = raw.at(i);
    if (far)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= tiny ? 0x1p100f : 0x1p-100f;
    const float s = __uint_as_float(scale << 16) * (far ? (tiny ? 0x1p100f : 0x1p-100f) : 1.0f), half = 0.5f * s;
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    uint32_t k[8];      // the bits of ROUND + n
    float e[8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (WIDE) {
            const float r = __fmaf_rn(x[i], inv, ROUND);
            k[i] = __float_as_uint(r);
            e[i] = __fmaf_rn(__fsub_rn(ROUND, r), s, x[i]);
            most = fmaxf(most, fabsf(e[i]));
        } else {
            const float y = x[i] * inv;
            k[i] = __float_as_uint(__fadd_rn(__fmaf_rn(__fmaf_rn(-y, s, x[i]), inv, y), ROUND));
        }
    }
    if (WIDE && most >= half) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (fabsf(e[i]) > half || (fabsf(e[i]) == half && (k[i] & 1u))) k[i] += e[i] > 0.0f ? 1u : ~0u;
    }
    if (scale < 0x80u)      // subnormal: it may be far below amax / 7
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = min(max(k[i], 0x4b400000u - 7u), 0x4b400000u + 7u);
    uint32_t w = 0;      // sum of (n + 8) 16^i, modulo 2^32
#pragma unroll
    for (int i = 7; i >= 0; --i) w = 16u * w + k[i];
    return w + (0x88888888u - 0x11111111u * 0x4b400000u);
}

// A warp's rows r, r + 1, ... of sequence b (grid: rows of a sequence, sequences).
struct Rows {
    int b, t, h, left;        // the next row, the rows from it to the sequence's last
    int n;                    // tokens that are no padding
    long long start;

    template <int R>
    static __device__ __forceinline__ Rows of(const RowParams &p) {
        Rows w;
        const unsigned r = (blockIdx.x * (ROW_THREADS / 32) + (threadIdx.x >> 5)) * R;
        w.b = static_cast<int>(blockIdx.y);
        w.t = static_cast<int>(r / static_cast<unsigned>(p.H));
        w.h = static_cast<int>(r - static_cast<unsigned>(w.t) * p.H);
        w.left = static_cast<int>(static_cast<unsigned>(p.T) * p.H - r);
        w.n = p.count ? p.count[w.b] : p.T;
        w.start = p.start[w.b];
        return w;
    }
    __device__ __forceinline__ void next(const RowParams &p) {
        --left;
        if (++h == p.H) h = 0, ++t;
    }
    // Page block of the row's position, nullptr if the token is padding or (status word) has no place.
    __device__ __forceinline__ uint8_t *block(const RowParams &p, int &off) const {
        if (t >= n) return nullptr;
        const long long pos = start + t;
        const int page = static_cast<int>(pos >> p.pages.shift);
        if (pos >= 0 && pos < static_cast<long long>(p.pages.max_pages) << p.pages.shift) {
            const int pid = p.pages.table[static_cast<long long>(b) * p.pages.max_pages + page];
            off = static_cast<int>(pos) & ((1 << p.pages.shift) - 1);
            if (pid >= 0 && pid < p.pages.n_pages)
                return p.pages.cache + ((static_cast<long long>(pid) * p.pages.heads + h) * ROW_BYTES << p.pages.shift);
        }
        atomicOr(p.err, ERR_PARAM);
        return nullptr;
    }
};

template <typename T, int R>
__global__ void __launch_bounds__(ROW_THREADS) kv4_append_kernel(const RowParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    const int kv = (threadIdx.x >> 4) & 1, l = threadIdx.x & 15, g = l >> 2, j = l & 3;
    const int page = 1 << prm.pages.shift;
    const long long s0 = kv ? prm.vs[0] : prm.ks[0], s1 = kv ? prm.vs[1] : prm.ks[1], s2 = kv ? prm.vs[2] : prm.ks[2];
    Rows row = Rows::of<R>(prm);
    const T *base = static_cast<const T *>(kv ? prm.v : prm.k) + row.b * s0 + 8 * l;
    Raw8<T> x[R];
    uint8_t *blk[R];
    int off[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        blk[i] = nullptr;
        if (row.left <= 0) continue;
        const T *src = base + row.t * s1 + row.h * s2;
        if ((reinterpret_cast<uintptr_t>(src) & 15) == 0) x[i].template load<true>(src, 8);      // beside the reads of the table
        else x[i].template load<false>(src, 8);
        blk[i] = row.block(prm, off[i]);
        row.next(prm);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (!blk[i]) continue;
        uint32_t scale;
        const uint32_t w = quant8(x[i], scale);
        uint8_t *codes = blk[i] + (kv ? v_codes(page) : 0) + off[i] * 64 + 16 * j;
        if (kv) {
            *reinterpret_cast<uint16_t *>(codes + 2 * g) = static_cast<uint16_t>(w);
            *reinterpret_cast<uint16_t *>(codes + 8 + 2 * g) = static_cast<uint16_t>(w >> 16);
        } else {
            *reinterpret_cast<uint32_t *>(codes + 4 * g) = w;
        }
        if (j == 0)
            reinterpret_cast<uint16_t *>(blk[i] + (kv ? v_scales(page) : k_scales(page)))[off[i] * 4 + g] =
                static_cast<uint16_t>(scale);
    }
}

template <typename T, int R>
__global__ void __launch_bounds__(ROW_THREADS) kv4_read_kernel(const RowParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    const int kv = (threadIdx.x >> 4) & 1, l = threadIdx.x & 15, g = l >> 2, j = l & 3;
    const int page = 1 << prm.pages.shift;
    const Rows first = Rows::of<R>(prm);
    Rows row = first;
    uint32_t w[R], s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        int off = 0;
        w[i] = 0x88888888u, s[i] = 0;      // without a place in the cache: codes of 0, so 0 and not -0
        const uint8_t *blk = row.left > 0 ? row.block(prm, off) : nullptr;
        row.next(prm);
        if (!blk) continue;
        const uint8_t *codes = blk + (kv ? v_codes(page) : 0) + off * 64 + 16 * j;
        w[i] = kv ? *reinterpret_cast<const uint16_t *>(codes + 2 * g) |
                        static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(codes + 8 + 2 * g)) << 16
                  : *reinterpret_cast<const uint32_t *>(codes + 4 * g);
        s[i] = reinterpret_cast<const uint16_t *>(blk + (kv ? v_scales(page) : k_scales(page)))[off * 4 + g];
    }
    T *out = static_cast<T *>(kv ? prm.vo : prm.ko) +
             ((static_cast<long long>(first.b) * prm.T + first.t) * prm.H + first.h) * DH + 8 * l;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (i >= first.left) break;
        float x[8];
#pragma unroll
        for (int c = 0; c < 8; ++c)      // 2^23 + u is the f32 number of these bits; a scale of 0 gives 0
            x[c] = __fsub_rn(__uint_as_float(0x4b000000u | ((w[i] >> (4 * c)) & 15u)), 8388616.0f) *
                   __uint_as_float(s[i] << 16);
        store8(out + i * DH, x);      // rows follow one another
    }
}

// ---- attention over the pages -------------------------------------------
//
// o[r] = sum_j p_rj v_j / sum_j p_rj, p_rj = exp(scale q_r k_j - max), for the G T query
// rows r = t G + g that share a cache head, 8 NT rows to a CTA.  Every code is read once per row
// tile, by asynchronous copies into a ring of each warp, and goes from there into the
// fragments of the fp16 warp MMA (m16n8k16) with tokens or channels as its 16 rows and the
// query rows as its 8 columns: with 8 rows the MMA's half-empty other form would cost
// as much as the codes' conversion.
//
// What bounds it (64 sequences of 4096 tokens, 8 heads, one row each): 75 us for 302 MB, 4.0
// TB/s; the copies alone take 53 us, copies and scores 55 us.  An instruction that turns
// codes into fragments works on two codes a lane, which makes some 340 instructions for 16
// tokens (171 on the integer pipe, which would take 85 cycles at full rate) where the bytes
// take 101 cycles an SM; with three CTAs an SM the warps cannot hide all their latencies.
//
// Scores: a nibble u = c + 8 masked out of its word is the subnormal fp16 number u 2^-24
// (or u 2^-20), exact in the MMA, so a fragment costs one instruction; the accumulators
// start from -8 sum q, which leaves sum q c.  Each group of 32 channels has its own
// accumulator, and the scales multiply these in f32.  q enters as fp16 times a power of two
// of its row (largest magnitude in [2^14, 2^15)): exact but for elements more than 2^24
// smaller than the largest, which lose parts below 2^-39 of it.
//
// Softmax: running reference and sum in f32, per warp over its own tokens (32 at a time).
//
// Output: p times the V scale, relative to the running largest exponent of the V scales that
// the row sees and times 2^HEAD, rounds to fp16 (half a step 2^-11; terms below 2^-23 of the
// largest fade out gradually): the codes enter exactly as u - 8, and the sums are f32.  A choice
// for the MMA's rate, since a second piece of p s would double the output product.  It is not
// free: the error of fp16 outputs against 64 bits is 1.15 to 1.3 times that of f32 arithmetic
// rounded once (33 queries over 1500 tokens 2.4e-4 for 2.1e-4, one over 375 2.6e-4 for 2.0e-4);
// that of bf16 outputs is their own rounding (1.7e-3 either way).
//
// Split: the keys of all items in a row, cut into units of 128, are dealt in equal shares to
// one wave of CTAs, whatever the lengths: each CTA sums up the lengths to find where its
// share begins.  A share may end one item, hold some and begin another; only the first and
// the last of its parts can be parts of an item, and these two go to the workspace, where
// a second kernel joins them in order.  (Equal chunks of every item instead, 912 of them for
// 608 CTAs at a time: 64 sequences of 4096 tokens, 8 heads: 84 us; ragged to 8192: 102 us.)
// The workspace carries nothing from one call to the next.  The warps of a CTA merge in
// shared memory.

constexpr int ATT_WARPS = 4;
constexpr int ATT_THREADS = 32 * ATT_WARPS;
constexpr int CTAS_8 = 3, CTAS_16 = 2;        // CTAs on an SM with 8 and 16 rows
constexpr int UNIT = 128;                     // keys of a unit of work: 32 to a warp
constexpr int OVER = 3;                       // units that beginning an item is counted as (ragged to 8192: 1 91 us, 2 85, 3 78)
constexpr int MAX_SCAN = 2048;                // row tiles of all sequences that a CTA will sum up
constexpr int PART = DH + 4;                  // floats of a partial row: output, maximum, sum, two unused

struct AttParams {
    const void *q;
    void *out;
    long long qs[3];
    const int32_t *lengths, *count;
    int B, T, H, G;                           // H cache heads, G query heads to each
    int causal, max_len;
    int tiles;                                // row tiles of (b, h)
    int split;                                // 0: a CTA per item
    float scale_log2;                         // softmax scale times log2 e
    Pages pages;
    int2 *open;                               // [CTA]: item that its last part leaves open (-1: none), CTAs
    float *part;                              // [CTA][2][R][PART]
    int *err;
};

// A work item: the R = 8 NT query rows of tile e mod tiles of sequence e / tiles, cache head h.
struct Item {
    int b, h, row0, rows;
    int n, cnt;               // cached tokens, query tokens
    int kv_end, kv_full;      // keys that some row sees; that all rows see which see any

    __device__ Item(const AttParams &p, int e, int head, int R) {
        b = static_cast<int>(static_cast<unsigned>(e) / static_cast<unsigned>(p.tiles));
        h = head;
        const int tile = e - b * p.tiles;
        n = p.lengths[b];
        n = n < 0 ? 0 : (n > p.max_len ? p.max_len : n);
        cnt = p.count ? p.count[b] : p.T;
        cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
        row0 = tile * R;
        rows = p.G * p.T - row0 < R ? p.G * p.T - row0 : R;
        const int t_lo = row0 / p.G, t_hi = (row0 + rows - 1) / p.G, t_last = t_hi < cnt ? t_hi : cnt - 1;
        kv_end = t_last < t_lo ? 0 : (p.causal ? n - cnt + t_last + 1 : n);
        kv_end = kv_end < 0 ? 0 : kv_end;
        kv_full = p.causal ? n - cnt + t_lo + 1 : n;
    }
    // its work: units of 128 keys, one at least (its rows have to be written)
    __device__ int units() const { return kv_end <= UNIT ? 1 : (kv_end + UNIT - 1) / UNIT; }
    // keys that a row sees: the first limit(row) positions
    __device__ int limit(const AttParams &p, int row) const {
        const int t = (row0 + row) / p.G;
        if (row >= rows || t >= cnt) return 0;
        const int l = p.causal ? n - cnt + t + 1 : n;
        return l < 0 ? 0 : l;
    }
    template <typename T>
    __device__ T *out(const AttParams &p, int row) const {
        const int t = (row0 + row) / p.G, g = (row0 + row) - t * p.G;
        return static_cast<T *>(p.out) +
               ((static_cast<long long>(b) * p.T + t) * p.H * p.G + static_cast<long long>(h) * p.G + g) * DH;
    }
};

__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                      uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9},"
        " {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with d = (c0, c1, c0, c1) + A B.
__device__ __forceinline__ void mma16_from(float (&d)[4], const float (&c)[2], uint32_t a0, uint32_t a1,
                                           uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9},"
        " {%10,%11,%10,%11};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {      // of an 8 x 8 matrix of 16-bit values
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Nibbles 0 and 4 (or 1 and 5) of w as fp16 u - 8: 0x6400 | u is 1024 + u, 0x6400 | 16 u is
// 1024 + 16 u.
__device__ __forceinline__ uint32_t centred_lo(uint32_t w) {
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"((w & 0x000f000fu) | 0x64006400u), "r"(0xe408e408u));
    return r;
}
__device__ __forceinline__ uint32_t centred_hi(uint32_t w) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;"
        : "=r"(r)
        : "r"((w & 0x00f000f0u) | 0x64006400u), "r"(0x2c002c00u), "r"(0xd480d480u));   // / 16 - 72
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A row's output: 0 if it sees no key.
__device__ __forceinline__ float row_value(int limit, float acc, float sum) {
    return limit > 0 && sum != 0.0f ? __fdiv_rn(acc, sum) : 0.0f;
}

// 32 tokens of a warp in shared memory: K codes, V codes, K scales, V scales, copied as they
// lie in their pages, STAGES deep.
constexpr int STAGES = 2;
constexpr int HEAD = 9, SLACK = 4;      // p s / 2^e < 2^(SLACK + 1), so its fp16 value is below 2^14
constexpr int BATCH = 32, BATCH_BYTES = BATCH * ROW_BYTES;
constexpr int RING = STAGES * BATCH_BYTES;
// a warp's rows: [R][DH], then maximum and sum [R][2]
__host__ __device__ constexpr int row_floats(int R) { return R * (DH + 2); }
__host__ __device__ constexpr int smem_bytes(int R) { return ATT_WARPS * (RING + row_floats(R) * 4); }
constexpr int B_V = BATCH * 64, B_KS = 2 * BATCH * 64, B_VS = B_KS + BATCH * 8;

template <int D = 0, int S = 0>
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0+%2], [%1+%3], 16;" ::"r"(dst), "l"(src), "n"(D), "n"(S)
                 : "memory");
}
template <int O>
__device__ __forceinline__ uint4 at128(const uint8_t *p) { return *reinterpret_cast<const uint4 *>(p + O); }
template <int O>
__device__ __forceinline__ uint2 at64(const uint8_t *p) { return *reinterpret_cast<const uint2 *>(p + O); }

template <typename T, int NT, int PAGE>
__global__ void __launch_bounds__(ATT_THREADS, NT == 1 ? CTAS_8 : CTAS_16) kv4_attention_kernel(const AttParams prm) {
    constexpr int R = 8 * NT;
    extern __shared__ __align__(128) uint8_t s_mem[];     // per warp its ring, then its rows
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g8 = lane >> 2, t4 = lane & 3;
    pdl_launch_dependents();
    pdl_wait();

    // this CTA's share: `left` units of all, from unit u0 of item (e, head) on
    __shared__ int s_start[3], s_sum[ATT_WARPS];
    int e, head, u0 = 0, share = 0, left = 0x7fffffff, over = 0;
    if (prm.split) {
        const int tid = threadIdx.x, E = prm.B * prm.tiles, per = (E + ATT_THREADS - 1) / ATT_THREADS;
        int mine = 0;
        for (int i = 0; i < per; ++i)
            if (tid * per + i < E) mine += Item(prm, tid * per + i, 0, R).units() * prm.H;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) s_sum[warp] = upto;
        __syncthreads();
        int total = 0;
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) {
            if (w < warp) upto += s_sum[w];
            total += s_sum[w];
        }
        // beginning an item takes about as long as OVER units: it is counted so, unless there
        // is a CTA for every unit
        if (total > static_cast<int>(gridDim.x)) {
            over = OVER;
            total += over * E * prm.H;
            const int items = (tid * per < E ? (E - tid * per < per ? E - tid * per : per) : 0) * prm.H;
            mine += over * items;
            upto += over * prm.H * (tid * per + per < E ? tid * per + per : E);
        }
        share = (total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x);
        const long long pos = static_cast<long long>(blockIdx.x) * share;
        if (tid == 0) prm.open[blockIdx.x] = make_int2(-1, 0);
        if (pos >= total) return;
        left = total - pos < share ? static_cast<int>(total - pos) : share;
        if (pos >= upto - mine && pos < upto) {
            int at = upto - mine;
            for (int i = 0; i < per; ++i) {
                const int u = over + Item(prm, tid * per + i, 0, R).units();
                if (pos < at + u * prm.H) {
                    s_start[0] = tid * per + i;
                    s_start[1] = (static_cast<int>(pos) - at) / u;
                    s_start[2] = (static_cast<int>(pos) - at) % u;
                    break;
                }
                at += u * prm.H;
            }
        }
        __syncthreads();
        e = s_start[0];
        head = s_start[1];
        u0 = s_start[2] - over;       // below 0: inside what the item's beginning is counted as
    } else {
        e = static_cast<int>(blockIdx.x / static_cast<unsigned>(prm.H));
        head = static_cast<int>(blockIdx.x - static_cast<unsigned>(e) * prm.H);
    }

    // the part of item `it` that the share holds: units u0 .. u1 - 1; false if it ends before
    // the item's first key
    Item it(prm, e, head, R);
    int units = it.units(), u1 = 0;
    auto take = [&]() {
        u1 = units - u0 <= left ? units : u0 + left;
        left -= u1 - u0;
        u0 = u0 < 0 ? 0 : u0;
        if (u0 == 0 && u1 > 0 && head == 0 && threadIdx.x == 0 &&
            (prm.lengths[it.b] > prm.max_len || (it.kv_end > 0 && prm.pages.n_pages == 0)))
            atomicOr(prm.err, ERR_PARAM);
        return u1 > 0;
    };
    if (!take()) return;

    // the warp's batches: 32 tokens every 128; the copies run STAGES - 1 ahead of the products, the
    // page ids one more
    constexpr int STEP = BATCH * ATT_WARPS;
    uint8_t *const my_ring = s_mem + warp * RING;
    const uint32_t ring = smem_u32(my_ring);
    float *const my_rows = reinterpret_cast<float *>(s_mem + ATT_WARPS * RING) + warp * row_floats(R);
    int ahead = 0, end = 0, slot = 0, pid[2] = {0, 0};
    uint32_t use = 0;            // offset of the slot in use
    uint32_t dead = 0;           // two bits per copied batch, the newest lowest: half without a page
    const int32_t *table = nullptr;
    auto pages_ahead = [&]() {
        pid[0] = ahead < end ? table[static_cast<unsigned>(ahead) / PAGE] : 0;
        pid[1] = PAGE == 16 && ahead + 16 < end ? table[static_cast<unsigned>(ahead) / PAGE + 1] : pid[0];
    };
    auto copy = [&]() {
        dead <<= 2;
        if (ahead < end) {
            const bool bad0 = pid[0] < 0 || pid[0] >= prm.pages.n_pages;
            const bool bad1 = pid[1] < 0 || pid[1] >= prm.pages.n_pages;
            if (bad0 || bad1) {
                dead |= (bad0 ? 1u : 0u) | (bad1 ? 2u : 0u);
                if (lane == 0) atomicOr(prm.err, ERR_PARAM);
            }
            const uint32_t dst = ring + slot * BATCH_BYTES + lane * 16;
            const long long stride = static_cast<long long>(prm.H) * (ROW_BYTES * PAGE);
            const uint8_t *first = prm.pages.cache + it.h * (ROW_BYTES * PAGE);
            if (PAGE == 16) {
                // half a batch each from two pages; scales: a quarter of the lanes for K, K, V, V
                const uint8_t *p0 = first + (bad0 ? 0 : pid[0]) * stride, *p1 = first + (bad1 ? 0 : pid[1]) * stride;
                const uint8_t *c0 = p0 + lane * 16, *c1 = p1 + lane * 16;
                copy16(dst, c0);
                copy16<512, 512>(dst, c0);
                copy16<1024>(dst, c1);
                copy16<1536, 512>(dst, c1);
                copy16<B_V, v_codes(PAGE)>(dst, c0);
                copy16<B_V + 512, v_codes(PAGE) + 512>(dst, c0);
                copy16<B_V + 1024, v_codes(PAGE)>(dst, c1);
                copy16<B_V + 1536, v_codes(PAGE) + 512>(dst, c1);
                copy16<B_KS>(dst, (lane & 8 ? p1 : p0) + (lane & 16 ? v_scales(PAGE) : k_scales(PAGE)) + (lane & 7) * 16);
            } else {
                const int o0 = ahead & (PAGE - 1);
                const uint8_t *blk = first + (bad0 ? 0 : pid[0]) * stride + (o0 * 64 + lane * 16);
                copy16(dst, blk);
                copy16<512, 512>(dst, blk);
                copy16<1024, 1024>(dst, blk);
                copy16<1536, 1536>(dst, blk);
                copy16<B_V, v_codes(PAGE)>(dst, blk);
                copy16<B_V + 512, v_codes(PAGE) + 512>(dst, blk);
                copy16<B_V + 1024, v_codes(PAGE) + 1024>(dst, blk);
                copy16<B_V + 1536, v_codes(PAGE) + 1536>(dst, blk);
                // K scales by lanes 0-15, V scales by lanes 16-31
                copy16<B_KS>(dst, blk + ((lane < 16 ? k_scales(PAGE) : v_scales(PAGE) - 256) - o0 * 56));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += STEP;
        pages_ahead();
        slot = slot + 1 == STAGES ? 0 : slot + 1;
    };
    auto start = [&]() {          // the first copies of a part
        table = prm.pages.table + static_cast<long long>(it.b) * prm.pages.max_pages;
        ahead = u0 * UNIT + warp * BATCH;
        end = it.kv_end < u1 * UNIT ? it.kv_end : u1 * UNIT;
        end = prm.pages.n_pages > 0 ? end : 0;
        use = slot * BATCH_BYTES;
        pages_ahead();
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) copy();
    };
    start();

    for (;;) {
        const int b = it.b, h = it.h, row0 = it.row0, kv_end = it.kv_end, t_begin = u0 * UNIT + warp * BATCH, t_end = end;

        // query fragments (row g8 of each eight), group sums and per-row constants (rows 2 t4, 2 t4 + 1)
        uint32_t qf[NT][4][4];
        float qsum[NT][4][2], rscale[NT][2];
        int lim[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = nt * 8 + g8;
            const bool live = it.limit(prm, row) > 0;
            float x[4][8], top = 0.0f;
            const int t = (row0 + row) / prm.G, g = (row0 + row) - t * prm.G;
            const T *src = static_cast<const T *>(prm.q) +
                           (live ? b * prm.qs[0] + t * prm.qs[1] + (static_cast<long long>(h) * prm.G + g) * prm.qs[2] : 0);
            const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
#pragma unroll
            for (int gr = 0; gr < 4; ++gr) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[gr][i] = 0.0f;
                if (live) load8(src + 32 * gr + 8 * t4, vec, x[gr]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[gr][i]));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int ex = 268 - static_cast<int>(__float_as_uint(top) >> 23);
            const int fe = ex > 254 ? 254 : ex;
            const float up = __uint_as_float(static_cast<uint32_t>(fe) << 23);
            // > 0, since it multiplies -inf, and finite, since it multiplies 0: at the upper end (a
            // query of 2^121 at 1 / sqrt(128)) scores that differ still do by 2^7 and more, as long as
            // their keys are above 2^-96
            const float rs = fminf(fmaxf(ldexpf(prm.scale_log2, 24 - (fe - 127)), 0x1p-126f), 0x1p127f);
            float sums[4];
#pragma unroll
            for (int gr = 0; gr < 4; ++gr) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[gr][i] *= up;
                    s += x[gr][i];
                }
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
                sums[gr] = s * -0x1p-21f;      // -8 2^-24
                // nibbles 0, 4 and 2, 6 (u 2^-24), then 1, 5 and 3, 7 (u 2^-20: q by 2^-4)
                qf[nt][gr][0] = pack_half2(x[gr][0], x[gr][4]);
                qf[nt][gr][1] = pack_half2(x[gr][2], x[gr][6]);
                qf[nt][gr][2] = pack_half2(x[gr][1] * 0.0625f, x[gr][5] * 0.0625f);
                qf[nt][gr][3] = pack_half2(x[gr][3] * 0.0625f, x[gr][7] * 0.0625f);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int from = (2 * t4 + i) * 4;       // a lane of that row
#pragma unroll
                for (int gr = 0; gr < 4; ++gr) qsum[nt][gr][i] = __shfl_sync(0xffffffffu, sums[gr], from);
                rscale[nt][i] = __shfl_sync(0xffffffffu, rs, from);
                lim[nt][i] = it.limit(prm, nt * 8 + 2 * t4 + i);
            }
        }

        // Row i of the score MMA is token i / 2 of its eight for even i, 4 + (i / 2 ^ 1) for odd i: the
        // 16-byte reads of neighbouring rows fall on different banks, and the transposed
        // probabilities of lane (g8, t4) belong to the tokens t4 and 4 + (t4 ^ 1) of each eight.
        const int tok = g8 & 1 ? 4 + ((g8 >> 1) ^ 1) : g8 >> 1, odd4 = 4 + (t4 ^ 1);
        const uint8_t *at_k = my_ring + tok * 64 + t4 * 16, *at_s = my_ring + tok * 8;
        const uint8_t *at_v = my_ring + t4 * 64 + g8 * 8, *at_vo = my_ring + odd4 * 64 + g8 * 8;
        // m: the reference of the row's exponentials (-inf: no key yet, and then none in the later
        // batches either, a row sees the first keys), mr: in units of log2.  It is raised to the
        // maximum only when a score exceeds it by more than SLACK there (lift: the score that does):
        // the probabilities reach 2^SLACK at most, and most batches skip the rescaling.
        // far: a row's reference is 2^20 or more, where the rounding of mr begins to show in the
        // exponents (2^25: a step of 1).  Then the scores are taken less m before they are scaled,
        // and every score above m raises it.
        bool far = false;
        float o[NT][8][4], m[NT][2], mr[NT][2], l[NT][2], lift[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[nt][i] = lift[nt][i] = -INFINITY;
                mr[nt][i] = l[nt][i] = 0.0f;
            }
        }
        // 2^(HEAD - (ev - 127)) for ev, the running largest exponent field of the V scales that the
        // row sees (all rows alike until a batch that some see in part)
        float norm[NT][2];
        uint32_t ev_top = (17u << 7) - 1u;            // largest scale of the lane's smallest ev
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) norm[nt][0] = norm[nt][1] = __uint_as_float((254u + HEAD - 16u) << 23);

        for (int t0 = t_begin; t0 < t_end; t0 += STEP) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();     // all lanes' copies have landed, and all have read the slot before
            copy();
            const uint32_t gone = (dead >> (2 * (STAGES - 1))) & 3u;       // this batch was copied so long ago
            const bool full = t0 + BATCH <= it.kv_full && gone == 0;

            // scores: rows 2 t4 and 2 t4 + 1 for the tokens tok, 8 + tok, 16 + tok, 24 + tok
            float s[NT][8];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint4 k0 = hf ? at128<1024>(at_k + use) : at128<0>(at_k + use);
                const uint4 k1 = hf ? at128<1536>(at_k + use) : at128<512>(at_k + use);
                const uint2 c0 = hf ? at64<B_KS + 128>(at_s + use) : at64<B_KS>(at_s + use);
                const uint2 c1 = hf ? at64<B_KS + 192>(at_s + use) : at64<B_KS + 64>(at_s + use);
#pragma unroll
                for (int gr = 0; gr < 4; ++gr) {
                    const uint32_t w0 = gr == 0 ? k0.x : (gr == 1 ? k0.y : (gr == 2 ? k0.z : k0.w)), y0 = w0 >> 8;
                    const uint32_t w1 = gr == 0 ? k1.x : (gr == 1 ? k1.y : (gr == 2 ? k1.z : k1.w)), y1 = w1 >> 8;
                    const uint32_t s0 = gr < 2 ? c0.x : c0.y, s1 = gr < 2 ? c1.x : c1.y;
                    const float f0 = gr & 1 ? bf16_hi(s0) : bf16_lo(s0), f1 = gr & 1 ? bf16_hi(s1) : bf16_lo(s1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4], (&r)[8] = s[nt];
                        mma16_from(acc, qsum[nt][gr], w0 & 0x000f000fu, w1 & 0x000f000fu, y0 & 0x000f000fu,
                                   y1 & 0x000f000fu, qf[nt][gr][0], qf[nt][gr][1]);
                        mma16(acc, w0 & 0x00f000f0u, w1 & 0x00f000f0u, y0 & 0x00f000f0u, y1 & 0x00f000f0u,
                              qf[nt][gr][2], qf[nt][gr][3]);
                        r[4 * hf] = gr == 0 ? f0 * acc[0] : fmaf(f0, acc[0], r[4 * hf]);
                        r[4 * hf + 1] = gr == 0 ? f0 * acc[1] : fmaf(f0, acc[1], r[4 * hf + 1]);
                        r[4 * hf + 2] = gr == 0 ? f1 * acc[2] : fmaf(f1, acc[2], r[4 * hf + 2]);
                        r[4 * hf + 3] = gr == 0 ? f1 * acc[3] : fmaf(f1, acc[3], r[4 * hf + 3]);
                    }
                }
            }
            uint2 vs[4] = {at64<B_VS>(at_s + use), at64<B_VS + 64>(at_s + use), at64<B_VS + 128>(at_s + use),
                           at64<B_VS + 192>(at_s + use)};
            if (!full) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int pos = t0 + 8 * i + tok;
                    const bool none = (gone >> (i >> 1)) & 1u;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (none || pos >= lim[nt][j]) s[nt][2 * i + j] = -INFINITY;
                    // V scales of tokens that no row sees may hold anything
                    if (none || pos >= kv_end) vs[i] = make_uint2(0, 0);
                }
                // a scale that is no number times a probability of 0 would reach the rows that do not see
                // it: it goes straight to the sums of those that do
                uint32_t hit[NT][2] = {};      // a bit per group
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int gr = 0; gr < 4; ++gr) {
                        uint32_t &w = gr < 2 ? vs[i].x : vs[i].y;
                        if (((w >> (gr & 1 ? 23 : 7)) & 0xffu) != 255u) continue;
                        w &= gr & 1 ? 0xffffu : 0xffff0000u;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                if (s[nt][2 * i + j] != -INFINITY) hit[nt][j] |= 1u << gr;
                    }
                uint32_t any = 0;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) any |= hit[nt][0] | hit[nt][1];
                if (__any_sync(0xffffffffu, any != 0)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t x = hit[nt][j];
                            x |= __shfl_xor_sync(0xffffffffu, x, 4);
                            x |= __shfl_xor_sync(0xffffffffu, x, 8);
                            x |= __shfl_xor_sync(0xffffffffu, x, 16);
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                if ((x >> (c >> 1)) & 1u) o[nt][c][j] = o[nt][c][2 + j] = __uint_as_float(0x7fc00000u);
                        }
                }
            }
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    raise |= fmaxf(fmaxf(s[nt][j], s[nt][2 + j]), fmaxf(s[nt][4 + j], s[nt][6 + j])) > lift[nt][j];
            uint32_t top = __vimax3_u16x2(vs[0].x, vs[0].y, vs[1].x);
            top = __vimax3_u16x2(__vimax3_u16x2(top, vs[1].y, vs[2].x), vs[2].y, vs[3].x);
            top = __vimax3_u16x2(top, vs[3].y, 0u);
            raise |= (top >> 16) > ev_top || (top & 0xffffu) > ev_top;
            if (__any_sync(0xffffffffu, raise)) {
                int field[4];       // of the largest scale of each token
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    field[i] = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {     // a NaN (field 255) must not hide the others' range
                        const int f = static_cast<int>((j < 2 ? vs[i].x : vs[i].y) >> (j & 1 ? 23 : 7)) & 0xff;
                        field[i] = f < 255 && f > field[i] ? f : field[i];
                    }
                }
                ev_top = 0xffffu;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float t = m[nt][j];
#pragma unroll
                        for (int i = 0; i < 4; ++i) t = fmaxf(t, s[nt][2 * i + j]);
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                        const float tr = t == -INFINITY ? 0.0f : t * rscale[nt][j];
                        const float a = m[nt][j] == -INFINITY ? 0.0f : fast_exp2(mr[nt][j] - tr);
                        m[nt][j] = t;
                        mr[nt][j] = tr;
                        lift[nt][j] = t + __fdividef(static_cast<float>(SLACK), rscale[nt][j]);
                        l[nt][j] *= a;
                        const int ev = 254 + HEAD - static_cast<int>(__float_as_uint(norm[nt][j]) >> 23);
                        int en = ev;
#pragma unroll
                        for (int i = 0; i < 4; ++i) en = s[nt][2 * i + j] != -INFINITY ? max(en, field[i]) : en;
                        en = max(en, __shfl_xor_sync(0xffffffffu, en, 4));
                        en = max(en, __shfl_xor_sync(0xffffffffu, en, 8));
                        en = max(en, __shfl_xor_sync(0xffffffffu, en, 16));
                        norm[nt][j] = __uint_as_float(static_cast<uint32_t>(254 + HEAD - en) << 23);
                        ev_top = min(ev_top, (static_cast<uint32_t>(en + 1) << 7) - 1u);
                        const float ad = ev - en < -126 ? 0.0f : a * __uint_as_float(static_cast<uint32_t>(127 + ev - en) << 23);
#pragma unroll
                        for (int c = 0; c < 8; ++c) o[nt][c][j] *= ad, o[nt][c][2 + j] *= ad;
                    }
                bool high = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) high |= fmaxf(fabsf(mr[nt][0]), fabsf(mr[nt][1])) >= 0x1p20f;
                far = __any_sync(0xffffffffu, high);
                if (far)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) lift[nt][0] = m[nt][0], lift[nt][1] = m[nt][1];
            }
            float less[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) less[nt][0] = mr[nt][0], less[nt][1] = mr[nt][1];
            if (far) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[nt][i] -= m[nt][i & 1] == -INFINITY ? 0.0f : m[nt][i & 1];
                    less[nt][0] = less[nt][1] = 0.0f;
                }
            }
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                float p[NT][4];           // norm times the probabilities
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e1 = fast_exp2(fmaf(s[nt][4 * hf + i], rscale[nt][i & 1], -less[nt][i & 1]));
                        l[nt][i & 1] += e1;
                        p[nt][i] = e1 * norm[nt][i & 1];
                    }
                const uint2 v0 = hf ? at64<B_V + 1024>(at_v + use) : at64<B_V>(at_v + use);
                const uint2 v1 = hf ? at64<B_V + 1024>(at_vo + use) : at64<B_V>(at_vo + use);
                const uint2 v2 = hf ? at64<B_V + 1536>(at_v + use) : at64<B_V + 512>(at_v + use);
                const uint2 v3 = hf ? at64<B_V + 1536>(at_vo + use) : at64<B_V + 512>(at_vo + use);
#pragma unroll
                for (int gr = 0; gr < 4; ++gr) {
                    const uint32_t x0 = gr < 2 ? vs[2 * hf].x : vs[2 * hf].y, x1 = gr < 2 ? vs[2 * hf + 1].x : vs[2 * hf + 1].y;
                    const float f0 = gr & 1 ? bf16_hi(x0) : bf16_lo(x0), f1 = gr & 1 ? bf16_hi(x1) : bf16_lo(x1);
                    const uint32_t sel = gr & 1 ? 0x7632 : 0x5410;
                    const uint32_t a = gr < 2 ? __byte_perm(v0.x, v1.x, sel) : __byte_perm(v0.y, v1.y, sel);
                    const uint32_t c = gr < 2 ? __byte_perm(v2.x, v3.x, sel) : __byte_perm(v2.y, v3.y, sel);
                    const uint32_t a8 = a >> 8, c8 = c >> 8;
                    const uint32_t a0 = centred_lo(a), a1 = centred_hi(a), a2 = centred_lo(c), a3 = centred_hi(c);
                    const uint32_t d0 = centred_lo(a8), d1 = centred_hi(a8), d2 = centred_lo(c8), d3 = centred_hi(c8);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        // p s rounded to fp16, then tokens against rows turned into the MMA's order
                        const uint32_t b0 = transpose8(pack_half2(p[nt][0] * f0, p[nt][1] * f0));
                        const uint32_t b1 = transpose8(pack_half2(p[nt][2] * f1, p[nt][3] * f1));
                        mma16(o[nt][2 * gr], a0, a1, a2, a3, b0, b1);
                        mma16(o[nt][2 * gr + 1], d0, d1, d2, d3, b0, b1);
                    }
                }
            }
            use = use + BATCH_BYTES == STAGES * BATCH_BYTES ? 0 : use + BATCH_BYTES;
        }

        // the share's next part: its first copies run while this part's rows are joined
        const Item done = it;
        const int d0 = u0, d1 = u1, d_units = units, d_item = e * prm.H + head;
        bool more = prm.split && u1 == units && left > 0;
        if (more) {
            u0 = -over;
            if (++head == prm.H) head = 0, ++e;
            it = Item(prm, e, head, R);
            units = it.units();
            more = take();
            __syncwarp();
            if (more) start();
        }
        __syncthreads();              // the rows before these have been read

        // a warp's rows to shared memory: output over norm, maximum, sum
        {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float sum = l[nt][i];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                    if (g8 == 0) {
                        float *ml = my_rows + R * DH + 2 * (nt * 8 + 2 * t4 + i);
                        ml[0] = m[nt][i] == -INFINITY ? -INFINITY : mr[nt][i];
                        ml[1] = sum;
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // 1 / norm
                    const float unit = ldexpf(1.0f, 127 - static_cast<int>(__float_as_uint(norm[nt][i]) >> 23));
#pragma unroll
                    for (int c = 0; c < 8; ++c)      // m-tile c: channels 32 (c / 2) + 4 g8 + 2 (c & 1), + 1
                        *reinterpret_cast<float2 *>(my_rows + (nt * 8 + 2 * t4 + i) * DH + 32 * (c >> 1) + 4 * g8 +
                                                    2 * (c & 1)) = make_float2(o[nt][c][i] * unit, o[nt][c][2 + i] * unit);
                }
            }
        }
        __syncthreads();

        const int d = threadIdx.x;                    // one channel a thread
        const bool whole = d0 == 0 && d1 == d_units;
        const float *all_rows = reinterpret_cast<const float *>(s_mem + ATT_WARPS * RING);
        for (int row = 0; row < done.rows; ++row) {
            const float *ml = all_rows + R * DH + 2 * row, *src = all_rows + row * DH + d;
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < ATT_WARPS; ++w) mx = fmaxf(mx, ml[w * row_floats(R)]);
            const float ref = mx == -INFINITY ? 0.0f : mx;
            float acc = 0.0f, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < ATT_WARPS; ++w) {
                const float a = fast_exp2(ml[w * row_floats(R)] - ref);
                acc += a * src[w * row_floats(R)];
                sum += a * ml[w * row_floats(R) + 1];
            }
            if (whole) {
                done.out<T>(prm, row)[d] = from_f32<T>(row_value(done.limit(prm, row), acc, sum));
            } else {
                float *dst = prm.part + ((static_cast<long long>(blockIdx.x) * 2 + (d0 > 0 ? 0 : 1)) * R + row) * PART;
                dst[d] = acc;
                if (d == 0) dst[DH] = mx, dst[DH + 1] = sum;
            }
        }
        // the item goes on in the next CTAs: the one where it begins says so
        if (d1 < d_units && d0 == 0 && threadIdx.x == 0)
            prm.open[blockIdx.x] = make_int2(d_item, 1 + (d_units - d1 + share - 1) / share);
        if (!more) return;
    }
}

// One query row of an item that lies in several CTAs, by the CTA (x) where it begins: part 1
// of that one, part 0 of the next ones.  Each thread first weighs the parts t, t + 128, ... of a
// round by their maxima, then warp w adds the parts w, w + 4, ..., four channels a lane.
template <typename T, int NT>
__global__ void __launch_bounds__(ATT_THREADS) kv4_join_kernel(const AttParams prm) {
    constexpr int R = 8 * NT;
    __shared__ float s_w[ATT_THREADS], s_red[2][ATT_WARPS], s_o[ATT_WARPS][DH];
    pdl_launch_dependents();
    pdl_wait();
    const int2 open = prm.open[blockIdx.x];
    if (open.x < 0) return;
    const int parts = open.y;
    const Item it(prm, open.x / prm.H, open.x % prm.H, R);
    const int row = blockIdx.y;
    if (row >= it.rows) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr long long step = 2ll * R * PART;
    // part c > 0 is part 0 of CTA x + c; part 0 lies R rows further on
    const float *src = prm.part + (static_cast<long long>(blockIdx.x) * 2 * R + row) * PART;
    auto at = [&](int c) { return src + c * step + (c == 0 ? R * PART : 0); };
    float mx = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < parts; c0 += ATT_THREADS) {
        const int left = parts - c0 < ATT_THREADS ? parts - c0 : ATT_THREADS;
        const float2 ml = tid < left ? *reinterpret_cast<const float2 *>(at(c0 + tid) + DH)
                                     : make_float2(-INFINITY, 0.0f);
        float t = ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
        if (lane == 0) s_red[0][warp] = t;
        __syncthreads();
        t = mx;
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) t = fmaxf(t, s_red[0][w]);
        const float ref = t == -INFINITY ? 0.0f : t;
        const float e = fast_exp2(ml.x - ref), a = fast_exp2(mx - ref);
        s_w[tid] = e;
        float l = ml.y * e;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (lane == 0) s_red[1][warp] = l;
        __syncthreads();
        mx = t;
        sum *= a;
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) sum += s_red[1][w];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= a;
        int c = warp;
        for (; c + 7 * ATT_WARPS < left; c += 8 * ATT_WARPS) {
            float4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const float4 *>(at(c0 + c + i * ATT_WARPS) + 4 * lane);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = s_w[c + i * ATT_WARPS];
                acc[0] = fmaf(w, v[i].x, acc[0]);
                acc[1] = fmaf(w, v[i].y, acc[1]);
                acc[2] = fmaf(w, v[i].z, acc[2]);
                acc[3] = fmaf(w, v[i].w, acc[3]);
            }
        }
#pragma unroll 4
        for (; c < left; c += ATT_WARPS) {
            const float4 v = *reinterpret_cast<const float4 *>(at(c0 + c) + 4 * lane);
            const float w = s_w[c];
            acc[0] = fmaf(w, v.x, acc[0]);
            acc[1] = fmaf(w, v.y, acc[1]);
            acc[2] = fmaf(w, v.z, acc[2]);
            acc[3] = fmaf(w, v.w, acc[3]);
        }
        __syncthreads();      // the weights are read before the next round's
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[warp][4 * lane + i] = acc[i];
    __syncthreads();
    float o = 0.0f;
#pragma unroll
    for (int w = 0; w < ATT_WARPS; ++w) o += s_o[w][tid];
    it.out<T>(prm, row)[tid] = from_f32<T>(row_value(it.limit(prm, row), o, sum));
}

}  // namespace ipv
