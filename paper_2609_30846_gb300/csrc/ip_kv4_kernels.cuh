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

// Block of the page of position pos, nullptr (and the status word) if the table has none.
__device__ __forceinline__ uint8_t *page_block(const Pages &p, int b, int pos, int h, int *err) {
    const int pid = p.table[static_cast<long long>(b) * p.max_pages + (pos >> p.shift)];
    if (pid < 0 || pid >= p.n_pages) {
        atomicOr(err, ERR_PARAM);
        return nullptr;
    }
    return p.cache + ((static_cast<long long>(pid) * p.heads + h) * ROW_BYTES << p.shift);
}

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

constexpr int ROW_THREADS = 256;             // a warp per token and head

// The bf16 value nearest to amax / 7, ties to even.  The f32 quotient decides unless it
// falls on the middle of two bf16 values: seven times that middle (twelve bits) is exact.
__device__ __forceinline__ uint32_t scale4(float amax) {
    const float q = __fdiv_rn(amax, 7.0f);
    const uint32_t bits = __float_as_uint(q), lo = bits >> 16, rem = bits & 0xffffu;
    if (rem != 0x8000u) return lo + (rem > 0x8000u ? 1u : 0u);
    const float t = 7.0f * q;
    return lo + (amax > t ? 1u : (amax < t ? 0u : (lo & 1u)));
}

// Nibble of x for the scale s > 0: the integer nearest to x / s, ties to even, within
// -7 .. 7, plus 8.  Near a half integer |x| is compared with (n + 1/2) s, twelve bits and exact.
__device__ __forceinline__ uint32_t code4(float x, float s, float inv) {
    const float ax = fabsf(x), y = ax * inv;
    int n = __float2int_rn(fminf(y, 8.0f));
    const float f = rintf(y - 0.5f);
    if (fabsf(y - 0.5f - f) < 0x1p-12f) {
        const float t = (f + 0.5f) * s;
        const int ni = static_cast<int>(f);
        n = ax > t ? ni + 1 : (ax < t ? ni : ni + (ni & 1));
    }
    n = min(n, 7);
    return static_cast<uint32_t>(8 + (x < 0.0f ? -n : n));
}

// One row of a warp: lane l holds channels 4 l .. 4 l + 3 of group l / 8; returns its four
// nibbles and the group's scale (bf16 bits).
__device__ __forceinline__ uint32_t quant4(const float (&x)[4], uint32_t &scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top >= 0x7f800000u) {      // a NaN or an infinity: the group reads back as NaN
        scale = 0x7fc0u;
        return 0x8888u;
    }
    scale = scale4(__uint_as_float(top));
    if (scale == 0) return 0x8888u;
    // a tiny scale and its row brought up by 2^100, exactly
    const float up = scale < (27u << 7) ? 0x1p100f : 1.0f;
    const float s = __uint_as_float(scale << 16) * up, inv = __fdiv_rn(1.0f, s);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= code4(x[i] * up, s, inv) << (4 * i);
    return w;
}

// The row of one warp of the launch; false if the warp has none.
__device__ __forceinline__ bool row_of(const RowParams &p, int &b, int &t, int &h) {
    const long long r = static_cast<long long>(blockIdx.x) * (ROW_THREADS / 32) + (threadIdx.x >> 5);
    if (r >= static_cast<long long>(p.B) * p.T * p.H) return false;
    const unsigned bt = static_cast<unsigned>(r / p.H);
    h = static_cast<int>(r - static_cast<long long>(bt) * p.H);
    b = static_cast<int>(bt / static_cast<unsigned>(p.T));
    t = static_cast<int>(bt - static_cast<unsigned>(b) * p.T);
    return true;
}

// Page block of the warp's position, nullptr if the token is padding or has no place.
__device__ __forceinline__ uint8_t *row_block(const RowParams &p, int b, int t, int h, int &off) {
    const int n = p.count ? p.count[b] : p.T;
    if (t >= n) return nullptr;
    const long long pos = static_cast<long long>(p.start[b]) + t;
    if (pos < 0 || pos >= static_cast<long long>(p.pages.max_pages) << p.pages.shift) {
        atomicOr(p.err, ERR_PARAM);
        return nullptr;
    }
    off = static_cast<int>(pos) & ((1 << p.pages.shift) - 1);
    return page_block(p.pages, b, static_cast<int>(pos), h, p.err);
}

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS) kv4_append_kernel(const RowParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    int b, t, h, off;
    if (!row_of(prm, b, t, h)) return;
    const int lane = threadIdx.x & 31;
    uint8_t *blk = row_block(prm, b, t, h, off);
    if (!blk) return;
    const int page = 1 << prm.pages.shift, g = lane >> 3, r = (lane & 7) * 4;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        const long long *st = kv ? prm.vs : prm.ks;
        const T *src = static_cast<const T *>(kv ? prm.v : prm.k) + b * st[0] + t * st[1] + h * st[2];
        float x[4];
        load4(src + 4 * lane, x);
        uint32_t scale;
        const uint32_t w = quant4(x, scale);
        uint8_t *codes = blk + (kv ? v_codes(page) : 0) + off * 64;
        const int byte = kv ? 8 * (r >> 2) + 2 * g : 16 * (r >> 3) + 4 * g + ((r & 7) >> 1);
        *reinterpret_cast<uint16_t *>(codes + byte) = static_cast<uint16_t>(w);
        if ((lane & 7) == 0)
            reinterpret_cast<uint16_t *>(blk + (kv ? v_scales(page) : k_scales(page)))[off * 4 + g] =
                static_cast<uint16_t>(scale);
    }
}

template <typename T>
__global__ void __launch_bounds__(ROW_THREADS) kv4_read_kernel(const RowParams prm) {
    pdl_launch_dependents();
    pdl_wait();
    int b, t, h, off = 0;
    if (!row_of(prm, b, t, h)) return;
    const int lane = threadIdx.x & 31;
    const uint8_t *blk = row_block(prm, b, t, h, off);
    const int page = 1 << prm.pages.shift, g = lane >> 3, r = (lane & 7) * 4;
    const long long at = ((static_cast<long long>(b) * prm.T + t) * prm.H + h) * DH + 4 * lane;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (blk) {
            const uint8_t *codes = blk + (kv ? v_codes(page) : 0) + off * 64;
            const int byte = kv ? 8 * (r >> 2) + 2 * g : 16 * (r >> 3) + 4 * g + ((r & 7) >> 1);
            const uint32_t w = *reinterpret_cast<const uint16_t *>(codes + byte);
            const uint32_t s = reinterpret_cast<const uint16_t *>(
                blk + (kv ? v_scales(page) : k_scales(page)))[off * 4 + g];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = static_cast<float>(static_cast<int>((w >> (4 * i)) & 15u) - 8) * __uint_as_float(s << 16);
        }
        store4(static_cast<T *>(kv ? prm.vo : prm.ko) + at, x);
    }
}

// ---- attention over the pages -------------------------------------------
//
// o[r] = sum_j p_rj v_j / sum_j p_rj, p_rj = exp(scale q_r k_j - max), for the G T query
// rows r = t G + g that share a cache head, 8 NT rows to a CTA and the keys cut into
// chunks.  Bound by the cache's bytes: every code is read once per row tile, straight from
// global memory into the fragments of the fp16 warp MMA (m16n8k16) with tokens or
// channels as its 16 rows and the query rows as its 8 columns.
//
// Scores: a nibble u = c + 8 masked out of its word is the subnormal fp16 number u 2^-24
// (or u 2^-20), exact in the MMA, so a fragment costs one instruction; the accumulators
// start from -8 sum q, which leaves sum q c.  Each group of 32 channels has its own
// accumulator, and the scales multiply these in f32.  q enters as fp16 times a power of two
// of its row (largest magnitude in [2^14, 2^15)): exact but for elements more than 2^24
// smaller than the largest, which lose parts below 2^-39 of it.
//
// Softmax: running maximum and sum in f32, per warp over its own tokens (16 at a time).
//
// Output: p times the V scale, relative to the running largest exponent of the V scales
// and times 2^13, rounds to fp16 (half a step 2^-11; terms below 2^-27 of the largest fade
// out gradually): the codes enter exactly as u - 8, and the sums are f32.  The
// rounding is below that of a bf16 output and no worse than that of an fp16 one.
//
// The warps of a CTA merge in shared memory, the chunks of an item through the workspace
// in a second kernel, in order (so the result does not depend on the schedule, and the
// workspace carries nothing from one call to the next).

constexpr int ATT_WARPS = 4;
constexpr int ATT_THREADS = 32 * ATT_WARPS;
constexpr int PART = DH + 2;                  // floats of a partial row: output, max, sum

struct AttParams {
    const void *q;
    void *out;
    long long qs[3];
    const int32_t *lengths, *count;
    int B, T, H, G;                           // H cache heads, G query heads to each
    int causal, max_len, chunk, chunks;       // tokens of a chunk, chunks an item has at most
    int tiles;                                // row tiles of (b, h)
    float scale_log2;                         // softmax scale times log2 e
    Pages pages;
    float *part;
    int *err;
};

// A work item: the 8 NT query rows `tile` of cache head h of sequence b.
struct Item {
    int b, h, row0, rows;
    int n, cnt;               // cached tokens, query tokens
    int kv_end, kv_full;      // keys that some row sees; that all rows see which see any
    int nchunks;

    __device__ Item(const AttParams &p, unsigned item, int R) {
        const unsigned bh = item / static_cast<unsigned>(p.tiles);
        const int tile = static_cast<int>(item - bh * p.tiles);
        b = static_cast<int>(bh / static_cast<unsigned>(p.H));
        h = static_cast<int>(bh - static_cast<unsigned>(b) * p.H);
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
        nchunks = (kv_end + p.chunk - 1) / p.chunk;
        nchunks = nchunks < 1 ? 1 : nchunks;
    }
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
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
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

// What a lane reads of 16 tokens.  Row i of the score MMA is token i / 2 + 4 (i & 1) of its
// half, so that the transposed probabilities of lane (g, t4) belong to tokens t4, t4 + 4,
// t4 + 8, t4 + 12.
struct Batch {
    uint4 k[2];
    uint2 ks[2], v[4], vs[4];
};

template <typename T, int NT>
__global__ void __launch_bounds__(ATT_THREADS, NT == 1 ? 3 : 2) kv4_attention_kernel(const AttParams prm) {
    constexpr int R = 8 * NT;
    __shared__ float s_o[ATT_WARPS][R][DH], s_ml[ATT_WARPS][R][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g8 = lane >> 2, t4 = lane & 3;
    pdl_launch_dependents();
    pdl_wait();

    const int chunk = blockIdx.y;
    const Item it(prm, blockIdx.x, R);
    if (chunk >= it.nchunks) return;
    if (chunk == 0 && threadIdx.x == 0 && prm.lengths[it.b] > prm.max_len) atomicOr(prm.err, ERR_PARAM);
    const int b = it.b, h = it.h, row0 = it.row0, rows = it.rows, kv_end = it.kv_end;
    const int begin = chunk * prm.chunk, end = kv_end < begin + prm.chunk ? kv_end : begin + prm.chunk;
    const int shift = prm.pages.shift, page = 1 << shift;
    const int32_t *table = prm.pages.table + static_cast<long long>(b) * prm.pages.max_pages;
    auto limit = [&](int row) { return it.limit(prm, row); };

    // query fragments, group sums and per-row constants
    uint32_t qf[NT][4][4];
    float qsum[NT][4][2], rscale[NT][2];
    int lim[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = nt * 8 + g8;
        const bool live = limit(row) > 0;
        float x[4][8], top = 0.0f;
        const int t = (row0 + row) / prm.G, g = (row0 + row) - t * prm.G;
        const T *src = static_cast<const T *>(prm.q) +
                       (live ? b * prm.qs[0] + t * prm.qs[1] + (static_cast<long long>(h) * prm.G + g) * prm.qs[2] : 0);
        const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
            if (live) load8(src + 32 * gr + 8 * t4, vec, 8, x[gr]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) x[gr][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[gr][i]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = 268 - static_cast<int>(__float_as_uint(top) >> 23);
        const int fe = e > 254 ? 254 : e;
        const float up = __uint_as_float(static_cast<uint32_t>(fe) << 23);
        const float rs = ldexpf(prm.scale_log2, 24 - (fe - 127));
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
            lim[nt][i] = limit(nt * 8 + 2 * t4 + i);
        }
    }

    const int tok = (g8 >> 1) + 4 * (g8 & 1);
    float o[NT][8][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) m[nt][i] = -INFINITY, l[nt][i] = 0.0f;
    }
    int ev = 16;          // running largest exponent field of the V scales

    // page of a batch, -1 if there is none
    auto page_of = [&](int t0) {
        if (t0 >= end) return -1;
        const int pid = table[t0 >> shift];
        return pid >= 0 && pid < prm.pages.n_pages ? pid : -1;
    };
    auto load = [&](int t0, int pid, Batch &x) {
        if (pid < 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) x.k[i] = make_uint4(0, 0, 0, 0), x.ks[i] = make_uint2(0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[i] = x.vs[i] = make_uint2(0, 0);
            return;
        }
        const uint8_t *blk = prm.pages.cache + ((static_cast<long long>(pid) * prm.H + h) * ROW_BYTES << shift);
        const int o0 = t0 & (page - 1);
        const uint8_t *kc = blk + (o0 + tok) * 64 + t4 * 16, *ks = blk + k_scales(page) + (o0 + tok) * 8;
        const uint8_t *vc = blk + v_codes(page) + (o0 + t4) * 64 + g8 * 8, *vs = blk + v_scales(page) + (o0 + t4) * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x.k[i] = ldg_stream128(kc + i * 512);
            x.ks[i] = ldg_stream64(ks + i * 64);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x.v[i] = ldg_stream64(vc + i * 256);
            x.vs[i] = ldg_stream64(vs + i * 32);
        }
    };

    auto compute = [&](int t0, int pid, const Batch &x) {
        const bool dead = pid < 0;      // no such page: all masked
        const bool full = t0 + 16 <= it.kv_full && !dead;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.0f;
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
            const uint32_t w0 = gr == 0 ? x.k[0].x : (gr == 1 ? x.k[0].y : (gr == 2 ? x.k[0].z : x.k[0].w));
            const uint32_t w1 = gr == 0 ? x.k[1].x : (gr == 1 ? x.k[1].y : (gr == 2 ? x.k[1].z : x.k[1].w));
            const uint32_t y0 = w0 >> 8, y1 = w1 >> 8;
            const uint32_t sw0 = gr < 2 ? x.ks[0].x : x.ks[0].y, sw1 = gr < 2 ? x.ks[1].x : x.ks[1].y;
            const float k0 = gr & 1 ? bf16_hi(sw0) : bf16_lo(sw0), k1 = gr & 1 ? bf16_hi(sw1) : bf16_lo(sw1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float acc[4] = {qsum[nt][gr][0], qsum[nt][gr][1], qsum[nt][gr][0], qsum[nt][gr][1]};
                mma16(acc, w0 & 0x000f000fu, w1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu,
                      qf[nt][gr][0], qf[nt][gr][1]);
                mma16(acc, w0 & 0x00f000f0u, w1 & 0x00f000f0u, y0 & 0x00f000f0u, y1 & 0x00f000f0u,
                      qf[nt][gr][2], qf[nt][gr][3]);
                s[nt][0] = fmaf(k0, acc[0], s[nt][0]);
                s[nt][1] = fmaf(k0, acc[1], s[nt][1]);
                s[nt][2] = fmaf(k1, acc[2], s[nt][2]);
                s[nt][3] = fmaf(k1, acc[3], s[nt][3]);
            }
        }
        bool raise = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] *= rscale[nt][i & 1];
            if (!full)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (dead || t0 + tok + 8 * (i >> 1) >= lim[nt][i & 1]) s[nt][i] = -INFINITY;
            raise |= fmaxf(s[nt][0], s[nt][2]) > m[nt][0] || fmaxf(s[nt][1], s[nt][3]) > m[nt][1];
        }
        // V scales; those of tokens that no row sees may hold anything
        uint2 vs[4];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vs[i] = x.vs[i];
            if (!full && (dead || t0 + t4 + 4 * i >= kv_end)) vs[i] = make_uint2(0, 0);
            top = __vmaxu2(top, __vmaxu2(vs[i].x, vs[i].y));
        }
        int et = static_cast<int>(max(top >> 16, top & 0xffffu) >> 7) & 0xff;
        if (et == 255) {       // a NaN among them: it must not hide the others' range
            et = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = j < 2 ? vs[i].x : vs[i].y;
                    const int f = static_cast<int>(w >> (j & 1 ? 23 : 7)) & 0xff;
                    et = f < 255 && f > et ? f : et;
                }
        }
        raise |= et > ev;
        if (__any_sync(0xffffffffu, raise)) {
            const int en = static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(et > ev ? et : ev)));
            const float down = ev - en < -126 ? 0.0f : __uint_as_float(static_cast<uint32_t>(127 + ev - en) << 23);
            ev = en;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float t = fmaxf(fmaxf(s[nt][i], s[nt][2 + i]), m[nt][i]);
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                    const float a = t == -INFINITY ? 1.0f : fast_exp2(m[nt][i] - t);
                    m[nt][i] = t;
                    l[nt][i] *= a;
                    const float ad = a * down;
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[nt][c][i] *= ad, o[nt][c][2 + i] *= ad;
                }
        }
        float p[NT][4];           // probability of query row 8 nt + g8 for tokens t4 + 4 i
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float m0 = m[nt][0] == -INFINITY ? 0.0f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.0f : m[nt][1];
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = fast_exp2(s[nt][i] - (i & 1 ? m1 : m0));
            l[nt][0] += e[0] + e[2];
            l[nt][1] += e[1] + e[3];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t a = __float_as_uint(e[2 * i]), c = __float_as_uint(e[2 * i + 1]);
                const uint32_t lo = transpose8(__byte_perm(a, c, 0x5410)), hi = transpose8(__byte_perm(a, c, 0x7632));
                p[nt][2 * i] = __uint_as_float(__byte_perm(lo, hi, 0x5410));
                p[nt][2 * i + 1] = __uint_as_float(__byte_perm(lo, hi, 0x7632));
            }
        }
        const float norm = __uint_as_float(static_cast<uint32_t>(267 - ev) << 23);    // 2^(13 - (ev - 127))
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = gr < 2 ? vs[i].x : vs[i].y;
                f[i] = (gr & 1 ? bf16_hi(w) : bf16_lo(w)) * norm;
            }
            const uint32_t sel = gr & 1 ? 0x7632 : 0x5410;
            const uint32_t a = gr < 2 ? __byte_perm(x.v[0].x, x.v[1].x, sel) : __byte_perm(x.v[0].y, x.v[1].y, sel);
            const uint32_t c = gr < 2 ? __byte_perm(x.v[2].x, x.v[3].x, sel) : __byte_perm(x.v[2].y, x.v[3].y, sel);
            const uint32_t a8 = a >> 8, c8 = c >> 8;
            const uint32_t a0 = centred_lo(a), a1 = centred_hi(a), a2 = centred_lo(c), a3 = centred_hi(c);
            const uint32_t d0 = centred_lo(a8), d1 = centred_hi(a8), d2 = centred_lo(c8), d3 = centred_hi(c8);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint32_t b0 = pack_half2(p[nt][0] * f[0], p[nt][1] * f[1]);
                const uint32_t b1 = pack_half2(p[nt][2] * f[2], p[nt][3] * f[3]);
                mma16(o[nt][2 * gr], a0, a1, a2, a3, b0, b1);
                mma16(o[nt][2 * gr + 1], d0, d1, d2, d3, b0, b1);
            }
        }
    };

    {
        int t0 = begin + warp * 16;
        constexpr int STEP = 16 * ATT_WARPS;
        // the pages run two batches ahead of the products, the rows one
        int pid = page_of(t0), pid1 = page_of(t0 + STEP);
        Batch x;
        if (t0 < end) load(t0, pid, x);
        while (t0 < end) {
            const int pid2 = page_of(t0 + 2 * STEP);
            Batch y;
            if (t0 + STEP < end) load(t0 + STEP, pid1, y);
            if (pid < 0 && lane == 0) atomicOr(prm.err, ERR_PARAM);
            compute(t0, pid, x);
            x = y;
            pid = pid1;
            pid1 = pid2;
            t0 += STEP;
        }
    }

    // a warp's rows to shared memory: output over 2^(ev - 140), maximum, sum
    {
        const float unit = ldexpf(1.0f, ev - 140);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = nt * 8 + 2 * t4 + i;
                float s = l[nt][i];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                if (g8 == 0) s_ml[warp][row][0] = m[nt][i], s_ml[warp][row][1] = s;
#pragma unroll
                for (int c = 0; c < 8; ++c)      // m-tile c: channels 32 (c / 2) + 4 g8 + 2 (c & 1), + 1
                    *reinterpret_cast<float2 *>(&s_o[warp][row][32 * (c >> 1) + 4 * g8 + 2 * (c & 1)]) =
                        make_float2(o[nt][c][i] * unit, o[nt][c][2 + i] * unit);
            }
    }
    __syncthreads();

    const int d = threadIdx.x;                    // one channel a thread
    for (int row = 0; row < rows; ++row) {
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) mx = fmaxf(mx, s_ml[w][row][0]);
        const float ref = mx == -INFINITY ? 0.0f : mx;
        float acc = 0.0f, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < ATT_WARPS; ++w) {
            const float a = fast_exp2(s_ml[w][row][0] - ref);
            acc += a * s_o[w][row][d];
            sum += a * s_ml[w][row][1];
        }
        if (it.nchunks == 1) {
            it.out<T>(prm, row)[d] = from_f32<T>(row_value(it.limit(prm, row), acc, sum));
        } else {
            float *dst = prm.part + ((static_cast<long long>(blockIdx.x) * prm.chunks + chunk) * R + row) * PART;
            dst[d] = acc;
            if (d == 0) dst[DH] = mx, dst[DH + 1] = sum;
        }
    }
}

// The chunks of one query row: a CTA per row, warp w the chunks w, w + 4, ..., four channels
// a lane, then the warps in order.
template <typename T, int NT>
__global__ void __launch_bounds__(ATT_THREADS) kv4_join_kernel(const AttParams prm) {
    constexpr int R = 8 * NT;
    __shared__ float s_o[ATT_WARPS][DH], s_ml[ATT_WARPS][2];
    pdl_launch_dependents();
    pdl_wait();
    const Item it(prm, blockIdx.x, R);
    const int row = blockIdx.y;
    if (it.nchunks == 1 || row >= it.rows) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float *src = prm.part + (static_cast<long long>(blockIdx.x) * prm.chunks * R + row) * PART;
    const long long step = static_cast<long long>(R) * PART;
    float mx = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int c = warp; c < it.nchunks; c += ATT_WARPS) {
        const float *p = src + c * step;
        const float2 lo = *reinterpret_cast<const float2 *>(p + 4 * lane);
        const float2 hi = *reinterpret_cast<const float2 *>(p + 4 * lane + 2);
        const float2 ml = *reinterpret_cast<const float2 *>(p + DH);
        const float t = fmaxf(mx, ml.x), ref = t == -INFINITY ? 0.0f : t;
        const float a = fast_exp2(mx - ref), e = fast_exp2(ml.x - ref);
        mx = t;
        sum = sum * a + ml.y * e;
        acc[0] = acc[0] * a + lo.x * e;
        acc[1] = acc[1] * a + lo.y * e;
        acc[2] = acc[2] * a + hi.x * e;
        acc[3] = acc[3] * a + hi.y * e;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[warp][4 * lane + i] = acc[i];
    if (lane == 0) s_ml[warp][0] = mx, s_ml[warp][1] = sum;
    __syncthreads();
    const int d = threadIdx.x;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < ATT_WARPS; ++w) top = fmaxf(top, s_ml[w][0]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float o = 0.0f, l = 0.0f;
#pragma unroll
    for (int w = 0; w < ATT_WARPS; ++w) {
        const float a = fast_exp2(s_ml[w][0] - ref);
        o += a * s_o[w][d];
        l += a * s_ml[w][1];
    }
    it.out<T>(prm, row)[d] = from_f32<T>(row_value(it.limit(prm, row), o, l));
}

}  // namespace ipv
