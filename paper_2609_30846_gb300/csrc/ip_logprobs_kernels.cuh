// Device code of the log probabilities of given tokens for sm_103a, with the entropy and the best
// tokens of each row of logits.
#pragma once

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "ip_ptx.cuh"
#include "ip_real.cuh"

namespace ipl {

using namespace ipk;
using namespace ipr;

// With a_i = scale x_i, m their maximum, s = sum exp(a_i - m), u = sum (a_i - m) exp(a_i - m):
//   log p_t = (a_t - m) - log s,   entropy = log s - u / s,
// both terms of the entropy >= 0, so that nothing cancels.  An a of -inf has no weight.  Differences are taken of halves,
// x / 2 - m / 2 by one fma, and scaled twice as much: those of logits of opposite signs can pass f32's range,
// where `scale` brings them back.
//
// A row (or one of its parts) is held in registers: one pass over memory, the maximum before the
// exponentials, so one of them an element.  A short row is a warp's, a longer one a CTA's, a longer one
// still a cluster's, whose first CTA joins the parts' sums and best tokens in its shared memory; what
// sixteen CTAs do not hold is cut into parts for a second kernel, in a fixed order too.
//
// The `top` best: a token's key is its logit's bits in the order of the numbers (-0 as 0), then its
// index from behind, so that keys are different and among equal logits the lowest index is the
// larger key.  A lower bound of the key wanted last comes from the lanes' maxima (best).  The elements that
// reach it (few more than `top` where logits are not sorted) go to shared memory, and each one's rank is
// the number of larger keys there.  Where more reach it than there is room for, the best are found one
// after the other.
//
// What bounds it: for many short rows latency, with the few warps that the rows in registers leave room for: 12000 x 1025 bf16 take 10.3 us
// from DRAM (2.4 TB/s), 8.1 from L2, where a third of the warps are active and no unit is a third busy (the loads are the
// main stall); for few long ones the latency of the load, the reductions and the join (64 x 65536 9.7 us from DRAM,
// 8.8 from L2).  Where more elements reach the bound than there is room for, as in rows of which fewer than `top` tokens are
// left, every one of the best is a pass: 64 x 65536 with ten left and twenty asked for 143 us, with all 10.7.

constexpr int MAX_TOP = 32, MAX_CLUSTER = 16;
constexpr int WARP_CANDS = 512, CTA_CANDS = 512;

typedef unsigned long long Key;

struct LogprobParams {
    const void *x;
    long long rows, ld;
    int V, top;
    int parts, per;                       // parts a row, elements a part (a multiple of eight)
    float scale;                          // of the logits
    const void *tokens;
    int tokens64;
    float *logprob, *entropy, *top_logprob;
    int *top_token;
    float *sums;                          // [rows][parts] of PARTS, as Sums
    Key *keys;                            // [rows][parts][top]
};

__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ Key key_of(uint32_t order, int i) {
    return static_cast<Key>(order) << 32 | static_cast<uint32_t>(~i);
}
__device__ __forceinline__ Key key_from(float least) { return static_cast<Key>(order_of(least)) << 32; }
__device__ __forceinline__ int index_of(Key k) { return static_cast<int>(~static_cast<uint32_t>(k)); }

// Where the warps of a CTA leave what they reduce.  Each reduction of a kernel has its own, so that one barrier does.
typedef uint2 *Slot;

// The group of threads that holds a row: a warp or a CTA of 256.
template <int TPR>
struct Group {
    static constexpr int WARPS = TPR / 32;
    static __device__ __forceinline__ void sync() {
        if (WARPS == 1) __syncwarp();
        else __syncthreads();
    }
    // Two sums over the group.
    static __device__ __forceinline__ void sum2(float &a, float &b, Slot red) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (WARPS > 1) {
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_uint2(__float_as_uint(a), __float_as_uint(b));
            __syncthreads();
            a = __uint_as_float(red[0].x), b = __uint_as_float(red[0].y);
#pragma unroll
            for (int i = 1; i < WARPS; ++i) a += __uint_as_float(red[i].x), b += __uint_as_float(red[i].y);
        }
    }
    // The largest of the warps' values, which are a warp's lanes' own already.
    static __device__ __forceinline__ uint2 max2_of_warps(uint2 v, Slot red) {
        if (WARPS > 1) {
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
            __syncthreads();
            v = red[0];
#pragma unroll
            for (int i = 1; i < WARPS; ++i) v.x = max(v.x, red[i].x), v.y = max(v.y, red[i].y);
        }
        return v;
    }
    static __device__ __forceinline__ uint32_t max_u32(uint32_t v, Slot red) {
        return max2_of_warps(make_uint2(__reduce_max_sync(0xffffffffu, v), 0u), red).x;
    }
};

__device__ __forceinline__ Key warp_max_key(Key v) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(v >> 32) == hi ? static_cast<uint32_t>(v) : 0u);
    return static_cast<Key>(hi) << 32 | lo;
}

// The lanes' value of rank `top` (from 1 on; equal ones share the rank of the last), in all lanes.  For few by
// taking the largest away, for more by every lane's rank.
__device__ __forceinline__ uint32_t lane_max_of_rank(uint32_t v, int top) {
    if (top <= 8) {
        uint32_t m = 0;
        for (int left = top; left > 0;) {
            m = __reduce_max_sync(0xffffffffu, v);
            const unsigned lanes = __ballot_sync(0xffffffffu, v == m);
            left -= __popc(lanes);
            if (m == 0) break;
            if (v == m) v = 0;
        }
        return m;
    }
    const int lane = threadIdx.x & 31;
    int rank = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const uint32_t o = __shfl_sync(0xffffffffu, v, i);
        rank += o > v || (o == v && i < lane);
    }
    return __reduce_max_sync(0xffffffffu, rank == top - 1 ? v : 0u);
}

// The `top` largest of a group's keys, in order, to put(rank, key).  each(least, f): f(have, key), by all lanes
// together, for those of the threads' keys whose logit is not below `least`; lane_top: the largest of
// the upper halves of a thread's (0: none).
template <int TPR, int CANDS, typename Each, typename Put>
__device__ __forceinline__ void best(int top, uint32_t lane_top, Each each, Put put, Key *cand, Slot red) {
    using G = Group<TPR>;
    const int lane = threadIdx.x & 31, t = threadIdx.x % TPR;
    uint32_t *count = reinterpret_cast<uint32_t *>(cand);      // the keys from cand[1] on
    if (t == 0) *count = 0;
    // `top` elements reach a warp's lane maximum of rank `top`, or every warp's of rank top / warps
    uint2 lim = make_uint2(top == 1 ? __reduce_max_sync(0xffffffffu, lane_top) : lane_max_of_rank(lane_top, top), 0u);
    if (G::WARPS > 1 && top > 1) lim.y = ~lane_max_of_rank(lane_top, (top - 1) / G::WARPS + 1);
    lim = G::max2_of_warps(lim, red);
    const uint32_t bound = G::WARPS > 1 && top > 1 ? max(lim.x, ~lim.y) : lim.x;
    uint32_t found = 0;
    if (__any_sync(0xffffffffu, lane_top != 0 && lane_top >= bound))
        each(value_of(max(bound, order_of(-INFINITY))), [&](bool have, Key k) {
            const unsigned lanes = __ballot_sync(0xffffffffu, have);
            uint32_t p = found;
            if (G::WARPS > 1) {
                if (lane == 0) p = atomicAdd(count, static_cast<uint32_t>(__popc(lanes)));
                p = __shfl_sync(0xffffffffu, p, 0);
            }
            found += __popc(lanes);
            p += __popc(lanes & ((1u << lane) - 1));
            if (have && p < CANDS) cand[1 + p] = k;
        });
    G::sync();
    if (G::WARPS > 1) found = *count;
    if (found <= CANDS) {
        // up to four a thread at a time
        for (uint32_t p = t; p < found; p += 4 * TPR) {
            Key k[4];
            int r[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = p + i * TPR < found ? cand[1 + p + i * TPR] : ~Key(0);
            if (found <= TPR) {
                for (uint32_t j = 0; j < found; ++j) r[0] += cand[1 + j] > k[0];
            } else {
                for (uint32_t j = 0; j < found; ++j) {
                    const Key o = cand[1 + j];
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] += o > k[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p + i * TPR < found && r[i] < top) put(r[i], k[i]);
        }
        for (int r = static_cast<int>(found) + t; r < top; r += TPR) put(r, Key(0));
    } else {
        Key last = ~Key(0);
        for (int r = 0; r < top; ++r) {
            Key k = 0;
            each(-INFINITY, [&](bool have, Key o) { k = have && o < last && o > k ? o : k; });
            k = warp_max_key(k);
            if (G::WARPS > 1) {
                __syncthreads();
                if (lane == 0) cand[threadIdx.x >> 5] = k;
                __syncthreads();
                for (int i = 0; i < G::WARPS; ++i) k = cand[i] > k ? cand[i] : k;
            }
            if (t == 0) put(r, k);
            last = k;
        }
    }
}

// Sums of a row or a part, u in units of log2.
struct alignas(16) Sums {      // travels between CTAs as one vector
    float m, s, u, unused;
};

// Writes a row's results: write(...) by one thread, put(rank, key) by any.
template <typename T>
struct RowOut {
    const LogprobParams &prm;
    long long row;
    float m, ls;
    bool none;          // no distribution: a NaN or +inf among the logits, or nothing but -inf

    __device__ __forceinline__ RowOut(const LogprobParams &p, long long r, const Sums &v)
        : prm(p), row(r), m(v.m), ls(logf(v.s)),
          none(!(v.m > -INFINITY && v.m < INFINITY) || v.s != v.s) {}
    __device__ __forceinline__ float nan() const { return __uint_as_float(0x7fc00000u); }
    __device__ __forceinline__ float logp(float x) const { return none ? nan() : __fmaf_rn(__fmaf_rn(x, 0.5f, -0.5f * m), 2.0f * prm.scale, -ls); }
    __device__ __forceinline__ void write(const Sums &v) const {
        prm.entropy[row] = none ? nan() : ls - 0.693147181f * (v.u / v.s);
        if (!prm.tokens) return;
        const long long tok = prm.tokens64 ? static_cast<const long long *>(prm.tokens)[row]
                                           : static_cast<long long>(static_cast<const int *>(prm.tokens)[row]);
        float lp = tok < 0 ? 0.0f : nan();
        if (tok >= 0 && tok < prm.V) lp = logp(to_f32(static_cast<const T *>(prm.x)[row * prm.ld + tok]));
        prm.logprob[row] = lp;
    }
    __device__ __forceinline__ void put(int r, Key k) const {
        prm.top_logprob[row * prm.top + r] = logp(value_of(static_cast<uint32_t>(k >> 32)));
        prm.top_token[row * prm.top + r] = none ? -1 : index_of(k);
    }
};

template <typename T>
__device__ __forceinline__ constexpr uint32_t neg_inf() {
    return sizeof(T) == 4 ? 0xff800000u : (std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u);
}

// Two f32 numbers in a register pair: one instruction for both.
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(Two v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }

// Adds the exponentials of two elements, 2^p for p = (x / 2 + minus_half) c, and p 2^p; p = -inf: 0.  The difference
// first, so that an error of p is relative to p and the largest element's is 0.
__device__ __forceinline__ void add_exp(float x0, float x1, Two minus_half, Two c, Two &s, Two &u) {
    Two p = two(x0, x1);
    asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(p) : "l"(two(0.5f, 0.5f)), "l"(minus_half));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(p) : "l"(c));
    float p0, p1, e0, e1;
    split(p, p0, p1);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(p0));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(p1));
    const Two e = two(e0, e1), q = two(fmaxf(p0, -1e30f), fmaxf(p1, -1e30f));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(s) : "l"(e));
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(u) : "l"(e), "l"(q));
}

// log2(e) x 2 scale: what half a difference of logits is multiplied by.
__device__ __forceinline__ float factor(float scale) { return scale * (2.0f * 1.44269504f); }

// Joins parts' sums, the thread's being first, first + step, ...; c: factor(scale).
template <int TPR, typename At>
__device__ __forceinline__ Sums join(int parts, int first, int step, float c, At at, Slot red) {
    using G = Group<TPR>;
    float most = -INFINITY;
    for (int i = first; i < parts; i += step) most = fmaxf(most, at(i).m);
    Sums v{value_of(G::max_u32(order_of(most), red)), 0.0f, 0.0f, 0.0f};
    for (int i = first; i < parts; i += step) {
        const Sums p = at(i);
        if (p.m == -INFINITY) {
            v.s += p.s;      // 0, or NaN
            continue;
        }
        const float d = __fmaf_rn(p.m, 0.5f, -0.5f * v.m) * c;
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d));
        v.s = __fmaf_rn(p.s, e, v.s);
        v.u = __fmaf_rn(__fmaf_rn(p.s, fmaxf(d, -1e30f), p.u), e, v.u);
    }
    G::sum2(v.s, v.u, red + 8);
    return v;
}

enum { WHOLE = 0, CLUSTER = 1, PARTS = 2 };      // what a group holds: a row, a part joined in the cluster, a part joined later

// TPR threads (32: four rows a CTA, or 256) hold a row or a part of one in U units of eight
// elements a thread, the first of them `shift` elements before the row, on 16 bytes, and S more elements a thread behind
// them (a row of a few more than U units hold would take twice as many for its last elements).
template <typename T, int TPR, int U, int S, int HOLDS>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, TPR == 32 ? (U > 4 ? 4 : (U == 4 ? 6 : 8)) : (U > 2 ? 4 : 5)) logprob_kernel(const LogprobParams prm) {
    using G = Group<TPR>;
    constexpr bool PART = HOLDS != WHOLE;
    constexpr int RPC = TPR == 32 ? 4 : 1, CANDS = TPR == 32 ? WARP_CANDS : CTA_CANDS;
    __shared__ Key cands[RPC][CANDS + 1];
    __shared__ uint2 red[HOLDS == CLUSTER ? 48 : 24];      // slots of eight: maximum, sums, bound; those of the join
    __shared__ Sums part_sums[HOLDS == CLUSTER ? MAX_CLUSTER : 1];
    __shared__ Key part_keys[HOLDS == CLUSTER ? MAX_CLUSTER * MAX_TOP : 1];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const long long row = static_cast<long long>(blockIdx.x) * RPC + sub;
    if (row >= prm.rows) return;      // whole warps (TPR = 32), else none
    const int first = PART ? static_cast<int>(blockIdx.y) * prm.per : 0;
    const int n = PART ? max(0, min(prm.per, prm.V - first)) : prm.V;
    const T *x = static_cast<const T *>(prm.x) + row * prm.ld + first;
    const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    Raw8<T> v[U];
    float tail[S + 1];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int c = (i * TPR + t) * 8 - shift;
        if (c >= 0 && c + 8 <= n) {
            v[i].template load<true>(x + c, 8);
        } else {
#pragma unroll
            for (int j = 0; j < Raw8<T>::WORDS; ++j) v[i].w[j] = neg_inf<T>();
            if (c + 8 > 0 && c < n)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j >= 0 && c + j < n) {
                        if constexpr (sizeof(T) == 4) {
                            v[i].w[j] = reinterpret_cast<const uint32_t *>(x)[c + j];
                        } else {
                            const uint32_t b = reinterpret_cast<const uint16_t *>(x)[c + j];
                            v[i].w[j >> 1] = j & 1 ? (v[i].w[j >> 1] & 0xffffu) | (b << 16) : (v[i].w[j >> 1] & 0xffff0000u) | b;
                        }
                    }
        }
    }
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int k = (U * 8 + i) * TPR + t - shift;
        tail[i] = k < n ? to_f32(x[k]) : -INFINITY;
    }
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, v[i].at(j));
#pragma unroll
    for (int i = 0; i < S; ++i) most = fmaxf(most, tail[i]);
    Sums sums{value_of(G::max_u32(order_of(most), red)), 0.0f, 0.0f, 0.0f};
    // nothing but -inf (and NaN): weights of 0, or NaN
    const float from = sums.m == -INFINITY ? 0.0f : sums.m, c = factor(prm.scale);
    const Two minus_half = two(-0.5f * from, -0.5f * from), c2 = two(c, c);
    Two s2 = two(0.0f, 0.0f), u2 = s2;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; j += 2) add_exp(v[i].at(j), v[i].at(j + 1), minus_half, c2, s2, u2);
#pragma unroll
    for (int i = 0; i < S; ++i) add_exp(tail[i], -INFINITY, minus_half, c2, s2, u2);
    float s0, s1, u0, u1;
    split(s2, s0, s1);
    split(u2, u0, u1);
    sums.s = s0 + s1;
    sums.u = u0 + u1;
    G::sum2(sums.s, sums.u, red + 8);
    // the few elements that reach a bound are read again: an index into registers would have every one's code unrolled
    auto each = [&](float least, auto f) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint32_t found = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) found |= v[i].at(j) >= least ? 1u << j : 0u;
            while (__any_sync(0xffffffffu, found != 0)) {
                const int k = (i * TPR + t) * 8 - shift + __ffs(static_cast<int>(found)) - 1;
                const bool have = found != 0 && static_cast<uint32_t>(k) < static_cast<uint32_t>(n);
                found &= found - 1;
                f(have, have ? key_of(order_of(to_f32(x[k])), first + k) : Key(0));
            }
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int k = (U * 8 + i) * TPR + t - shift;
            const bool have = tail[i] >= least && k < n;
            if (__any_sync(0xffffffffu, have)) f(have, key_of(order_of(tail[i]), first + k));
        }
    };
    // a thread without elements has nothing to offer (one whose elements are all -inf does)
    const uint32_t lane_top = t * 8 - shift < n ? order_of(most) : 0u;
    if constexpr (HOLDS == WHOLE) {
        const RowOut<T> out(prm, row, sums);
        if (t == 0) out.write(sums);
        if (prm.top > 0) best<TPR, CANDS>(prm.top, lane_top, each, [&](int r, Key k) { out.put(r, k); }, cands[sub], red + 16);
    } else if constexpr (HOLDS == PARTS) {
        const long long at = row * prm.parts + blockIdx.y;
        if (t == 0) *reinterpret_cast<float4 *>(prm.sums + 4 * at) = make_float4(sums.m, sums.s, sums.u, 0.0f);
        if (prm.top > 0)
            best<TPR, CANDS>(prm.top, lane_top, each, [&](int r, Key k) { prm.keys[at * prm.top + r] = k; }, cands[sub], red + 16);
    } else {
        // to the cluster's first CTA, which is not done before all have been there
        uint32_t to_sums, to_keys;
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to_sums) : "r"(smem_u32(part_sums + blockIdx.y)));
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to_keys) : "r"(smem_u32(part_keys + blockIdx.y * prm.top)));
        // no CTA writes to another one that has not started
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (t == 0)
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to_sums), "f"(sums.m), "f"(sums.s),
                         "f"(sums.u), "f"(0.0f)
                         : "memory");
        if (prm.top > 0)
            best<TPR, CANDS>(prm.top, lane_top, each, [&](int r, Key k) {
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to_keys + 8 * r), "l"(k) : "memory");
            }, cands[sub], red + 16);
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (blockIdx.y != 0) return;
        const Sums all = join<TPR>(prm.parts, t, TPR, c, [&](int i) { return part_sums[i]; }, red + 24);
        const RowOut<T> out(prm, row, all);
        if (t == 0) out.write(all);
        if (prm.top > 0) {
            const int keys = prm.parts * prm.top;
            uint32_t my_top = 0;
            for (int i = t; i < keys; i += TPR) my_top = max(my_top, static_cast<uint32_t>(part_keys[i] >> 32));
            best<TPR, CANDS>(prm.top, my_top, [&](float least, auto f) {
                for (int i = t; i - t < keys; i += TPR) {
                    const Key k = i < keys ? part_keys[i] : Key(0);
                    f(k >= key_from(least), k);
                }
            }, [&](int r, Key k) { out.put(r, k); }, cands[sub], red + 40);
        }
    }
}

// Joins a row's parts, a CTA a row.
template <typename T>
__global__ void __launch_bounds__(256) logprob_join_kernel(const LogprobParams prm) {
    __shared__ Key cands[CTA_CANDS + 1];
    __shared__ uint2 red[24];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const long long row = blockIdx.x;
    const float4 *parts = reinterpret_cast<const float4 *>(prm.sums) + row * prm.parts;
    const Sums all = join<256>(prm.parts, t, 256, factor(prm.scale), [&](int i) {
        const float4 p = parts[i];
        return Sums{p.x, p.y, p.z, p.w};
    }, red);
    const RowOut<T> out(prm, row, all);
    if (t == 0) out.write(all);
    if (prm.top > 0) {
        const Key *keys = prm.keys + row * prm.parts * prm.top;
        const int n = prm.parts * prm.top;
        uint32_t lane_top = 0;
        for (int i = t; i < n; i += 256) lane_top = max(lane_top, static_cast<uint32_t>(keys[i] >> 32));
        auto each = [&](float least, auto f) {
            for (int i = t; i - t < n; i += 256) {
                const Key k = i < n ? keys[i] : Key(0);
                f(k >= key_from(least), k);
            }
        };
        best<256, CTA_CANDS>(prm.top, lane_top, each, [&](int r, Key k) { out.put(r, k); }, cands, red + 16);
    }
}

}  // namespace ipl
