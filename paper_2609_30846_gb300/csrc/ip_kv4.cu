// Host side of the 4-bit key/value cache of the C ABI (include/ip_mhsa.h): argument
// validation, the split of the attention and the launches.  Device code:
// ip_kv4_kernels.cuh.
#include "ip_mhsa.h"
#include "ip_kv4_kernels.cuh"
#include "ip_host_util.h"

#include <cuda_runtime.h>

#include <mutex>

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t elem_size(int dtype) { return dtype == IP_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == IP_F32 || dtype == IP_F16 || dtype == IP_BF16; }
bool page_ok(int page) { return page == 16 || page == 32 || page == 64; }

int launched(cudaError_t rc) {
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? IP_OK : IP_ERR_CUDA;
}

// What the calls on a cache share: IP_OK if its description is sound.
int check_cache(const int32_t *page_table, int max_pages, const void *cache, int n_pages, int page, int H,
                int dh, const void *workspace, size_t workspace_bytes, size_t need) {
    if (dh != IP_DH || !page_ok(page)) return IP_ERR_UNSUPPORTED;
    if (H < 1 || H > IP_MAX_H || max_pages < 1 || n_pages < 0 ||
        static_cast<long long>(max_pages) * page > IP_KV4_MAX_LEN)
        return IP_ERR_SHAPE;
    if (!page_table || !cache || !workspace) return IP_ERR_NULL;
    if (!aligned(page_table, 4) || !aligned(cache, 16) || !aligned(workspace, 256)) return IP_ERR_ALIGN;
    return workspace_bytes < need ? IP_ERR_WORKSPACE : IP_OK;
}

ipv::Pages pages_of(const int32_t *page_table, int max_pages, const void *cache, int n_pages, int page, int H) {
    ipv::Pages p;
    p.cache = static_cast<uint8_t *>(const_cast<void *>(cache));
    p.table = page_table;
    p.max_pages = max_pages;
    p.n_pages = n_pages;
    p.shift = page == 16 ? 4 : (page == 32 ? 5 : 6);
    p.heads = H;
    return p;
}

// Element strides of batch, token and head: any that keep an offset within 63 bits.
bool strides_ok(const long long *s) {
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] > (1ll << 40)) return false;
    return true;
}

// Two rows to a warp where one each would be more warps than the GPU holds at a time (6000
// tokens of 8 heads: append 13.5 us for 15.1; four: 13.1, but in 32 bits 18.4 for 15.8).
constexpr long long WAVE_ROWS = 152 * 64;
template <typename F>
int launch_rows(F *one, F *two, const ipv::RowParams &prm, long long rows, cudaStream_t st) {
    const bool pairs = rows * prm.B > WAVE_ROWS;
    const int per = ipv::ROW_THREADS / 32 * (pairs ? 2 : 1);
    const dim3 grid(static_cast<unsigned>((rows + per - 1) / per), static_cast<unsigned>(prm.B)), block(ipv::ROW_THREADS);
    return launched(iph::launch_pdl(pairs ? two : one, grid, block, 0, st, prm));
}
template <typename T>
int launch_append(const ipv::RowParams &prm, long long rows, cudaStream_t st) {
    return launch_rows(ipv::kv4_append_kernel<T, 1>, ipv::kv4_append_kernel<T, 2>, prm, rows, st);
}
template <typename T>
int launch_read(const ipv::RowParams &prm, long long rows, cudaStream_t st) {
    return launch_rows(ipv::kv4_read_kernel<T, 1>, ipv::kv4_read_kernel<T, 2>, prm, rows, st);
}

// How the attention deals its work: one wave of CTAs (as many as fit on 152 SMs) in equal
// shares, or a CTA per item where an item is short, so that the second launch and the search
// for the share would cost more than they give (us, CTA per item / shares; 1 sequence, 8 heads:
// 384 tokens 6.4 / 8.3, 768 8.8 / 8.5, 2048 17 / 9.1; 64 sequences: 384 16 / 20, 768 27 / 29,
// 2048 52 / 49), or where there are too many row tiles or units to sum up.  The plan depends on
// the call's sizes alone.  SMS is the whole GPU's, whatever part of it a process has: on fewer SMs the
// CTAs take turns, none waits for another.
constexpr int WHOLE_UNITS = 5;
constexpr long long SMS = 152;
struct Plan {
    int nt, tiles;
    bool split;
    long long ctas;
    size_t open_bytes, bytes;
};
bool plan_of(int B, int T, int H, int Hkv, int max_len, Plan *p) {
    const long long rows = static_cast<long long>(H / Hkv) * T;
    p->nt = rows > 8 ? 2 : 1;
    p->tiles = static_cast<int>((rows + 8 * p->nt - 1) / (8 * p->nt));
    const long long tiles = static_cast<long long>(B) * p->tiles, items = tiles * Hkv;
    const long long units = max_len < ipv::UNIT ? 1 : (max_len + ipv::UNIT - 1ll) / ipv::UNIT;
    if (items > 0x7fffffffll) return false;      // a grid's width
    // sums of units stay within 31 bits, rounded up to whole shares too
    p->split = tiles <= ipv::MAX_SCAN && units > WHOLE_UNITS && items * (units + ipv::OVER) <= 0x7ffff000ll;
    p->ctas = items;
    p->open_bytes = 0;
    p->bytes = 256;
    if (p->split) {
        const long long wave = SMS * (p->nt == 1 ? ipv::CTAS_8 : ipv::CTAS_16);
        p->ctas = items * units < wave ? items * units : wave;
        p->open_bytes = (static_cast<size_t>(p->ctas) * sizeof(int2) + 255) / 256 * 256;
        p->bytes += p->open_bytes + static_cast<size_t>(p->ctas) * 2 * 8 * p->nt * ipv::PART * sizeof(float);
    }
    return true;
}

bool attention_shape_ok(int B, int T, int H, int Hkv, int max_len) {
    return B >= 0 && B <= IP_MAX_B && T >= 1 && T <= IP_MAX_T && H >= 1 && H <= IP_MAX_H && Hkv >= 1 &&
           H % Hkv == 0 && max_len >= 0 && max_len <= IP_KV4_MAX_LEN;
}

std::mutex g_mu;

template <typename T, int NT, int PAGE>
int launch_pages(const ipv::AttParams &prm, const Plan &p, cudaStream_t st) {
    static bool set[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IP_ERR_CUDA;
    auto *fn = ipv::kv4_attention_kernel<T, NT, PAGE>;
    constexpr int smem = ipv::smem_bytes(8 * NT);
    {
        std::lock_guard<std::mutex> lock(g_mu);
        if (!set[dev]) {
            if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
                return IP_ERR_CUDA;
            set[dev] = true;
        }
    }
    return launched(iph::launch_pdl(fn, dim3(static_cast<unsigned>(p.ctas)), dim3(ipv::ATT_THREADS), smem, st, prm));
}

template <typename T, int NT>
int launch_attention(const ipv::AttParams &prm, const Plan &p, cudaStream_t st) {
    const int rc = prm.pages.shift == 4 ? launch_pages<T, NT, 16>(prm, p, st)
                                        : (prm.pages.shift == 5 ? launch_pages<T, NT, 32>(prm, p, st)
                                                                : launch_pages<T, NT, 64>(prm, p, st));
    if (rc != IP_OK || !p.split) return rc;
    const int r = prm.G * prm.T < 8 * NT ? prm.G * prm.T : 8 * NT;      // rows that an item can have
    const dim3 rows(static_cast<unsigned>(p.ctas), static_cast<unsigned>(r));
    return launched(iph::launch_pdl(ipv::kv4_join_kernel<T, NT>, rows, dim3(ipv::ATT_THREADS), 0, st, prm));
}

}  // namespace

extern "C" {

size_t ip_kv4_page_bytes(int page, int dh) {
    return dh == IP_DH && page_ok(page) ? static_cast<size_t>(ipv::ROW_BYTES) * page : 0;
}

int ip_kv4_append(const void *k, const void *v, int dtype, const long long *k_strides,
                  const long long *v_strides, const int32_t *start, const int32_t *count, int B, int T, int H,
                  int dh, const int32_t *page_table, int max_pages, void *cache, int n_pages, int page,
                  void *workspace, size_t workspace_bytes, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (B < 0 || B > IP_MAX_B || T < 0 || static_cast<long long>(B) * T > IP_LINEAR_MAX_FRAMES) return IP_ERR_SHAPE;
    if (B == 0 || T == 0) return IP_OK;
    const int rc = check_cache(page_table, max_pages, cache, n_pages, page, H, dh, workspace, workspace_bytes, 256);
    if (rc != IP_OK) return rc;
    if (!k || !v || !k_strides || !v_strides || !start) return IP_ERR_NULL;
    if (!aligned(k, elem_size(dtype)) || !aligned(v, elem_size(dtype)) || !aligned(start, 4) ||
        (count && !aligned(count, 4)))
        return IP_ERR_ALIGN;
    if (!strides_ok(k_strides) || !strides_ok(v_strides)) return IP_ERR_SHAPE;
    const long long rows = static_cast<long long>(T) * H;      // of a sequence, a warp each
    if (rows > 0x7fffffffll) return IP_ERR_SHAPE;
    ipv::RowParams prm{};
    prm.k = k;
    prm.v = v;
    for (int i = 0; i < 3; ++i) prm.ks[i] = k_strides[i], prm.vs[i] = v_strides[i];
    prm.start = start;
    prm.count = count;
    prm.B = B;
    prm.T = T;
    prm.H = H;
    prm.pages = pages_of(page_table, max_pages, cache, n_pages, page, H);
    prm.err = static_cast<int *>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return launch_append<float>(prm, rows, st);
    if (dtype == IP_F16) return launch_append<__half>(prm, rows, st);
    return launch_append<__nv_bfloat16>(prm, rows, st);
}

int ip_kv4_read(const void *cache, int n_pages, int page, const int32_t *page_table, int max_pages,
                const int32_t *start, const int32_t *count, int B, int T, int H, int dh, void *k, void *v,
                int dtype, void *workspace, size_t workspace_bytes, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (B < 0 || B > IP_MAX_B || T < 0 || static_cast<long long>(B) * T > IP_LINEAR_MAX_FRAMES) return IP_ERR_SHAPE;
    if (B == 0 || T == 0) return IP_OK;
    const int rc = check_cache(page_table, max_pages, cache, n_pages, page, H, dh, workspace, workspace_bytes, 256);
    if (rc != IP_OK) return rc;
    if (!k || !v || !start) return IP_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(start, 4) || (count && !aligned(count, 4)))
        return IP_ERR_ALIGN;
    const long long rows = static_cast<long long>(T) * H;      // of a sequence, a warp each
    if (rows > 0x7fffffffll) return IP_ERR_SHAPE;
    ipv::RowParams prm{};
    prm.ko = k;
    prm.vo = v;
    prm.start = start;
    prm.count = count;
    prm.B = B;
    prm.T = T;
    prm.H = H;
    prm.pages = pages_of(page_table, max_pages, cache, n_pages, page, H);
    prm.err = static_cast<int *>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return launch_read<float>(prm, rows, st);
    if (dtype == IP_F16) return launch_read<__half>(prm, rows, st);
    return launch_read<__nv_bfloat16>(prm, rows, st);
}

size_t ip_kv4_attention_workspace_bytes(int B, int T, int H, int Hkv, int max_len) {
    Plan p;
    if (!attention_shape_ok(B, T, H, Hkv, max_len) || !plan_of(B, T, H, Hkv, max_len, &p)) return 0;
    return p.bytes;
}

int ip_kv4_attention(const void *q, int dtype, const long long *q_strides, const int32_t *lengths,
                     const int32_t *count, int causal, float scale, int B, int T, int H, int Hkv, int dh,
                     int max_len, const int32_t *page_table, int max_pages, const void *cache, int n_pages,
                     int page, void *out, void *workspace, size_t workspace_bytes, ip_stream_t stream) {
    if (dtype != IP_F16 && dtype != IP_BF16) return IP_ERR_PARAM;
    if ((causal != 0 && causal != 1) || !(scale > 0.0f && scale < 1e30f)) return IP_ERR_PARAM;
    Plan p;
    if (!attention_shape_ok(B, T, H, Hkv, max_len) || !plan_of(B, T, H, Hkv, max_len, &p)) return IP_ERR_SHAPE;
    if (B == 0) return IP_OK;
    const int rc = check_cache(page_table, max_pages, cache, n_pages, page, Hkv, dh, workspace, workspace_bytes,
                               p.bytes);
    if (rc != IP_OK) return rc;
    if (!q || !q_strides || !lengths || !out) return IP_ERR_NULL;
    if (!aligned(q, 2) || !aligned(out, 16) || !aligned(lengths, 4) || (count && !aligned(count, 4)))
        return IP_ERR_ALIGN;
    if (!strides_ok(q_strides)) return IP_ERR_SHAPE;
    ipv::AttParams prm{};
    prm.q = q;
    prm.out = out;
    for (int i = 0; i < 3; ++i) prm.qs[i] = q_strides[i];
    prm.lengths = lengths;
    prm.count = count;
    prm.B = B;
    prm.T = T;
    prm.H = Hkv;
    prm.G = H / Hkv;
    prm.causal = causal;
    prm.max_len = max_len < max_pages * page ? max_len : max_pages * page;
    prm.tiles = p.tiles;
    prm.split = p.split ? 1 : 0;
    prm.scale_log2 = scale * 1.44269504088896f;
    prm.pages = pages_of(page_table, max_pages, cache, n_pages, page, Hkv);
    prm.open = reinterpret_cast<int2 *>(static_cast<char *>(workspace) + 256);
    prm.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + 256 + p.open_bytes);
    prm.err = static_cast<int *>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F16)
        return p.nt == 1 ? launch_attention<__half, 1>(prm, p, st) : launch_attention<__half, 2>(prm, p, st);
    return p.nt == 1 ? launch_attention<__nv_bfloat16, 1>(prm, p, st)
                     : launch_attention<__nv_bfloat16, 2>(prm, p, st);
}

}  // extern "C"
