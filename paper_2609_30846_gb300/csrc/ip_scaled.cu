// Host side of the operators with run-time scales of the C ABI (include/ip_mhsa.h):
// argument validation, tensor maps and launches.  Device code: ip_scaled_kernels.cuh.
#include "ip_mhsa.h"
#include "ip_scaled_kernels.cuh"
#include "ip_host_util.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                  const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                             cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// int8 rows [rows][K] of `ld` bytes each, boxes of BK x box_rows, elements outside read
// as zero (a K that BK does not divide, the rows behind the last).
bool make_map(CUtensorMap *m, const void *base, int K, long long rows, long long ld, unsigned box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld)};
    const cuuint32_t box[2] = {ips::BK, box_rows};
    const cuuint32_t estride[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estride,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

std::mutex g_mu;
int g_sms[64] = {0};

int sm_count() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    std::lock_guard<std::mutex> lock(g_mu);
    if (g_sms[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        g_sms[dev] = n;
    }
    return g_sms[dev];
}

size_t elem_size(int dtype) { return dtype == IP_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == IP_F32 || dtype == IP_F16 || dtype == IP_BF16; }

int launched(cudaError_t rc) {
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? IP_OK : IP_ERR_CUDA;
}

template <typename T, bool VEC>
int quantize(const ips::QuantParams &prm, cudaStream_t st) {
    // a warp a row while its lanes can hold the row, then four warps, then the CTA
    const int tpr = prm.d <= 32 * 8 * ips::QUANT_UNITS ? 32 : (prm.d <= 128 * 8 * ips::QUANT_UNITS ? 128 : 256);
    const int rpc = ips::QUANT_THREADS / tpr;
    const long long need = (prm.rows + rpc - 1) / rpc, cap = 1ll << 20;
    const dim3 grid(static_cast<unsigned>(need < cap ? need : cap)), block(ips::QUANT_THREADS);
    switch (tpr) {
        case 32: return launched(iph::launch_pdl(ips::quantize_rows_kernel<T, 32, VEC>, grid, block, 0, st, prm));
        case 128: return launched(iph::launch_pdl(ips::quantize_rows_kernel<T, 128, VEC>, grid, block, 0, st, prm));
        default: return launched(iph::launch_pdl(ips::quantize_rows_kernel<T, 256, VEC>, grid, block, 0, st, prm));
    }
}

template <typename T>
int quantize(const ips::QuantParams &prm, cudaStream_t st) {
    const bool vec = prm.d % 8 == 0 && aligned(prm.x, 16) && aligned(prm.q, 8) &&
                     (prm.rows == 1 || (prm.ldx * sizeof(T) % 16 == 0 && prm.ldq % 8 == 0));
    return vec ? quantize<T, true>(prm, st) : quantize<T, false>(prm, st);
}

template <typename T, int MT, int CPT, int KT>
int launch_vec(const ips::ScaledParams &prm, int nsm, cudaStream_t st) {
    constexpr int per = ips::VEC_THREADS / KT * CPT;
    const long long blocks = (prm.N + per - 1) / per, most = 4ll * nsm;
    const dim3 grid(static_cast<unsigned>(blocks < most ? blocks : most),
                    static_cast<unsigned>((prm.M + MT - 1) / MT)), block(ips::VEC_THREADS);
    if (prm.K <= KT * 16)
        return launched(iph::launch_pdl(ips::scaled_vec_kernel<T, MT, CPT, KT, true>, grid, block, 0, st, prm));
    return launched(iph::launch_pdl(ips::scaled_vec_kernel<T, MT, CPT, KT, false>, grid, block, 0, st, prm));
}

// Four channels a thread where every SM still gets one and a half CTAs, else one.
bool vec_four(int K, int N, int nsm) { return N >= nsm * (K > 2048 ? 6 : 24); }

template <typename T, int MT>
int launch_vec_m(const ips::ScaledParams &prm, int nsm, cudaStream_t st) {
    const bool four = vec_four(prm.K, prm.N, nsm);
    if (prm.K > 2048) return four ? launch_vec<T, MT, 4, 256>(prm, nsm, st) : launch_vec<T, MT, 1, 256>(prm, nsm, st);
    return four ? launch_vec<T, MT, 4, 64>(prm, nsm, st) : launch_vec<T, MT, 1, 64>(prm, nsm, st);
}

bool odd_rows(const ips::ScaledParams &prm, size_t es) {
    return ((reinterpret_cast<uintptr_t>(prm.y) | (static_cast<size_t>(prm.ldy) * es)) & 7) != 0;
}

template <typename T, int BN, bool LONG, bool PAIR, bool KSPLIT = false, bool ODD = false>
int launch_tc(const CUtensorMap &tx, const CUtensorMap &tw, const ips::ScaledParams &prm, int nsm,
              cudaStream_t st) {
    using C = ips::Tile<BN, PAIR>;
    static bool set[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IP_ERR_CUDA;
    auto *fn = ips::scaled_tc_kernel<T, BN, LONG, PAIR, KSPLIT, ODD>;
    {
        std::lock_guard<std::mutex> lock(g_mu);
        if (!set[dev]) {
            // the kernel deals out TC_REGS registers a thread: never launch a build with fewer
            cudaFuncAttributes attr;
            if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess ||
                cudaFuncGetAttributes(&attr, fn) != cudaSuccess ||
                (LONG && BN == 256 && attr.numRegs < ips::TC_REGS))
                return IP_ERR_CUDA;
            set[dev] = true;
        }
    }
    // parts of a tile do not loop over tiles
    const int ctas = KSPLIT ? prm.splits : C::CTAS;
    const long long most = KSPLIT ? prm.tiles : nsm / ctas, workers = prm.tiles < most ? prm.tiles : most;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(workers * ctas));
    cfg.blockDim = dim3(ips::TC_THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    return launched(cudaLaunchKernelEx(&cfg, fn, tx, tw, prm));
}

template <typename T, int BN, bool LONG, bool PAIR>
int launch_rows(const CUtensorMap &tx, const CUtensorMap &tw, const ips::ScaledParams &prm, int nsm, cudaStream_t st) {
    return odd_rows(prm, sizeof(T)) || prm.N % 16 != 0 ? launch_tc<T, BN, LONG, PAIR, false, true>(tx, tw, prm, nsm, st)
                                                       : launch_tc<T, BN, LONG, PAIR>(tx, tw, prm, nsm, st);
}

template <typename T, int BN, bool PAIR>
int run_tc(ips::ScaledParams prm, int nsm, cudaStream_t st) {
    using C = ips::Tile<BN, PAIR>;
    CUtensorMap tx, tw;
    if (!make_map(&tx, prm.x, prm.K, prm.M, prm.ldx, ips::TILE_M) ||
        !make_map(&tw, prm.w, prm.K, prm.N, prm.ldw, C::BR))
        return IP_ERR_CUDA;
    prm.tiles_n = (prm.N + BN - 1) / BN;
    prm.tiles = (prm.M + ips::TILE_M * C::CTAS - 1) / (ips::TILE_M * C::CTAS) * prm.tiles_n;
    if constexpr (BN == 32) {
        const int stages = (prm.K + ips::BK - 1) / ips::BK;
        if (prm.splits > 1)
            return (stages + prm.splits - 1) / prm.splits > ips::SEG
                       ? launch_tc<T, BN, true, PAIR, true>(tx, tw, prm, nsm, st)
                       : launch_tc<T, BN, false, PAIR, true>(tx, tw, prm, nsm, st);
    }
    if (prm.K > ips::SEG * ips::BK) return launch_rows<T, BN, true, PAIR>(tx, tw, prm, nsm, st);
    return launch_rows<T, BN, false, PAIR>(tx, tw, prm, nsm, st);
}

// The form that a launch is expected to take the least time in, ns.  Fitted on GB300 to sweeps of
// M = 16 .. 4096 tokens over N = 512 .. 16384 at K = 1024 and 4096, every form timed at each point
// (beyond these K and N it is extrapolated, but for the vector kernel's rate, taken at K = 9000 too):
// the vector kernel reads the weights once per eight tokens; the tensor-core forms take so
// long per fp16 stage (64 of K) of a round of tiles over the SMs.  (us, vector / 32 / 128 / pairs:
// 32 x 1024 -> 512 3.0 / 7.0 / 7.8 / 12.0, 128 x 1024 -> 1024 12.5 / 7.1 / 8.3 / 12.9, 32 x 4096 -> 4096
// 18.5 / 19.6 / 23.1 / 34.6, 32 x 4096 -> 16384 - / 70.6 / 23.8 / 35.9, 2048 x 1024 -> 16384 - / - / 86 / 69.)
enum Form { FORM_VEC, FORM_32, FORM_128, FORM_PAIR };
struct Choice {
    Form form;
    int splits;
};

long long rounds(long long tiles, int workers) { return (tiles + workers - 1) / workers; }

Choice choose(const ips::ScaledParams &prm, size_t es, int nsm) {
    const long long stages = (prm.K + ips::BK - 1) / ips::BK;
    const long long tm = (prm.M + ips::TILE_M - 1) / ips::TILE_M;
    const long long t32 = tm * ((prm.N + 31) / 32), t128 = tm * ((prm.N + 127) / 128);
    const long long pairs = (tm + 1) / 2 * ((prm.N + 255) / 256);
    // output rows that are not aligned to 8 bytes are turned in shared memory first: so long for each
    // of a warp's columns, half the tile's
    const long long odd = odd_rows(prm, es) ? 45 : 0;
    Choice best = {FORM_32, 1};
    long long least = 3400 + (265 * stages + 16 * odd) * rounds(t32, nsm);
    // few tiles: up to four parts of K that fit the SMs at once (512 x 1024 -> 512: one part 7.1 us, two
    // 8.4; 128 x 4096 -> 512: one 19.8, four 9.5; eight are slower, 12 x 4096 -> 512 13.5 us for 10)
    for (int splits = 2; splits <= 4 && splits * t32 <= nsm && splits <= stages; splits *= 2) {
        const long long ns = 5800 + 265 * ((stages + splits - 1) / splits);
        if (ns < least) best = {FORM_32, splits}, least = ns;
    }
    const long long ns128 = 3800 + (305 * stages + 64 * odd) * rounds(t128, nsm);
    if (ns128 < least) best = {FORM_128, 1}, least = ns128;
    const long long ns_pair = 5700 + (475 * stages + 128 * odd) * rounds(pairs, nsm / 2);
    if (ns_pair < least) best = {FORM_PAIR, 1}, least = ns_pair;
    const long long blocks = (prm.M + 7) / 8, kv = prm.K > 1024 ? prm.K : 1024;     // a channel's reduction
    const long long rate = vec_four(prm.K, prm.N, nsm) ? (prm.K > 4096 ? 57 : (prm.K > 2048 ? 26 : 31)) : 63;
    if (blocks <= 65535 && 1900 + rate * (prm.N * kv * blocks) / 100000 < least) best = {FORM_VEC, 1};
    return best;
}

template <typename T>
int run_scaled(ips::ScaledParams prm, int nsm, cudaStream_t st) {
    const Choice c = choose(prm, sizeof(T), nsm);
    prm.splits = c.splits;
    switch (c.form) {
        case FORM_VEC:
            if (prm.M == 1) return launch_vec_m<T, 1>(prm, nsm, st);
            if (prm.M == 2) return launch_vec_m<T, 2>(prm, nsm, st);
            if (prm.M <= 4) return launch_vec_m<T, 4>(prm, nsm, st);
            return launch_vec_m<T, 8>(prm, nsm, st);
        case FORM_32: return run_tc<T, 32, false>(prm, nsm, st);
        case FORM_128: return run_tc<T, 128, false>(prm, nsm, st);
        default: return run_tc<T, 256, true>(prm, nsm, st);
    }
}

}  // namespace

extern "C" {

int ip_quantize_rows_i8(const void *x, int dtype, long long rows, int d, long long ldx, int8_t *q,
                        long long ldq, float *scale, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (rows < 0 || rows > IP_NORM_MAX_ROWS || d < 1 || d > IP_LINEAR_MAX_K) return IP_ERR_SHAPE;
    if (ldx < d || ldq < d) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!x || !q || !scale) return IP_ERR_NULL;
    if (!aligned(x, elem_size(dtype)) || !aligned(scale, 4)) return IP_ERR_ALIGN;
    const ips::QuantParams prm{x, rows, ldx, ldq, d, q, scale};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return quantize<float>(prm, st);
    if (dtype == IP_F16) return quantize<__half>(prm, st);
    return quantize<__nv_bfloat16>(prm, st);
}

int ip_linear_scaled_i8(const int8_t *x, long long ldx, const float *sx, const int8_t *w,
                        long long ldw, const float *sw, const float *bias, int act, long long rows,
                        int K, int N, void *y, long long ldy, int dtype, void *workspace,
                        size_t workspace_bytes, ip_stream_t stream) {
    if (!dtype_ok(dtype) || (act != IP_ACT_NONE && act != IP_ACT_SWISH)) return IP_ERR_PARAM;
    if (rows < 0 || rows > IP_LINEAR_MAX_FRAMES || K < 1 || K > IP_LINEAR_MAX_K || N < 1 ||
        N > IP_LINEAR_MAX_N || ldx < K || ldw < K || ldy < N || ldx > (1ll << 40) || ldw > (1ll << 40) ||
        ldy > (1ll << 31))
        return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!x || !sx || !w || !sw || !y || !workspace) return IP_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || ldx % 16 != 0 || ldw % 16 != 0 || !aligned(sx, 4) ||
        !aligned(sw, 4) || (bias && !aligned(bias, 4)) || !aligned(y, elem_size(dtype)) ||
        !aligned(workspace, 256))
        return IP_ERR_ALIGN;
    if (workspace_bytes < 256) return IP_ERR_WORKSPACE;
    const int nsm = sm_count();
    if (nsm <= 0) return IP_ERR_CUDA;
    ips::ScaledParams prm;
    prm.x = x;
    prm.w = w;
    prm.sx = sx;
    prm.sw = sw;
    prm.bias = bias;
    prm.y = y;
    prm.M = rows;
    prm.ldx = ldx;
    prm.ldw = ldw;
    prm.ldy = ldy;
    prm.K = K;
    prm.N = N;
    prm.act = act;
    prm.splits = 1;
    prm.tiles_n = 0;
    prm.tiles = 0;
    prm.err = static_cast<int *>(workspace);
    prm.timeout_cycles = iph::wait_limit();
    prm.stall = iph::stall_injection();
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return run_scaled<float>(prm, nsm, st);
    if (dtype == IP_F16) return run_scaled<__half>(prm, nsm, st);
    return run_scaled<__nv_bfloat16>(prm, nsm, st);
}

}  // extern "C"
