// Host side of the product of 4-bit rows of the C ABI (include/ip_mhsa.h): argument validation,
// tensor maps and launches.  Device code: ip_fp4_kernels.cuh.
#include "ip_mhsa.h"
#include "ip_fp4_kernels.cuh"
#include "ip_host_util.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
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

// Rows of `bytes` bytes of codes, `ld` apart, boxes of 128 x box_rows in the 128-byte swizzled
// layout; what lies outside reads as zero (a K that 256 does not divide, the rows behind the last).
bool make_map(CUtensorMap *m, const void *base, int bytes, long long rows, long long ld, unsigned box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(bytes), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld)};
    const cuuint32_t box[2] = {ip4::BKB, box_rows};
    const cuuint32_t estride[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estride,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Block scales of `rows` rows as [rows / 128][steps of 64 elements][512 bytes], boxes of four steps of
// `tiles` times 128 rows; what lies outside reads as zero.
bool make_scale_map(CUtensorMap *m, const void *base, int steps, long long rows, unsigned tiles) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(steps), static_cast<cuuint64_t>((rows + 127) / 128)};
    const cuuint64_t strides[2] = {512, static_cast<cuuint64_t>(steps) * 512};
    const cuuint32_t box[3] = {128, 4, tiles};
    const cuuint32_t estride[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void *>(base), dims, strides, box, estride,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The output's rows, boxes of `columns` x 32 rows in the swizzled layout of their width (64 or 32 bytes).
bool make_out_map(CUtensorMap *m, void *y, CUtensorMapDataType type, int es, int columns, int N, long long rows, long long ld) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(N), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * es};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(columns), 32};
    const cuuint32_t estride[2] = {1, 1};
    return fn(m, type, 2, y, dims, strides, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE, columns * es == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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

int launched(cudaError_t rc) {
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? IP_OK : IP_ERR_CUDA;
}

struct Operands {
    const uint8_t *x, *w, *xb, *wb;
    long long ldx, ldw;
    int bytes;            // of a row's codes
};

template <typename T, int BN, bool PAIR, bool ODD, int PARTS = 1>
int launch(const CUtensorMap (&maps)[5], const ip4::Params &prm, int nsm, cudaStream_t st) {
    using C = ip4::Tile<BN, PAIR>;
    static bool set[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IP_ERR_CUDA;
    auto *fn = ip4::fp4_kernel<T, BN, PAIR, ODD, PARTS>;
    {
        std::lock_guard<std::mutex> lock(g_mu);
        if (!set[dev]) {
            // the kernel deals out REGS registers a thread: never launch a build with fewer
            cudaFuncAttributes attr;
            if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess ||
                cudaFuncGetAttributes(&attr, fn) != cudaSuccess || (BN == 256 && attr.numRegs < ip4::REGS))
                return IP_ERR_CUDA;
            set[dev] = true;
        }
    }
    const long long most = PARTS > 1 ? prm.tiles : nsm / C::CTAS, workers = prm.tiles < most ? prm.tiles : most;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(workers * C::CTAS * PARTS));
    cfg.blockDim = dim3(ip4::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = C::CTAS * PARTS;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR || PARTS > 1 ? 2 : 1;
    return launched(cudaLaunchKernelEx(&cfg, fn, maps[0], maps[1], maps[2], maps[3], maps[4], prm));
}

template <typename T, int BN, bool PAIR, int PARTS = 1>
int run(const Operands &o, ip4::Params prm, int nsm, cudaStream_t st) {
    using C = ip4::Tile<BN, PAIR>;
    CUtensorMap maps[5];
    if (!make_map(&maps[0], o.x, o.bytes, prm.M, o.ldx, ip4::TILE_M) || !make_map(&maps[1], o.w, o.bytes, prm.N, o.ldw, C::BR) ||
        !make_scale_map(&maps[2], o.xb, prm.steps, prm.M, 1) || !make_scale_map(&maps[3], o.wb, prm.steps, prm.N, C::WT))
        return IP_ERR_CUDA;
    prm.tiles_n = (prm.N + BN - 1) / BN;
    prm.tiles = (prm.M + ip4::TILE_M * C::CTAS - 1) / (ip4::TILE_M * C::CTAS) * prm.tiles_n;
    if constexpr (PARTS > 1) {
        maps[4] = maps[0];      // not used
        return launch<T, BN, PAIR, true, PARTS>(maps, prm, nsm, st);
    }
    constexpr int es = static_cast<int>(sizeof(T));
    const bool odd = !aligned(prm.y, 16) || prm.ldy * es % 16 != 0 || prm.N * es % 16 != 0;
    constexpr CUtensorMapDataType type = es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    if (odd) maps[4] = maps[0];      // not used
    else if (!make_out_map(&maps[4], prm.y, type, es, ip4::block_columns<T, BN>(), prm.N, prm.M, prm.ldy)) return IP_ERR_CUDA;
    return odd ? launch<T, BN, PAIR, true>(maps, prm, nsm, st) : launch<T, BN, PAIR, false>(maps, prm, nsm, st);
}

long long rounds(long long tiles, int workers) { return (tiles + workers - 1) / workers; }

// The times, ns, that the forms of tiles are expected to take: a start, and for each round of tiles over the
// SMs the stages (all forms are held up by shared memory, which serves the MMAs, the copies in and the
// scales) with what does not overlap of the hand-over to the output warps, or their time where K is short.
// t64s: tiles of 64 channels whose K four CTAs share (125 x 4096 -> 1024 6.2 us, by whole tiles 8.0; x 1024 -> 1024 5.1 and 4.1).
struct Times {
    long long t64, t128, pair, t64s;
    long long least() const { return std::min(std::min(t64, t128), std::min(pair, t64s)); }
};
Times tile_times(long long M, int N, int steps, int nsm) {
    const long long stages = (steps + 3) / 4, tm = (M + ip4::TILE_M - 1) / ip4::TILE_M;
    auto time = [&](long long start, long long tiles, int workers, long long stage, long long over, long long out) {
        const long long tile = stage * stages + over;
        return start + rounds(tiles, workers) * (tile > out ? tile : out);
    };
    const long long t64 = tm * ((N + 63) / 64), share = (stages + 3) / 4;
    // one tile a cluster, all clusters at once (of 152 SMs 32 find room, 38 take two rounds), and each part has stages
    const bool shared = t64 * 4 <= nsm * 27 / 32 && 3 * share < stages;
    return {time(3300, t64, nsm, 340, 300, 930), time(3700, tm * ((N + 127) / 128), nsm, 340, 360, 1200),
            time(5100, (tm + 1) / 2 * ((N + 255) / 256), nsm / 2, 385, 1200, 2050),
            shared ? 5500 + 340 * share : LLONG_MAX};
}

template <typename T>
int run(const Operands &o, const ip4::Params &prm, const Times &t, int nsm, cudaStream_t st) {
    if (t.t64s == t.least()) return run<T, 64, false, 4>(o, prm, nsm, st);
    if (t.pair < t.t64 && t.pair < t.t128) return run<T, 256, true>(o, prm, nsm, st);
    return t.t128 < t.t64 ? run<T, 128, false>(o, prm, nsm, st) : run<T, 64, false>(o, prm, nsm, st);
}

// Up to this many rows ordinary lanes may take, with one reading of the weights (few_rows_kernel).
constexpr int FEW_ROWS = 8;

// Rows that the few-rows kernel is built for, 0 for more than it takes.
int few_rows(long long M) { return M > FEW_ROWS ? 0 : (M <= 2 ? static_cast<int>(M) : (M <= 4 ? 4 : 8)); }

template <typename T, int MR>
int run_few(const ip4::FewParams &prm, cudaStream_t st) {
    const unsigned sets = static_cast<unsigned>((prm.N + 127) / 128) * 32;
    // a warp's lanes take 1024 elements at a time: longer rows are shared by a CTA's four
    return launched(prm.bytes <= 512 ? iph::launch_pdl(ip4::few_rows_kernel<T, MR, 1>, dim3(sets / 4), dim3(128), 0, st, prm)
                                     : iph::launch_pdl(ip4::few_rows_kernel<T, MR, 4>, dim3(sets), dim3(128), 0, st, prm));
}
template <typename T>
int run_few(const ip4::FewParams &prm, cudaStream_t st) {
    switch (few_rows(prm.M)) {
    case 1: return run_few<T, 1>(prm, st);
    case 2: return run_few<T, 2>(prm, st);
    case 4: return run_few<T, 4>(prm, st);
    default: return run_few<T, 8>(prm, st);
    }
}

// Its time, ns: a start, and the elements of the weights with each row's products of them (1024 -> 4096 with 1, 2, 4 and 8
// rows 2.7, 2.8, 3.4 and 5.2 us, by tiles 4.3; 4096 -> 1024 as long, by tiles 7.8; 1024 -> 65536 11, 16, 22, 32 and 12).
long long few_time(int rows, int K, int N) {
    return 1600 + 130 * rows + static_cast<long long>(K) * N * (100 + 48 * rows) / 1000000;
}

}  // namespace

extern "C" {

int ip_linear_fp4(const uint8_t *x, long long ldx, const uint8_t *x_blocks, const float *sx, const uint8_t *w,
                  long long ldw, const uint8_t *w_blocks, const float *sw, const float *bias, int act, long long rows,
                  int K, int N, void *y, long long ldy, int dtype, void *workspace, size_t workspace_bytes,
                  ip_stream_t stream) {
    if ((dtype != IP_F32 && dtype != IP_F16 && dtype != IP_BF16) || (act != IP_ACT_NONE && act != IP_ACT_SWISH))
        return IP_ERR_PARAM;
    if (rows < 0 || rows > IP_LINEAR_MAX_FRAMES || K < 1 || K > IP_LINEAR_MAX_K || N < 1 || N > IP_LINEAR_MAX_N) return IP_ERR_SHAPE;
    const int bytes = (K + 1) / 2;
    if (ldx < bytes || ldw < bytes || ldy < N || ldx > (1ll << 39) || ldw > (1ll << 39) || ldy > (1ll << 31)) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!x || !x_blocks || !sx || !w || !w_blocks || !sw || !y || !workspace) return IP_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || ldx % 16 != 0 || ldw % 16 != 0 || !aligned(x_blocks, 16) ||
        !aligned(w_blocks, 16) || !aligned(sx, 4) || !aligned(sw, 4) || (bias && !aligned(bias, 4)) ||
        !aligned(y, dtype == IP_F32 ? 4 : 2) || !aligned(workspace, 256))
        return IP_ERR_ALIGN;
    if (workspace_bytes < 256) return IP_ERR_WORKSPACE;
    const int nsm = sm_count();
    if (nsm <= 0) return IP_ERR_CUDA;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const Times times = tile_times(rows, N, (K + 63) / 64, nsm);
    const int few_m = few_rows(rows);
    if (few_m && few_time(few_m, K, N) <= times.least()) {
        const ip4::FewParams few{x, x_blocks, w, w_blocks, sx, sw, bias, y, ldx, ldw, ldy, static_cast<int>(rows), N, act, bytes, (K + 63) / 64};
        if (dtype == IP_F32) return run_few<float>(few, st);
        if (dtype == IP_F16) return run_few<__half>(few, st);
        return run_few<__nv_bfloat16>(few, st);
    }
    ip4::Params prm;
    prm.sx = sx;
    prm.sw = sw;
    prm.bias = bias;
    prm.y = y;
    prm.M = rows;
    prm.ldy = ldy;
    prm.N = N;
    prm.act = act;
    prm.steps = (K + 63) / 64;
    prm.tiles_n = 0;
    prm.tiles = 0;
    prm.err = static_cast<int *>(workspace);
    prm.timeout_cycles = iph::wait_limit();
    prm.stall = iph::stall_injection();
    const Operands o{x, w, x_blocks, w_blocks, ldx, ldw, bytes};
    if (dtype == IP_F32) return run<float>(o, prm, times, nsm, st);
    if (dtype == IP_F16) return run<__half>(o, prm, times, nsm, st);
    return run<__nv_bfloat16>(o, prm, times, nsm, st);
}

}  // extern "C"
