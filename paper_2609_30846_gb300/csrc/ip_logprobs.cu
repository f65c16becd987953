// Host side of the log probabilities of the C ABI (include/ip_mhsa.h): argument validation, the plan
// of the rows and launches.  Device code: ip_logprobs_kernels.cuh.
#include "ip_mhsa.h"
#include "ip_logprobs_kernels.cuh"
#include "ip_host_util.h"

#include <cuda_runtime.h>

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int launched(cudaError_t rc) {
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? IP_OK : IP_ERR_CUDA;
}

// Elements that U units a thread hold: all, where rows start on 16 bytes, or eight less (up to seven before a row).
constexpr int hold(int threads, int units, bool on16 = false) { return threads * units * 8 - (on16 ? 0 : 8); }

// SMs of a GB300.  A constant, so that the workspace's size needs no device.
constexpr int SMS = 152;

// Parts of a row and their elements: one while a CTA holds the row; else a cluster's, as many as come to
// four CTAs an SM, few rows by sixteen CTAs of few elements (1 x 65536 with twenty 6.7 us by 16 CTAs, by 8 7.5) and many by those
// whose registers the parts fill; parts that a second kernel joins for what sixteen CTAs do not hold.
struct Plan {
    int parts, per, cluster;
};
Plan plan(long long rows, int V, bool on16 = false) {
    const int most = hold(256, 4, on16);
    if (V <= most) return {1, V, 0};
    auto per_of = [&](int parts) { return ((V + parts - 1) / parts + 7) / 8 * 8; };
    int parts = 2;
    while (parts < ipl::MAX_CLUSTER && per_of(parts) > most) parts *= 2;
    if (per_of(parts) > most) return {(V + hold(256, 4) - 1) / hold(256, 4), hold(256, 4), 0};
    while (parts < ipl::MAX_CLUSTER && rows * parts * 2 <= 4 * SMS) parts *= 2;
    return {parts, per_of(parts), 1};
}

bool shape_ok(long long rows, int V, int top) {
    return rows >= 0 && rows <= IP_LINEAR_MAX_FRAMES && V >= 1 && V <= IP_LOGPROBS_MAX_V && top >= 0 &&
           top <= IP_LOGPROBS_MAX_TOP && top <= V;
}

size_t keys_at(long long rows, const Plan &p) { return 256 + static_cast<size_t>(rows) * p.parts * 16; }
size_t space(long long rows, const Plan &p, int top) {
    return p.parts == 1 || p.cluster ? 256 : keys_at(rows, p) + static_cast<size_t>(rows) * p.parts * top * 8;
}

template <typename T, int TPR, int U, int S, int HOLDS>
int launch(const ipl::LogprobParams &prm, cudaStream_t st) {
    auto *fn = ipl::logprob_kernel<T, TPR, U, S, HOLDS>;
    const long long ctas = TPR == 32 ? (prm.rows + 3) / 4 : prm.rows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(HOLDS == ipl::WHOLE ? 1 : prm.parts));
    cfg.blockDim = dim3(TPR == 32 ? 128 : TPR);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = static_cast<unsigned>(prm.parts);
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = HOLDS == ipl::CLUSTER ? 2 : 1;
    if (HOLDS == ipl::CLUSTER && prm.parts > 8 &&
        cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
        return IP_ERR_CUDA;
    return launched(cudaLaunchKernelEx(&cfg, fn, prm));
}

template <typename T>
int run(const ipl::LogprobParams &prm, bool cluster, bool on16, cudaStream_t st) {
    if (cluster)
        return prm.per <= hold(256, 1, on16) ? launch<T, 256, 1, 0, ipl::CLUSTER>(prm, st)
               : prm.per <= hold(256, 2, on16) ? launch<T, 256, 2, 0, ipl::CLUSTER>(prm, st)
               : prm.per <= hold(256, 3, on16) ? launch<T, 256, 3, 0, ipl::CLUSTER>(prm, st) : launch<T, 256, 4, 0, ipl::CLUSTER>(prm, st);
    if (prm.parts > 1) {
        const int rc = launch<T, 256, 4, 0, ipl::PARTS>(prm, st);
        if (rc != IP_OK) return rc;
        return launched(iph::launch_pdl(ipl::logprob_join_kernel<T>, dim3(static_cast<unsigned>(prm.rows)), dim3(256), 0, st, prm));
    }
    // A warp's lanes: units by powers of two, and one element more a lane where that spares twice the units (12000 bf16
    // rows of 280 4.5 us for 4.9, 536 5.2 for 6.8, 1048 7.4 and 1049, with eight units, 12.1).  Not behind eight: the CTA's form that
    // follows is sooner with few rows (1 x 2056 1.65 us, by a warp 1.93).
    if (prm.V <= hold(32, 1)) return launch<T, 32, 1, 0, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 1) + 32) return launch<T, 32, 1, 1, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 2)) return launch<T, 32, 2, 0, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 2) + 32) return launch<T, 32, 2, 1, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 4)) return launch<T, 32, 4, 0, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 4) + 32) return launch<T, 32, 4, 1, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(32, 8)) return launch<T, 32, 8, 0, ipl::WHOLE>(prm, st);
    if (prm.V <= hold(256, 2, on16)) return launch<T, 256, 2, 0, ipl::WHOLE>(prm, st);
    return launch<T, 256, 4, 0, ipl::WHOLE>(prm, st);
}

}  // namespace

extern "C" {

size_t ip_token_logprobs_workspace_bytes(long long rows, int V, int top) {
    return shape_ok(rows, V, top) ? space(rows, plan(rows, V), top) : 0;
}

int ip_token_logprobs(const void *logits, int dtype, long long rows, int V, long long ld, const void *tokens,
                      int tokens_i64, float scale, int top, float *logprob, float *entropy, float *top_logprob,
                      int32_t *top_token, void *workspace, size_t workspace_bytes, ip_stream_t stream) {
    if ((dtype != IP_F32 && dtype != IP_F16 && dtype != IP_BF16) || !(scale > 0.0f && scale < 1e30f) ||
        (tokens_i64 != 0 && tokens_i64 != 1))
        return IP_ERR_PARAM;
    if (!shape_ok(rows, V, top) || ld < V || ld > (1ll << 40)) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!logits || !entropy || !workspace || (tokens && !logprob) || (top > 0 && (!top_logprob || !top_token))) return IP_ERR_NULL;
    if (!aligned(logits, dtype == IP_F32 ? 4 : 2) || !aligned(entropy, 4) || !aligned(workspace, 256) ||
        (tokens && (!aligned(tokens, tokens_i64 ? 8 : 4) || !aligned(logprob, 4))) ||
        (top > 0 && (!aligned(top_logprob, 4) || !aligned(top_token, 4))))
        return IP_ERR_ALIGN;
    // rows that start on 16 bytes may do with a cluster where others do not, never the other way round
    const bool on16 = aligned(logits, 16) && (rows == 1 || ld * (dtype == IP_F32 ? 4 : 2) % 16 == 0);
    const Plan p = plan(rows, V, on16);
    if (workspace_bytes < space(rows, p, top)) return IP_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    const ipl::LogprobParams prm{logits, rows, ld, V, top, p.parts, p.per, scale, tokens, tokens_i64, logprob, entropy,
                                 top_logprob, top_token, reinterpret_cast<float *>(ws + 256),
                                 reinterpret_cast<ipl::Key *>(ws + keys_at(rows, p))};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return run<float>(prm, p.cluster, on16, st);
    if (dtype == IP_F16) return run<__half>(prm, p.cluster, on16, st);
    return run<__nv_bfloat16>(prm, p.cluster, on16, st);
}

}  // extern "C"
