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

// Elements that U units a thread hold wherever the row starts (up to seven before it).
constexpr int hold(int threads, int units) { return threads * units * 8 - 8; }

// Parts of a row and their elements: one while a CTA holds the row, else small parts while they
// come to two CTAs an SM, and parts that fill the registers beyond that.
struct Plan {
    int parts, per;
};
Plan plan(long long rows, int V) {
    if (V <= hold(256, 4)) return {1, V};
    Plan p = {1, V};
    for (int units = 1; units <= 4; units *= 2) {
        p.per = hold(256, units);
        p.parts = (V + p.per - 1) / p.per;
        if (rows * p.parts <= 304) break;
    }
    return p;
}

bool shape_ok(long long rows, int V, int top) {
    return rows >= 0 && rows <= IP_LINEAR_MAX_FRAMES && V >= 1 && V <= IP_LOGPROBS_MAX_V && top >= 0 &&
           top <= IP_LOGPROBS_MAX_TOP && top <= V;
}

size_t keys_at(long long rows, const Plan &p) { return 256 + static_cast<size_t>(rows) * p.parts * 16; }
size_t space(long long rows, const Plan &p, int top) {
    return p.parts == 1 ? 256 : keys_at(rows, p) + static_cast<size_t>(rows) * p.parts * top * 8;
}

template <typename T, int TPR, int U, bool PART>
int launch(const ipl::LogprobParams &prm, cudaStream_t st) {
    const long long ctas = TPR == 32 ? (prm.rows + 3) / 4 : prm.rows;
    return launched(iph::launch_pdl(ipl::logprob_kernel<T, TPR, U, PART>,
                                    dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(PART ? prm.parts : 1)),
                                    dim3(TPR == 32 ? 128 : TPR), 0, st, prm));
}

template <typename T>
int run(const ipl::LogprobParams &prm, cudaStream_t st) {
    if (prm.parts > 1) {
        const int rc = prm.per <= hold(256, 1) ? launch<T, 256, 1, true>(prm, st)
                       : prm.per <= hold(256, 2) ? launch<T, 256, 2, true>(prm, st) : launch<T, 256, 4, true>(prm, st);
        if (rc != IP_OK) return rc;
        return launched(iph::launch_pdl(ipl::logprob_join_kernel<T>, dim3(static_cast<unsigned>(prm.rows)), dim3(256), 0, st, prm));
    }
    if (prm.V <= hold(32, 2)) return launch<T, 32, 2, false>(prm, st);
    if (prm.V <= hold(32, 5)) return launch<T, 32, 5, false>(prm, st);
    if (prm.V <= hold(32, 8)) return launch<T, 32, 8, false>(prm, st);
    if (prm.V <= hold(256, 2)) return launch<T, 256, 2, false>(prm, st);
    return launch<T, 256, 4, false>(prm, st);
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
    const Plan p = plan(rows, V);
    if (workspace_bytes < space(rows, p, top)) return IP_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    const ipl::LogprobParams prm{logits, rows, ld, V, top, p.parts, p.per, scale, tokens, tokens_i64, logprob, entropy,
                                 top_logprob, top_token, reinterpret_cast<float *>(ws + 256),
                                 reinterpret_cast<ipl::Key *>(ws + keys_at(rows, p))};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return run<float>(prm, st);
    if (dtype == IP_F16) return run<__half>(prm, st);
    return run<__nv_bfloat16>(prm, st);
}

}  // extern "C"
