// Host side of the norm with quantised rows, the 4-bit rows and the values of rows of the C ABI
// (include/ip_mhsa.h): argument validation and launches.  Device code: ip_rows_kernels.cuh.
#include "ip_mhsa.h"
#include "ip_rows_kernels.cuh"
#include "ip_host_util.h"

#include <cuda_runtime.h>

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t elem_size(int dtype) { return dtype == IP_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == IP_F32 || dtype == IP_F16 || dtype == IP_BF16; }
bool shape_ok(long long rows, int d) { return rows >= 0 && rows <= IP_NORM_MAX_ROWS && d >= 1 && d <= IP_LINEAR_MAX_K; }
bool stride_ok(long long ld, long long d) { return ld >= d && ld <= (1ll << 40); }

int launched(cudaError_t rc) {
    return rc == cudaSuccess && cudaGetLastError() == cudaSuccess ? IP_OK : IP_ERR_CUDA;
}

unsigned grid_of(long long need) { return static_cast<unsigned>(need < (1 << 20) ? need : (1 << 20)); }

template <typename T, int TPR, int UNITS, bool VEC, int OUT, bool NORM>
int launch_rows(const ipw::RowsParams &prm, cudaStream_t st) {
    constexpr int THREADS = TPR < 128 ? 128 : TPR, RPC = THREADS / TPR;
    return launched(iph::launch_pdl(ipw::rows_kernel<T, TPR, UNITS, VEC, OUT, NORM>, dim3(grid_of((prm.rows + RPC - 1) / RPC)),
                                    dim3(THREADS), 0, st, prm));
}

template <typename T, bool VEC, int OUT, bool NORM>
int run_rows(const ipw::RowsParams &prm, cudaStream_t st) {
    // a warp a row while its lanes can hold the row, then four warps, then eight
    if (prm.d <= 512) return launch_rows<T, 32, 1, VEC, OUT, NORM>(prm, st);
    if (prm.d <= 1024) return launch_rows<T, 32, 2, VEC, OUT, NORM>(prm, st);
    if (prm.d <= 2048) return launch_rows<T, 128, 1, VEC, OUT, NORM>(prm, st);
    if (prm.d <= 4096) return launch_rows<T, 128, 2, VEC, OUT, NORM>(prm, st);
    return launch_rows<T, 256, 2, VEC, OUT, NORM>(prm, st);
}

template <typename T, int OUT, bool NORM>
int run_rows(const ipw::RowsParams &prm, cudaStream_t st) {
    auto rows16 = [&](const void *p, long long ld) { return aligned(p, 16) && (prm.rows == 1 || ld * static_cast<long long>(sizeof(T)) % 16 == 0); };
    const bool vec = prm.d % 8 == 0 && rows16(prm.x, prm.ldx) && (!NORM || aligned(prm.weight, 16)) &&
                     (!prm.res || (rows16(prm.res, prm.ldres) && rows16(prm.sum, prm.ldsum))) &&
                     (OUT == ipw::OUT_FP4 || (aligned(prm.q, 16) && (prm.rows == 1 || prm.ldq % 16 == 0)));
    return vec ? run_rows<T, true, OUT, NORM>(prm, st) : run_rows<T, false, OUT, NORM>(prm, st);
}

template <int OUT, bool NORM>
int run_rows(int dtype, const ipw::RowsParams &prm, ip_stream_t stream) {
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return run_rows<float, OUT, NORM>(prm, st);
    if (dtype == IP_F16) return run_rows<__half, OUT, NORM>(prm, st);
    return run_rows<__nv_bfloat16, OUT, NORM>(prm, st);
}

// What the two norms have in common; IP_OK if the call may go on.
int check_norm(const void *x, long long ldx, const void *res, long long ldres, const void *weight, float eps, int dtype,
               long long rows, int d, const void *sum, long long ldsum) {
    if (!dtype_ok(dtype) || !(eps >= 0.0f && eps < 1e30f)) return IP_ERR_PARAM;
    if (!shape_ok(rows, d) || !stride_ok(ldx, d) || (res && (!stride_ok(ldres, d) || !stride_ok(ldsum, d)))) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!x || !weight || (res && !sum)) return IP_ERR_NULL;
    const size_t es = elem_size(dtype);
    if (!aligned(x, es) || !aligned(weight, es) || (res && (!aligned(res, es) || !aligned(sum, es)))) return IP_ERR_ALIGN;
    return IP_OK;
}

// Rows of 4-bit codes.
int check_fp4(long long rows, int d, const void *q, long long ldq, const void *blocks, const void *scale) {
    if (!stride_ok(ldq, (d + 1) / 2)) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!q || !blocks || !scale) return IP_ERR_NULL;
    if (!aligned(q, 16) || ldq % 16 != 0 || !aligned(blocks, 16) || !aligned(scale, 4)) return IP_ERR_ALIGN;
    return IP_OK;
}

template <typename T, int IN>
int run_values(const ipw::ValuesParams &prm, bool vec, cudaStream_t st) {
    const dim3 grid(grid_of((prm.rows * prm.units + 255) / 256)), block(256);
    auto *fn = !vec ? ipw::values_kernel<T, false, false, IN>
                    : (prm.d % 16 == 0 ? ipw::values_kernel<T, true, true, IN> : ipw::values_kernel<T, true, false, IN>);
    return launched(iph::launch_pdl(fn, grid, block, 0, st, prm));
}

template <int IN>
int run_values(int dtype, ipw::ValuesParams prm, ip_stream_t stream) {
    prm.units = (prm.d + 15) / 16;
    prm.magic = iph::div_magic(static_cast<unsigned long long>(prm.units));
    const long long es = static_cast<long long>(elem_size(dtype));
    const int qa = IN == ipw::OUT_I8 ? 16 : 8;
    const bool one = prm.rows == 1;
    prm.wide = aligned(prm.y, 32) && (one || prm.ldy * es % 32 == 0);
    prm.qvec = aligned(prm.q, qa) && (one || prm.ldq % qa == 0);
    // f32 rows on 8 bytes only are turned like others (6000 x 1002 8.7 us, by pairs of elements 16.8)
    const bool vec = prm.qvec && (prm.wide || (dtype != IP_F32 && aligned(prm.y, 8) && (one || prm.ldy * es % 8 == 0)));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == IP_F32) return run_values<float, IN>(prm, vec, st);
    if (dtype == IP_F16) return run_values<__half, IN>(prm, vec, st);
    return run_values<__nv_bfloat16, IN>(prm, vec, st);
}

}  // namespace

extern "C" {

int ip_rmsnorm_i8(const void *x, long long ldx, const void *residual, long long ldres, const void *weight, float eps,
                  int dtype, long long rows, int d, void *sum, long long ldsum, int8_t *q, long long ldq, float *scale,
                  ip_stream_t stream) {
    const int rc = check_norm(x, ldx, residual, ldres, weight, eps, dtype, rows, d, sum, ldsum);
    if (rc != IP_OK) return rc;
    if (!stride_ok(ldq, d)) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!q || !scale) return IP_ERR_NULL;
    if (!aligned(scale, 4)) return IP_ERR_ALIGN;
    const ipw::RowsParams prm{x, residual, weight, rows, ldx, ldres, ldsum, ldq, d, eps, sum,
                              reinterpret_cast<uint8_t *>(q), nullptr, scale, aligned(q, 16) && (rows == 1 || ldq % 16 == 0)};
    return run_rows<ipw::OUT_I8, true>(dtype, prm, stream);
}

int ip_rmsnorm_fp4(const void *x, long long ldx, const void *residual, long long ldres, const void *weight, float eps,
                   int dtype, long long rows, int d, void *sum, long long ldsum, uint8_t *q, long long ldq,
                   uint8_t *blocks, float *scale, ip_stream_t stream) {
    int rc = check_norm(x, ldx, residual, ldres, weight, eps, dtype, rows, d, sum, ldsum);
    if (rc == IP_OK) rc = check_fp4(rows, d, q, ldq, blocks, scale);
    if (rc != IP_OK || rows == 0) return rc;
    const ipw::RowsParams prm{x, residual, weight, rows, ldx, ldres, ldsum, ldq, d, eps, sum, q, blocks, scale, true};
    return run_rows<ipw::OUT_FP4, true>(dtype, prm, stream);
}

size_t ip_fp4_block_bytes(long long rows, int d) {
    return shape_ok(rows, d) ? static_cast<size_t>((rows + 127) / 128) * static_cast<size_t>((d + 63) / 64) * 512 : 0;
}

int ip_quantize_fp4(const void *x, int dtype, long long rows, int d, long long ldx, uint8_t *q, long long ldq,
                    uint8_t *blocks, float *scale, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (!shape_ok(rows, d) || !stride_ok(ldx, d)) return IP_ERR_SHAPE;
    const int rc = check_fp4(rows, d, q, ldq, blocks, scale);
    if (rc != IP_OK || rows == 0) return rc;
    if (!x) return IP_ERR_NULL;
    if (!aligned(x, elem_size(dtype))) return IP_ERR_ALIGN;
    const ipw::RowsParams prm{x, nullptr, nullptr, rows, ldx, 0, 0, ldq, d, 0.0f, nullptr, q, blocks, scale, true};
    return run_rows<ipw::OUT_FP4, false>(dtype, prm, stream);
}

int ip_dequantize_i8(const int8_t *q, long long ldq, const float *scale, long long rows, int d, void *y, long long ldy,
                     int dtype, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (!shape_ok(rows, d) || !stride_ok(ldq, d) || !stride_ok(ldy, d)) return IP_ERR_SHAPE;
    if (rows == 0) return IP_OK;
    if (!q || !scale || !y) return IP_ERR_NULL;
    if (!aligned(scale, 4) || !aligned(y, elem_size(dtype))) return IP_ERR_ALIGN;
    return run_values<ipw::OUT_I8>(dtype, ipw::ValuesParams{reinterpret_cast<const uint8_t *>(q), nullptr, scale, rows, ldq, ldy, d, y, 0, 0, 0, false}, stream);
}

int ip_dequantize_fp4(const uint8_t *q, long long ldq, const uint8_t *blocks, const float *scale, long long rows, int d,
                      void *y, long long ldy, int dtype, ip_stream_t stream) {
    if (!dtype_ok(dtype)) return IP_ERR_PARAM;
    if (!shape_ok(rows, d) || !stride_ok(ldy, d)) return IP_ERR_SHAPE;
    const int rc = check_fp4(rows, d, q, ldq, blocks, scale);
    if (rc != IP_OK || rows == 0) return rc;
    if (!y) return IP_ERR_NULL;
    if (!aligned(y, elem_size(dtype))) return IP_ERR_ALIGN;
    return run_values<ipw::OUT_FP4>(dtype, ipw::ValuesParams{q, blocks, scale, rows, ldq, ldy, d, y, 0, 0, 0, false}, stream);
}

}  // extern "C"
