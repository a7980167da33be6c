// C entry points of tq_mx.h and tq_distill.h: argument checks, then the launch helpers of the kernel files.
#include <hip/hip_runtime.h>

#include "tq_distill.h"
#include "tq_mx.h"

hipError_t tq_launch_mx_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int rounding, uint64_t seed,
                                 uint32_t worker, uint32_t step, void* codes, void* scales, void* codes_t, void* scales_t,
                                 hipStream_t st);
hipError_t tq_launch_mx_dequantize(const void* codes, const void* scales, uint64_t rows, uint64_t cols, void* out, int dtype,
                                   uint64_t ldo, hipStream_t st);
uint64_t tq_mx_matmul_workspace_bytes_impl(uint64_t m, uint64_t n, uint64_t k);
hipError_t tq_launch_mx_matmul(const void* a, const void* sa, const void* b, const void* sb, uint64_t m, uint64_t n, uint64_t k,
                               const float* add, uint64_t lda, void* out, int dtype, uint64_t ldo, void* workspace, hipStream_t st);
bool tq_mx_linear_in_one(uint64_t m, uint64_t n, uint64_t k);
hipError_t tq_launch_mx_linear_few(const void* x, int x_dtype, uint64_t m, uint64_t ldx, const void* w, const void* sw, uint64_t n,
                                   uint64_t k, void* out, int dtype, uint64_t ldo, hipStream_t st);
hipError_t tq_launch_distill(const void* z, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids, int ids_bytes,
                             const float* t, uint64_t top, float temperature, const float* stats_in, const float* grad, float* loss,
                             float* stats, void* dz, uint64_t lddz, hipStream_t st);

namespace {

bool aligned(const void* p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
uint64_t size_of(int dtype) { return dtype == TQ_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == TQ_F32 || dtype == TQ_BF16 || dtype == TQ_F16; }
int from_hip(hipError_t e) { return e == hipSuccess ? TQ_OK : (e == hipErrorInvalidValue ? TQ_EUNSUPPORTED : TQ_EHIP); }

constexpr uint64_t kMaxAxis = 0x7FFFFFFFull, kMaxElements = 1ull << 40;

// rows x cols elements, `ld` from row to row.
int check_matrix(uint64_t rows, uint64_t cols, uint64_t ld)
{
    if (rows == 0 || cols == 0 || ld < cols) return TQ_EINVAL;
    if (rows > kMaxAxis || cols > kMaxAxis || ld > kMaxElements / rows) return TQ_EUNSUPPORTED;
    return TQ_OK;
}

// A matrix in 4-bit form; its rows are padded, which counts.
int check_form(const void* codes, const void* scales, uint64_t rows, uint64_t cols)
{
    const int rc = check_matrix(rows, cols, cols + 127);
    if (rc) return rc;
    if (!codes || !scales) return TQ_EINVAL;
    return aligned(codes, 16) && aligned(scales, 16) ? TQ_OK : TQ_EALIGN;
}

int check_dense(const void* p, int dtype, uint64_t rows, uint64_t cols, uint64_t ld)
{
    const int rc = check_matrix(rows, cols, ld);
    if (rc) return rc;
    if (!p || !known(dtype)) return TQ_EINVAL;
    return aligned(p, size_of(dtype)) ? TQ_OK : TQ_EALIGN;
}

int check_workspace(const void* workspace, uint64_t bytes, uint64_t needed)
{
    if (needed == 0) return TQ_OK;
    if (!workspace || bytes < needed) return TQ_EINVAL;
    return aligned(workspace, 16) ? TQ_OK : TQ_EALIGN;
}

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

extern "C" {

uint64_t tq_mx_code_bytes(uint64_t rows, uint64_t cols)
{
    return check_matrix(rows, cols, cols + 127) ? 0 : rows * ((cols + 127) / 128) * 64;
}

uint64_t tq_mx_scale_bytes(uint64_t rows, uint64_t cols)
{
    return check_matrix(rows, cols, cols + 127) ? 0 : rows * ((cols + 127) / 128) * 4;
}

int tq_mx_quantize(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int rounding, uint64_t seed,
                   uint32_t worker, uint32_t step, void* codes_dev, void* scales_dev, void* codes_t_dev, void* scales_t_dev,
                   void* stream)
{
    int rc;
    if ((rc = check_dense(x_dev, dtype, rows, cols, ld))) return rc;
    if (rounding != TQ_MX_NEAREST && rounding != TQ_MX_STOCHASTIC) return TQ_EINVAL;
    if (!codes_dev != !scales_dev || !codes_t_dev != !scales_t_dev || (!codes_dev && !codes_t_dev)) return TQ_EINVAL;
    if (codes_dev && (rc = check_form(codes_dev, scales_dev, rows, cols))) return rc;
    if (codes_t_dev && (rc = check_form(codes_t_dev, scales_t_dev, cols, rows))) return rc;
    return from_hip(tq_launch_mx_quantize(x_dev, dtype, rows, cols, ld, rounding, seed, worker, step, codes_dev, scales_dev,
                                          codes_t_dev, scales_t_dev, static_cast<hipStream_t>(stream)));
}

int tq_mx_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* out_dev, int out_dtype,
                     uint64_t ldo, void* stream)
{
    int rc;
    if ((rc = check_form(codes_dev, scales_dev, rows, cols)) || (rc = check_dense(out_dev, out_dtype, rows, cols, ldo))) return rc;
    if (out_dtype == TQ_F16) return TQ_EINVAL;
    return from_hip(tq_launch_mx_dequantize(codes_dev, scales_dev, rows, cols, out_dev, out_dtype, ldo,
                                            static_cast<hipStream_t>(stream)));
}

uint64_t tq_mx_matmul_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    if (check_matrix(m, k, k + 127) || check_matrix(n, k, k + 127) || check_matrix(m, n, n)) return 0;
    return tq_mx_matmul_workspace_bytes_impl(m, n, k);
}

int tq_mx_matmul(const void* a_codes_dev, const void* a_scales_dev, const void* b_codes_dev, const void* b_scales_dev, uint64_t m,
                 uint64_t n, uint64_t k, const float* add_dev, uint64_t lda, void* out_dev, int out_dtype, uint64_t ldo,
                 void* workspace_dev, uint64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_form(a_codes_dev, a_scales_dev, m, k)) || (rc = check_form(b_codes_dev, b_scales_dev, n, k)) ||
        (rc = check_dense(out_dev, out_dtype, m, n, ldo)))
        return rc;
    if (add_dev && (rc = check_dense(add_dev, TQ_F32, m, n, lda))) return rc;
    if (add_dev == out_dev && (out_dtype != TQ_F32 || lda != ldo)) return TQ_EINVAL;
    if ((rc = check_workspace(workspace_dev, workspace_bytes, tq_mx_matmul_workspace_bytes_impl(m, n, k)))) return rc;
    return from_hip(tq_launch_mx_matmul(a_codes_dev, a_scales_dev, b_codes_dev, b_scales_dev, m, n, k, add_dev, lda, out_dev,
                                        out_dtype, ldo, workspace_dev, static_cast<hipStream_t>(stream)));
}

uint64_t tq_mx_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    if (check_matrix(m, k, k + 127) || check_matrix(n, k, k + 127) || check_matrix(m, n, n)) return 0;
    if (tq_mx_linear_in_one(m, n, k)) return 0;
    return padded(tq_mx_code_bytes(m, k)) + padded(tq_mx_scale_bytes(m, k)) + tq_mx_matmul_workspace_bytes_impl(m, n, k);
}

int tq_mx_linear(const void* x_dev, int dtype, uint64_t m, uint64_t ldx, const void* w_codes_dev, const void* w_scales_dev,
                 uint64_t n, uint64_t k, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev, uint64_t workspace_bytes,
                 void* stream)
{
    int rc;
    if ((rc = check_dense(x_dev, dtype, m, k, ldx)) || (rc = check_form(w_codes_dev, w_scales_dev, n, k)) ||
        (rc = check_dense(out_dev, out_dtype, m, n, ldo)) ||
        (rc = check_workspace(workspace_dev, workspace_bytes, tq_mx_linear_workspace_bytes(m, n, k))))
        return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (tq_mx_linear_in_one(m, n, k))
        return from_hip(tq_launch_mx_linear_few(x_dev, dtype, m, ldx, w_codes_dev, w_scales_dev, n, k, out_dev, out_dtype, ldo, st));
    char* codes = static_cast<char*>(workspace_dev);
    char* scales = codes + padded(tq_mx_code_bytes(m, k));
    rc = from_hip(tq_launch_mx_quantize(x_dev, dtype, m, k, ldx, TQ_MX_NEAREST, 0, 0, 0, codes, scales, nullptr, nullptr, st));
    if (rc) return rc;
    return from_hip(tq_launch_mx_matmul(codes, scales, w_codes_dev, w_scales_dev, m, n, k, nullptr, 0, out_dev, out_dtype, ldo,
                                        scales + padded(tq_mx_scale_bytes(m, k)), st));
}

// Checks shared by the three distillation calls.
static int check_distill(const void* z, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids, int ids_bytes,
                         const float* t, uint64_t top, float temperature)
{
    const int rc = check_dense(z, dtype, rows, vocab, ldz);
    if (rc) return rc;
    if (!ids || !t || (ids_bytes != 4 && ids_bytes != 8) || top == 0) return TQ_EINVAL;
    if (!(temperature >= 1e-4f && temperature <= 1e4f)) return TQ_EINVAL;
    if (top > TQ_DISTILL_MAX_TOP) return TQ_EUNSUPPORTED;
    return aligned(ids, ids_bytes) && aligned(t, 4) ? TQ_OK : TQ_EALIGN;
}

// dz is apart from z, or z itself with the same rows.
static int check_gradient(const void* z, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const float* grad, const void* dz,
                          uint64_t lddz)
{
    const int rc = check_dense(dz, dtype, rows, vocab, lddz);
    if (rc) return rc;
    if (!grad || (dz == z && lddz != ldz)) return TQ_EINVAL;
    return aligned(grad, 4) ? TQ_OK : TQ_EALIGN;
}

int tq_distill_forward(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev, int ids_bytes,
                       const float* t_dev, uint64_t top, float temperature, float* loss_dev, float* stats_dev, void* stream)
{
    const int rc = check_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature);
    if (rc) return rc;
    if (!loss_dev || !stats_dev) return TQ_EINVAL;
    if (!aligned(loss_dev, 4) || !aligned(stats_dev, 4)) return TQ_EALIGN;
    return from_hip(tq_launch_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature, nullptr, nullptr,
                                      loss_dev, stats_dev, nullptr, 0, static_cast<hipStream_t>(stream)));
}

int tq_distill_backward(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev, int ids_bytes,
                        const float* t_dev, uint64_t top, float temperature, const float* stats_dev, const float* grad_dev, void* dz_dev,
                        uint64_t lddz, void* stream)
{
    int rc;
    if ((rc = check_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature)) ||
        (rc = check_gradient(z_dev, dtype, rows, vocab, ldz, grad_dev, dz_dev, lddz)))
        return rc;
    if (!stats_dev) return TQ_EINVAL;
    if (!aligned(stats_dev, 4)) return TQ_EALIGN;
    return from_hip(tq_launch_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature, stats_dev, grad_dev,
                                      nullptr, nullptr, dz_dev, lddz, static_cast<hipStream_t>(stream)));
}

int tq_distill(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev, int ids_bytes,
               const float* t_dev, uint64_t top, float temperature, const float* grad_dev, float* loss_dev, void* dz_dev, uint64_t lddz,
               void* stream)
{
    int rc;
    if ((rc = check_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature)) ||
        (rc = check_gradient(z_dev, dtype, rows, vocab, ldz, grad_dev, dz_dev, lddz)))
        return rc;
    if (!loss_dev) return TQ_EINVAL;
    if (!aligned(loss_dev, 4)) return TQ_EALIGN;
    return from_hip(tq_launch_distill(z_dev, dtype, rows, vocab, ldz, ids_dev, ids_bytes, t_dev, top, temperature, nullptr, grad_dev,
                                      loss_dev, nullptr, dz_dev, lddz, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
