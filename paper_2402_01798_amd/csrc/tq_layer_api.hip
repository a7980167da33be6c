// C entry points of tq_norm.h, tq_i8.h and tq_orth.h: argument checks, then the launch helpers of the kernel files.
#include <hip/hip_runtime.h>
#include <math.h>

#include "tq_i8.h"
#include "tq_norm.h"
#include "tq_orth.h"

hipError_t tq_launch_layernorm_forward(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* weight,
                                       const void* bias, int wtype, float eps, void* y, uint64_t ldy, float* stats, hipStream_t st);
uint64_t tq_layernorm_workspace_bytes_impl(uint64_t rows, uint64_t cols);
hipError_t tq_launch_layernorm_backward(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* dy, uint64_t lddy,
                                        const void* weight, int wtype, const float* stats, void* dx, uint64_t lddx, float* dweight,
                                        float* dbias, int accumulate, void* workspace, hipStream_t st);
hipError_t tq_launch_i8_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* codes, float* scales,
                                 hipStream_t st);
hipError_t tq_launch_i8_dequantize(const void* codes, const float* scales, uint64_t rows, uint64_t cols, void* out, int dtype,
                                   uint64_t ldo, hipStream_t st);
uint64_t tq_i8_matmul_workspace_bytes_impl(uint64_t m, uint64_t n, uint64_t k);
hipError_t tq_launch_i8_matmul(const void* a, const float* sa, const void* b, const float* sb, uint64_t m, uint64_t n, uint64_t k,
                               const float* bias, void* out, int dtype, uint64_t ldo, void* workspace, hipStream_t st);
bool tq_i8_linear_in_one(uint64_t m, uint64_t n, uint64_t k);
hipError_t tq_launch_i8_linear_few(const void* x, int x_dtype, uint64_t m, uint64_t ldx, const void* w, const float* sw, uint64_t n, uint64_t k,
                                   const float* bias, void* out, int dtype, uint64_t ldo, hipStream_t st);
uint64_t tq_orth_workspace_bytes_impl(uint64_t rows, uint64_t cols, int count, int precision);
hipError_t tq_launch_orth(const void* const* g, int count, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum, int nesterov,
                          float weight_decay, float scale, int steps, const float* coefficients, int precision, float eps,
                          const float* const* v, float* const* v_out, const float* const* theta, void* const* out, int out_dtype,
                          void* workspace, hipStream_t st);

namespace {

bool aligned(const void* p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
uint64_t size_of(int dtype) { return dtype == TQ_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == TQ_F32 || dtype == TQ_BF16 || dtype == TQ_F16; }
int from_hip(hipError_t e) { return e == hipSuccess ? TQ_OK : (e == hipErrorInvalidValue ? TQ_EUNSUPPORTED : TQ_EHIP); }
bool usable_eps(float eps) { return eps >= 1e-30f && eps < INFINITY; }

constexpr uint64_t kMaxAxis = 0x7FFFFFFFull, kMaxElements = 1ull << 40;

// rows x cols elements, `ld` from row to row.
int check_matrix(uint64_t rows, uint64_t cols, uint64_t ld)
{
    if (rows == 0 || cols == 0 || ld < cols) return TQ_EINVAL;
    if (rows > kMaxAxis || cols > kMaxAxis || ld > kMaxElements / rows) return TQ_EUNSUPPORTED;
    return TQ_OK;
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

// A matrix in 8-bit form; its rows are padded, which counts.
int check_form(const void* codes, const float* scales, uint64_t rows, uint64_t cols)
{
    const int rc = check_matrix(rows, cols, cols + 127);
    if (rc) return rc;
    if (!codes || !scales) return TQ_EINVAL;
    return aligned(codes, 16) && aligned(scales, 4) ? TQ_OK : TQ_EALIGN;
}

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

extern "C" {

int tq_layernorm_forward(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* weight_dev,
                         const void* bias_dev, int wtype, float eps, void* y_dev, uint64_t ldy, float* stats_dev, void* stream)
{
    int rc;
    if ((rc = check_dense(x_dev, dtype, rows, cols, ldx)) || (rc = check_dense(y_dev, dtype, rows, cols, ldy))) return rc;
    if (!known(wtype) || !usable_eps(eps) || (y_dev == x_dev && ldy != ldx)) return TQ_EINVAL;
    if (!aligned(weight_dev, size_of(wtype)) || !aligned(bias_dev, size_of(wtype)) || !aligned(stats_dev, 4)) return TQ_EALIGN;
    return from_hip(tq_launch_layernorm_forward(x_dev, dtype, rows, cols, ldx, weight_dev, bias_dev, wtype, eps, y_dev, ldy, stats_dev,
                                                static_cast<hipStream_t>(stream)));
}

uint64_t tq_layernorm_workspace_bytes(uint64_t rows, uint64_t cols)
{
    return check_matrix(rows, cols, cols) ? 0 : tq_layernorm_workspace_bytes_impl(rows, cols);
}

int tq_layernorm_backward(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* dy_dev, uint64_t lddy,
                          const void* weight_dev, int wtype, const float* stats_dev, void* dx_dev, uint64_t lddx, float* dweight_dev,
                          float* dbias_dev, int accumulate, void* workspace_dev, uint64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_dense(x_dev, dtype, rows, cols, ldx)) || (rc = check_dense(dy_dev, dtype, rows, cols, lddy))) return rc;
    if (dx_dev && (rc = check_dense(dx_dev, dtype, rows, cols, lddx))) return rc;
    if (!known(wtype) || !stats_dev || (accumulate != 0 && accumulate != 1) || (!dx_dev && !dweight_dev && !dbias_dev)) return TQ_EINVAL;
    if (dx_dev && ((dx_dev == dy_dev && lddx != lddy) || (dx_dev == x_dev && lddx != ldx))) return TQ_EINVAL;
    if (!aligned(weight_dev, size_of(wtype)) || !aligned(stats_dev, 4) || !aligned(dweight_dev, 4) || !aligned(dbias_dev, 4)) return TQ_EALIGN;
    if ((dweight_dev || dbias_dev) && (rc = check_workspace(workspace_dev, workspace_bytes, tq_layernorm_workspace_bytes_impl(rows, cols)))) return rc;
    return from_hip(tq_launch_layernorm_backward(x_dev, dtype, rows, cols, ldx, dy_dev, lddy, weight_dev, wtype, stats_dev, dx_dev, lddx,
                                                 dweight_dev, dbias_dev, accumulate, workspace_dev, static_cast<hipStream_t>(stream)));
}

uint64_t tq_i8_code_bytes(uint64_t rows, uint64_t cols)
{
    return check_matrix(rows, cols, cols + 127) ? 0 : rows * ((cols + 127) / 128 * 128);
}

int tq_i8_quantize(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, void* codes_dev, float* scales_dev,
                   void* stream)
{
    int rc;
    if ((rc = check_dense(x_dev, dtype, rows, cols, ldx)) || (rc = check_form(codes_dev, scales_dev, rows, cols))) return rc;
    return from_hip(tq_launch_i8_quantize(x_dev, dtype, rows, cols, ldx, codes_dev, scales_dev, static_cast<hipStream_t>(stream)));
}

int tq_i8_dequantize(const void* codes_dev, const float* scales_dev, uint64_t rows, uint64_t cols, void* out_dev, int out_dtype,
                     uint64_t ldo, void* stream)
{
    int rc;
    if ((rc = check_form(codes_dev, scales_dev, rows, cols)) || (rc = check_dense(out_dev, out_dtype, rows, cols, ldo))) return rc;
    return from_hip(tq_launch_i8_dequantize(codes_dev, scales_dev, rows, cols, out_dev, out_dtype, ldo, static_cast<hipStream_t>(stream)));
}

// A product's sizes.
static int check_product(uint64_t m, uint64_t n, uint64_t k)
{
    int rc;
    if ((rc = check_matrix(m, k, k + 127)) || (rc = check_matrix(n, k, k + 127)) || (rc = check_matrix(m, n, n))) return rc;
    return k > TQ_I8_MAX_K ? TQ_EUNSUPPORTED : TQ_OK;
}

uint64_t tq_i8_matmul_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    return check_product(m, n, k) ? 0 : tq_i8_matmul_workspace_bytes_impl(m, n, k);
}

int tq_i8_matmul(const void* a_codes_dev, const float* a_scales_dev, const void* b_codes_dev, const float* b_scales_dev, uint64_t m,
                 uint64_t n, uint64_t k, const float* bias_dev, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev,
                 uint64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_product(m, n, k)) || (rc = check_form(a_codes_dev, a_scales_dev, m, k)) ||
        (rc = check_form(b_codes_dev, b_scales_dev, n, k)) || (rc = check_dense(out_dev, out_dtype, m, n, ldo)))
        return rc;
    if (!aligned(bias_dev, 4)) return TQ_EALIGN;
    if ((rc = check_workspace(workspace_dev, workspace_bytes, tq_i8_matmul_workspace_bytes_impl(m, n, k)))) return rc;
    return from_hip(tq_launch_i8_matmul(a_codes_dev, a_scales_dev, b_codes_dev, b_scales_dev, m, n, k, bias_dev, out_dev, out_dtype, ldo,
                                        workspace_dev, static_cast<hipStream_t>(stream)));
}

uint64_t tq_i8_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    if (check_product(m, n, k) || tq_i8_linear_in_one(m, n, k)) return 0;
    return padded(tq_i8_code_bytes(m, k)) + padded(4 * m) + tq_i8_matmul_workspace_bytes_impl(m, n, k);
}

int tq_i8_linear(const void* x_dev, int dtype, uint64_t m, uint64_t ldx, const void* w_codes_dev, const float* w_scales_dev, uint64_t n,
                 uint64_t k, const float* bias_dev, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev,
                 uint64_t workspace_bytes, void* stream)
{
    int rc;
    if ((rc = check_product(m, n, k)) || (rc = check_dense(x_dev, dtype, m, k, ldx)) || (rc = check_form(w_codes_dev, w_scales_dev, n, k)) ||
        (rc = check_dense(out_dev, out_dtype, m, n, ldo)))
        return rc;
    if (!aligned(bias_dev, 4)) return TQ_EALIGN;
    if ((rc = check_workspace(workspace_dev, workspace_bytes, tq_i8_linear_workspace_bytes(m, n, k)))) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (tq_i8_linear_in_one(m, n, k))
        return from_hip(tq_launch_i8_linear_few(x_dev, dtype, m, ldx, w_codes_dev, w_scales_dev, n, k, bias_dev, out_dev, out_dtype, ldo, st));
    char* codes = static_cast<char*>(workspace_dev);
    float* scales = reinterpret_cast<float*>(codes + padded(tq_i8_code_bytes(m, k)));
    if ((rc = from_hip(tq_launch_i8_quantize(x_dev, dtype, m, k, ldx, codes, scales, st)))) return rc;
    return from_hip(tq_launch_i8_matmul(codes, scales, w_codes_dev, w_scales_dev, m, n, k, bias_dev, out_dev, out_dtype, ldo,
                                        reinterpret_cast<char*>(scales) + padded(4 * m), st));
}

// Sizes of matrices that are orthogonalised.
static int check_orth_sizes(uint64_t rows, uint64_t cols, int count, int precision)
{
    const int rc = check_matrix(rows, cols, cols);
    if (rc) return rc;
    if (count < 1 || (precision != TQ_ORTH_HALF && precision != TQ_ORTH_SPLIT)) return TQ_EINVAL;
    const uint64_t side = rows < cols ? rows : cols, length = rows < cols ? cols : rows;
    return count > TQ_ORTH_MAX_COUNT || side > TQ_ORTH_MAX_SIDE || length > TQ_ORTH_MAX_LENGTH ? TQ_EUNSUPPORTED : TQ_OK;
}

// Whether the steps keep singular values that begin in [0, 1] where the products' operands hold them: the largest magnitudes of
// s (a + b s^2 + c s^4) and of a + b s^2 + c s^4 for s up to the bound that the steps before leave, at the ends and where they turn.
static bool coefficients_fit(const float* f, int steps)
{
    double bound = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = f[3 * i], b = f[3 * i + 1], c = f[3 * i + 2];
        if (!(fabs(a) <= 12.0) || !(fabs(b) <= 1e3) || !(fabs(c) <= 1e3)) return false;
        const double top = bound * bound;
        double at[4] = {top, top, top, top};                       // of s^2
        if (c != 0.0) {
            at[1] = -b / (2.0 * c);                                // the factor turns
            const double root = 9.0 * b * b - 20.0 * a * c;        // a + 3 b s^2 + 5 c s^4 = 0: the product does
            if (root >= 0.0) {
                at[2] = (-3.0 * b + sqrt(root)) / (10.0 * c);
                at[3] = (-3.0 * b - sqrt(root)) / (10.0 * c);
            }
        } else if (b != 0.0) {
            at[2] = -a / (3.0 * b);
        }
        double next = 0.0;
        for (double s2 : at) {
            if (!(s2 >= 0.0 && s2 <= top)) continue;
            const double p = fabs(a + s2 * (b + s2 * c));
            if (!(p <= 12.0)) return false;
            next = fmax(next, sqrt(s2) * p);
        }
        if (!(next <= 3.0)) return false;
        bound = next;
    }
    return true;
}

static int check_orth(const void* const* g, int count, int dtype, uint64_t rows, uint64_t cols, int steps, const float* coefficients,
                      int precision, float eps, const void* workspace, uint64_t bytes)
{
    int rc;
    if ((rc = check_orth_sizes(rows, cols, count, precision))) return rc;
    if (!g || !known(dtype) || steps < 1 || !usable_eps(eps)) return TQ_EINVAL;
    if (steps > TQ_ORTH_MAX_STEPS) return TQ_EUNSUPPORTED;
    if (coefficients && !coefficients_fit(coefficients, steps)) return TQ_EINVAL;
    for (int i = 0; i < count; ++i) {
        if (!g[i]) return TQ_EINVAL;
        if (!aligned(g[i], size_of(dtype))) return TQ_EALIGN;
    }
    return check_workspace(workspace, bytes, tq_orth_workspace_bytes_impl(rows, cols, count, precision));
}

uint64_t tq_orthogonalize_workspace_bytes(uint64_t rows, uint64_t cols, int count, int precision)
{
    return check_orth_sizes(rows, cols, count, precision) ? 0 : tq_orth_workspace_bytes_impl(rows, cols, count, precision);
}

int tq_orthogonalize_multi(const void* const* g_host, int count, int dtype, uint64_t rows, uint64_t cols, int steps,
                           const float* coefficients_host, int precision, float eps, void* const* out_host, int out_dtype,
                           void* workspace_dev, uint64_t workspace_bytes, void* stream)
{
    const int rc = check_orth(g_host, count, dtype, rows, cols, steps, coefficients_host, precision, eps, workspace_dev, workspace_bytes);
    if (rc) return rc;
    if (!out_host || !known(out_dtype)) return TQ_EINVAL;
    for (int i = 0; i < count; ++i) {
        if (!out_host[i] || (out_host[i] == g_host[i] && out_dtype != dtype)) return TQ_EINVAL;
        for (int j = 0; j < count; ++j)
            if (j != i && (out_host[i] == g_host[j] || out_host[i] == out_host[j])) return TQ_EINVAL;
        if (!aligned(out_host[i], size_of(out_dtype))) return TQ_EALIGN;
    }
    return from_hip(tq_launch_orth(g_host, count, dtype, rows, cols, 0.0f, 0.0f, 0, 0.0f, 0.0f, steps, coefficients_host, precision, eps,
                                   nullptr, nullptr, nullptr, out_host, out_dtype, workspace_dev, static_cast<hipStream_t>(stream)));
}

int tq_orthogonalize(const void* g_dev, int dtype, uint64_t rows, uint64_t cols, int steps, const float* coefficients_host, int precision,
                     float eps, void* out_dev, int out_dtype, void* workspace_dev, uint64_t workspace_bytes, void* stream)
{
    return tq_orthogonalize_multi(&g_dev, 1, dtype, rows, cols, steps, coefficients_host, precision, eps, &out_dev, out_dtype,
                                  workspace_dev, workspace_bytes, stream);
}

int tq_orthogonal_update_multi(const void* const* g_host, int count, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum,
                               int nesterov, float weight_decay, float scale, int steps, const float* coefficients_host, int precision,
                               float eps, const float* const* velocity_host, float* const* velocity_out_host,
                               const float* const* theta_host, float* const* theta_out_host, void* workspace_dev,
                               uint64_t workspace_bytes, void* stream)
{
    const int rc = check_orth(g_host, count, dtype, rows, cols, steps, coefficients_host, precision, eps, workspace_dev, workspace_bytes);
    if (rc) return rc;
    if (!velocity_host || !velocity_out_host || !theta_host || !theta_out_host || (nesterov != 0 && nesterov != 1)) return TQ_EINVAL;
    if (!isfinite(eta) || !isfinite(momentum) || !isfinite(weight_decay) || !isfinite(scale)) return TQ_EINVAL;
    for (int i = 0; i < count; ++i) {
        const void* mine[5] = {g_host[i], velocity_host[i], velocity_out_host[i], theta_host[i], theta_out_host[i]};
        for (const void* p : mine) {
            if (!p) return TQ_EINVAL;
            if (p != g_host[i] && !aligned(p, 4)) return TQ_EALIGN;
        }
        // what is written is nothing else that any matrix reads or writes, but for its own buffer's old contents
        for (int j = 0; j < count; ++j) {
            const void* v = velocity_out_host[i];
            const void* t = theta_out_host[i];
            if (v == g_host[j] || t == g_host[j] || v == theta_host[j] || t == velocity_host[j] || v == theta_out_host[j]) return TQ_EINVAL;
            if (j != i && (v == velocity_host[j] || v == velocity_out_host[j] || t == theta_host[j] || t == theta_out_host[j])) return TQ_EINVAL;
        }
    }
    return from_hip(tq_launch_orth(g_host, count, dtype, rows, cols, eta, momentum, nesterov, weight_decay, scale, steps, coefficients_host,
                                   precision, eps, velocity_host, velocity_out_host, theta_host,
                                   reinterpret_cast<void* const*>(theta_out_host), TQ_F32, workspace_dev, static_cast<hipStream_t>(stream)));
}

int tq_orthogonal_update(const void* g_dev, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum, int nesterov,
                         float weight_decay, float scale, int steps, const float* coefficients_host, int precision, float eps,
                         const float* velocity_dev, float* velocity_out_dev, const float* theta_dev, float* theta_out_dev,
                         void* workspace_dev, uint64_t workspace_bytes, void* stream)
{
    return tq_orthogonal_update_multi(&g_dev, 1, dtype, rows, cols, eta, momentum, nesterov, weight_decay, scale, steps, coefficients_host,
                                      precision, eps, &velocity_dev, &velocity_out_dev, &theta_dev, &theta_out_dev, workspace_dev,
                                      workspace_bytes, stream);
}

}  // extern "C"
