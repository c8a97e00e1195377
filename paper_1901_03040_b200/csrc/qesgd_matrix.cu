// C ABI of the matrix operators: argument checks and dispatch.  Contracts are stated in include/qesgd.h.
#include "qesgd_internal.h"
#include "qesgd_orthogonalize.h"

namespace {

inline uint64_t element_bytes(uint32_t dtype) { return dtype == QESGD_F32 ? 4 : 2; }

// A call's plan becomes the context's where the call went through.
struct Plan {
    qesgd_ctx *ctx;
    uint32_t words[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int keep(int e)
    {
        if (e == 0)
            for (int i = 0; i < 8; ++i) ctx->matrix_plan[i] = words[i];
        return e;
    }
};

// A matrix of elements: pointer, row stride.  (rows, cols > 0 here.)
inline bool valid_matrix(const void *p, uint32_t dtype, uint64_t cols, uint64_t ld)
{
    return p && qesgd_aligned(p, element_bytes(dtype)) && ld >= cols && ld <= (1ull << 40);
}
inline bool valid_held(const uint8_t *codes, const uint8_t *scales)
{
    return codes && scales && qesgd_aligned(codes, 16) && qesgd_aligned(scales, 16);
}
inline bool valid_sides(uint64_t a, uint64_t b) { return a <= QESGD_MAX_MATRIX_SIDE && b <= QESGD_MAX_MATRIX_SIDE; }
inline bool rows_aligned(const void *p, uint32_t dtype, uint64_t ld)
{
    return qesgd_aligned(p, 16) && ld * element_bytes(dtype) % 16 == 0;
}
inline bool valid_exponent(const int32_t *e, uint32_t format)
{
    return !e || (format == QESGD_FP4_NV && qesgd_aligned(e, 4));
}

}  // namespace

extern "C" {

uint64_t qesgd_fp4_row_bytes(uint64_t cols)
{
    return cols > QESGD_MAX_MATRIX_SIDE ? 0 : qesgd_div_up(cols, 32) * 16;
}

uint64_t qesgd_fp4_scale_bytes(uint64_t rows, uint64_t cols, uint32_t format)
{
    if (format > QESGD_FP4_NV || !valid_sides(rows, cols)) return 0;
    return qesgd_div_up(rows, 128) * qesgd_div_up(cols, format == QESGD_FP4_MX ? 128 : 64) * 512;
}

int qesgd_fp4_tensor_exponent(qesgd_ctx *ctx, const void *x, uint32_t dtype, uint64_t rows, uint64_t cols,
                              uint64_t ldx, int32_t *exponent_out)
{
    if (!ctx || dtype > QESGD_F16 || !valid_sides(rows, cols)) return QESGD_EINVAL;
    if (rows == 0 || cols == 0) return QESGD_OK;
    if (!valid_matrix(x, dtype, cols, ldx) || !exponent_out || !qesgd_aligned(exponent_out, 4)) return QESGD_EINVAL;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return qesgd_cuda_fail(ctx, (int)cudaErrorInvalidDevice);
    const int e = qesgd_launch_fp4_tensor_exponent(x, dtype, rows, cols, ldx, rows_aligned(x, dtype, ldx), exponent_out,
                                                   ctx->d_status, ctx->sm_count, ctx->stream);
    if (e != 0) return qesgd_cuda_fail(ctx, e);
    ctx->launches += 1;
    return QESGD_OK;
}

int qesgd_fp4_quantize(qesgd_ctx *ctx, const void *x, uint32_t dtype, uint64_t rows, uint64_t cols,
                       uint64_t ldx, uint32_t format, const int32_t *tensor_exponent, uint32_t rounding,
                       uint64_t seed, uint32_t worker, uint32_t epoch, uint8_t *codes_out,
                       uint8_t *scales_out, uint8_t *codes_t_out, uint8_t *scales_t_out)
{
    if (!ctx || dtype > QESGD_F16 || format > QESGD_FP4_NV || rounding > QESGD_ROUND_STOCHASTIC) return QESGD_EINVAL;
    if (!valid_sides(rows, cols) || !valid_exponent(tensor_exponent, format)) return QESGD_EINVAL;
    if (rows == 0 || cols == 0) return QESGD_OK;
    const bool along = codes_out || scales_out, across = codes_t_out || scales_t_out;
    if (!valid_matrix(x, dtype, cols, ldx) || (!along && !across)) return QESGD_EINVAL;
    if ((along && !valid_held(codes_out, scales_out)) || (across && !valid_held(codes_t_out, scales_t_out))) return QESGD_EINVAL;
    Fp4QuantizeArgs a;
    a.x = x;
    a.rows = rows;
    a.cols = cols;
    a.ldx = ldx;
    a.tensor_exponent = tensor_exponent;
    for (uint32_t r = 0; r < 10; ++r) {   // Philox4x32 key schedule (Weyl sequence)
        a.round_key[r][0] = (uint32_t)seed + r * 0x9E3779B9u;
        a.round_key[r][1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
    a.worker = worker;
    a.epoch = epoch;
    a.codes = codes_out;
    a.scales = scales_out;
    a.codes_t = codes_t_out;
    a.scales_t = scales_t_out;
    a.vec = rows_aligned(x, dtype, ldx) ? 1u : 0u;
    a.status = ctx->d_status;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return qesgd_cuda_fail(ctx, (int)cudaErrorInvalidDevice);
    Plan plan = {ctx};
    const int e = plan.keep(qesgd_launch_fp4_quantize(a, dtype, format, rounding == QESGD_ROUND_STOCHASTIC, ctx->sm_count, ctx->stream, plan.words));
    if (e != 0) return qesgd_cuda_fail(ctx, e);
    ctx->launches += 1;
    return QESGD_OK;
}

int qesgd_fp4_dequantize(qesgd_ctx *ctx, const uint8_t *codes, const uint8_t *scales, uint64_t rows,
                         uint64_t cols, uint32_t format, const int32_t *tensor_exponent, void *out,
                         uint32_t dtype, uint64_t ldo)
{
    if (!ctx || dtype > QESGD_F16 || format > QESGD_FP4_NV) return QESGD_EINVAL;
    if (!valid_sides(rows, cols) || !valid_exponent(tensor_exponent, format)) return QESGD_EINVAL;
    if (rows == 0 || cols == 0) return QESGD_OK;
    if (!valid_matrix(out, dtype, cols, ldo) || !valid_held(codes, scales)) return QESGD_EINVAL;
    Fp4DequantizeArgs a;
    a.codes = codes;
    a.scales = scales;
    a.rows = rows;
    a.cols = cols;
    a.ldo = ldo;
    a.tensor_exponent = tensor_exponent;
    a.out = out;
    a.vec = rows_aligned(out, dtype, ldo) ? 1u : 0u;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return qesgd_cuda_fail(ctx, (int)cudaErrorInvalidDevice);
    const int e = qesgd_launch_fp4_dequantize(a, dtype, format, ctx->stream);
    if (e != 0) return qesgd_cuda_fail(ctx, e);
    ctx->launches += 1;
    return QESGD_OK;
}

int qesgd_fp4_matmul(qesgd_ctx *ctx, const uint8_t *a_codes, const uint8_t *a_scales,
                     const int32_t *a_exponent, const uint8_t *b_codes, const uint8_t *b_scales,
                     const int32_t *b_exponent, uint64_t M, uint64_t N, uint64_t K, uint32_t format,
                     void *c, uint32_t dtype, uint64_t ldc, uint32_t accumulate)
{
    if (!ctx || dtype > QESGD_F16 || format > QESGD_FP4_NV) return QESGD_EINVAL;
    if (!valid_sides(M, N) || !valid_sides(K, 0)) return QESGD_EINVAL;
    if (!valid_exponent(a_exponent, format) || !valid_exponent(b_exponent, format)) return QESGD_EINVAL;
    if (M == 0 || N == 0 || (K == 0 && accumulate)) return QESGD_OK;
    if (!valid_matrix(c, dtype, N, ldc)) return QESGD_EINVAL;
    if (K > 0 && (!valid_held(a_codes, a_scales) || !valid_held(b_codes, b_scales))) return QESGD_EINVAL;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return qesgd_cuda_fail(ctx, (int)cudaErrorInvalidDevice);
    const Fp4MatmulArgs a = {a_codes, a_scales, b_codes, b_scales, a_exponent, b_exponent, M, N, K, ldc, c, accumulate ? 1u : 0u, ctx->d_status};
    int launched = 0;
    Plan plan = {ctx};
    const int e = plan.keep(qesgd_launch_fp4_matmul(a, dtype, format, ctx->sm_count, ctx->stream, &launched, plan.words));
    ctx->launches += (uint64_t)launched;
    if (e != 0) return qesgd_cuda_fail(ctx, e);
    return QESGD_OK;
}

uint64_t qesgd_orthogonalize_workspace(uint64_t rows, uint64_t cols, uint64_t batch)
{
    if (rows > QESGD_MAX_ORTHO_SIDE || cols > QESGD_MAX_ORTHO_SIDE || batch > QESGD_MAX_ORTHO_BATCH) return 0;
    if (rows == 0 || cols == 0 || batch == 0) return 0;
    return qesgd_ortho_layout(rows, cols, batch).bytes;
}

int qesgd_orthogonalize(qesgd_ctx *ctx, const void *x, uint32_t dtype, uint64_t rows, uint64_t cols, uint64_t ldx,
                        uint64_t batch, uint64_t x_stride, uint32_t steps, float a, float b, float c,
                        void *out, uint64_t ldo, uint64_t out_stride, void *workspace,
                        uint64_t workspace_bytes)
{
    if (!ctx || dtype > QESGD_F16 || rows > QESGD_MAX_ORTHO_SIDE || cols > QESGD_MAX_ORTHO_SIDE) return QESGD_EINVAL;
    if (batch > QESGD_MAX_ORTHO_BATCH || steps < 1 || steps > QESGD_MAX_ORTHO_STEPS) return QESGD_EINVAL;
    if (!(a >= -16.0f && a <= 16.0f && b >= -32.0f && b <= 32.0f && c >= -32.0f && c <= 32.0f)) return QESGD_EINVAL;
    if (rows == 0 || cols == 0 || batch == 0) return QESGD_OK;
    if (!valid_matrix(x, dtype, cols, ldx) || !valid_matrix(out, QESGD_BF16, cols, ldo)) return QESGD_EINVAL;
    if (x_stride > (1ull << 40) || out_stride > (1ull << 40)) return QESGD_EINVAL;
    if (batch > 1 && (x_stride < (rows - 1) * ldx + cols || out_stride < (rows - 1) * ldo + cols)) return QESGD_EINVAL;
    if (!workspace || !qesgd_aligned(workspace, 256) || workspace_bytes < qesgd_ortho_layout(rows, cols, batch).bytes) return QESGD_EINVAL;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return qesgd_cuda_fail(ctx, (int)cudaErrorInvalidDevice);
    const OrthoArgs o = {x, dtype, rows, cols, ldx, batch, batch > 1 ? x_stride : 0, steps, a, b, c, out, ldo,
                         batch > 1 ? out_stride : 0, static_cast<uint8_t *>(workspace), ctx->d_status};
    int launched = 0;
    Plan plan = {ctx};
    const int e = plan.keep(qesgd_launch_orthogonalize(o, ctx->sm_count, ctx->stream, &launched, plan.words));
    ctx->launches += (uint64_t)launched;
    if (e != 0) return qesgd_cuda_fail(ctx, e);
    return QESGD_OK;
}

}  // extern "C"
