// Newton-Schulz orthogonalisation of a batch of matrices (definition in include/qesgd.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qesgd_internal.h"
#include "qesgd_orthogonalize.h"

namespace {

constexpr int THREADS = 256;
constexpr uint32_t FULL = 0xFFFFFFFFu;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// Sum of the squares of a part of a matrix, in 64 bits: no 32-bit value's square is out of range, and the sum is the
// same in every run.
template <typename T>
__global__ __launch_bounds__(THREADS) void qesgd_ortho_norm_kernel(const T *x, uint64_t rows, uint64_t cols, uint64_t ldx, uint64_t stride,
                                                                   double *parts)
{
    __shared__ double sums[THREADS / 32];
    qesgd_wait_for_previous();
    const T *const m = x + blockIdx.y * stride;
    const uint64_t per = (rows * cols + gridDim.x - 1) / gridDim.x;
    const uint64_t last = min(rows * cols, per * (blockIdx.x + 1));
    double sum = 0.0;
    for (uint64_t i = per * blockIdx.x + threadIdx.x; i < last; i += THREADS) {
        const double v = to_float(m[i / cols * ldx + i % cols]);
        sum = fma(v, v, sum);
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(FULL, sum, o);
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < THREADS / 32; ++i) sum += sums[i];
        parts[blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
}

__device__ __forceinline__ __half to_half(float v) { return __float2half_rn(fminf(fmaxf(v, -65504.0f), 65504.0f)); }

// X = G / ||G||, with fewer rows than columns, in two terms.
template <typename T>
__global__ __launch_bounds__(THREADS) void qesgd_ortho_start_kernel(const T *x, uint64_t rows, uint64_t cols, uint64_t ldx, uint64_t stride,
                                                                    const double *parts, uint32_t nparts, OrthoView v, uint32_t *status)
{
    __shared__ double inverse;
    qesgd_wait_for_previous();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (uint32_t i = 0; i < nparts; ++i) sum += parts[blockIdx.y * nparts + i];
        const bool fine = sum <= 1.7976931348623157e308;
        if (!fine && blockIdx.x == 0) atomicOr(status, QESGD_STATUS_NONFINITE);
        inverse = fine && sum > 0.0 ? 1.0 / sqrt(sum) : 0.0;
    }
    __syncthreads();
    const double inv = inverse;
    const T *const m = x + blockIdx.y * stride;
    __half *const hi = v.hi + blockIdx.y * v.x_stride, *const lo = v.lo + blockIdx.y * v.x_stride;
    for (uint64_t i = (uint64_t)blockIdx.x * THREADS + threadIdx.x; i < rows * cols; i += (uint64_t)gridDim.x * THREADS) {
        const uint64_t r = i / cols, c = i % cols;
        const float f = inv == 0.0 ? 0.0f : (float)((double)to_float(m[r * ldx + c]) * inv) * ORTHO_X_SCALE;
        const uint64_t at = rows <= cols ? r * v.ld + c : c * v.ld + r;
        hi[at] = to_half(f);
        lo[at] = to_half((f - __half2float(hi[at])) * ORTHO_LO_SCALE);
    }
}

// out = p * (P Q) + q * E, P [M][K], Q element (k, j) at Q[k * qk + j * qj]
struct Simple {
    const __half *P, *Q, *E, *E2;
    uint64_t M, N, K, ldp, qk, qj, lde, ldo, batch_p, batch_q, batch_e, batch_o;
    float p, q, q2;
    __half *hi, *lo;
    __nv_bfloat16 *out;   // last step
    bool turned;
};
__global__ __launch_bounds__(256) void qesgd_ortho_product_kernel(const __grid_constant__ Simple a)
{
    __shared__ float ps[16][65], qs[16][65];
    qesgd_wait_for_previous();
    const uint64_t m0 = (uint64_t)blockIdx.y * 64, n0 = (uint64_t)blockIdx.x * 64, b = blockIdx.z;
    const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (uint64_t k0 = 0; k0 < a.K; k0 += 16) {
        for (uint32_t i = threadIdx.x; i < 64 * 16; i += 256) {
            const uint64_t k = k0 + i % 16, r = m0 + i / 16, c = n0 + i / 16;
            ps[i % 16][i / 16] = k < a.K && r < a.M ? __half2float(a.P[b * a.batch_p + r * a.ldp + k]) : 0.0f;
            qs[i % 16][i / 16] = k < a.K && c < a.N ? __half2float(a.Q[b * a.batch_q + k * a.qk + c * a.qj]) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] += ps[k][ty + 16 * i] * qs[k][tx + 16 * j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const uint64_t r = m0 + ty + 16 * i, c = n0 + tx + 16 * j;
            if (r >= a.M || c >= a.N) continue;
            float v = acc[i][j] * a.p;
            if (a.E) v += a.q * __half2float(a.E[b * a.batch_e + r * a.lde + c]);
            if (a.E2) v += a.q2 * __half2float(a.E2[b * a.batch_e + r * a.lde + c]);
            if (a.out) {
                a.out[b * a.batch_o + (a.turned ? c * a.ldo + r : r * a.ldo + c)] = __float2bfloat16_rn(v);
                continue;
            }
            const __half h = to_half(v);
            a.hi[b * a.batch_o + r * a.ldo + c] = h;
            if (a.lo) a.lo[b * a.batch_o + r * a.ldo + c] = to_half((v - __half2float(h)) * ORTHO_LO_SCALE);
        }
}

template <typename T>
cudaError_t start(const OrthoArgs &a, const OrthoLayout &l, cudaStream_t stream)
{
    const T *const x = static_cast<const T *>(a.x);
    cudaError_t e = qesgd_launch(qesgd_ortho_norm_kernel<T>, dim3(l.parts, (unsigned)a.batch), dim3(THREADS), stream, x, a.rows, a.cols, a.ldx,
                                 a.x_stride, reinterpret_cast<double *>(a.workspace));
    if (e != cudaSuccess) return e;
    const OrthoView v = {reinterpret_cast<__half *>(a.workspace + l.off_hi[0]), reinterpret_cast<__half *>(a.workspace + l.off_lo[0]), l.ld_x, l.x_stride};
    return qesgd_launch(qesgd_ortho_start_kernel<T>, dim3(l.parts, (unsigned)a.batch), dim3(THREADS), stream, x, a.rows, a.cols, a.ldx,
                        a.x_stride, reinterpret_cast<const double *>(a.workspace), l.parts, v, a.status);
}

}  // namespace

int qesgd_launch_orthogonalize(const OrthoArgs &a, int, cudaStream_t stream, int *launched)
{
    const OrthoLayout l = qesgd_ortho_layout(a.rows, a.cols, a.batch);
    cudaError_t e = a.dtype == QESGD_F32 ? start<float>(a, l, stream) : a.dtype == QESGD_BF16 ? start<__nv_bfloat16>(a, l, stream) : start<__half>(a, l, stream);
    *launched = 2;
    __half *const A = reinterpret_cast<__half *>(a.workspace + l.off_a), *const B = reinterpret_cast<__half *>(a.workspace + l.off_b);
    for (uint32_t step = 0; step < a.steps && e == cudaSuccess; ++step) {
        __half *const hi = reinterpret_cast<__half *>(a.workspace + l.off_hi[step % 2]), *const lo = reinterpret_cast<__half *>(a.workspace + l.off_lo[step % 2]);
        __half *const hi2 = reinterpret_cast<__half *>(a.workspace + l.off_hi[(step + 1) % 2]), *const lo2 = reinterpret_cast<__half *>(a.workspace + l.off_lo[(step + 1) % 2]);
        const bool last = step + 1 == a.steps;
        const float xs = ORTHO_X_SCALE, as = ORTHO_A_SCALE, bs = ORTHO_B_SCALE;
        Simple g = {hi, hi, nullptr, nullptr, l.m, l.m, l.n, l.ld_x, 1, l.ld_x, 0, l.ld_a, l.x_stride, l.x_stride, 0, l.a_stride,
                    as / (xs * xs), 0.0f, 0.0f, A, nullptr, nullptr, false};
        const dim3 gm((unsigned)qesgd_div_up(l.m, 64), (unsigned)qesgd_div_up(l.m, 64), (unsigned)a.batch);
        e = qesgd_launch(qesgd_ortho_product_kernel, gm, dim3(256), stream, g);
        if (e != cudaSuccess) break;
        Simple p = {A, A, A, nullptr, l.m, l.m, l.m, l.ld_a, l.ld_a, 1, l.ld_a, l.ld_a, l.a_stride, l.a_stride, l.a_stride, l.a_stride,
                    a.c * bs / (as * as), a.b * bs / as, 0.0f, B, nullptr, nullptr, false};
        e = qesgd_launch(qesgd_ortho_product_kernel, gm, dim3(256), stream, p);
        if (e != cudaSuccess) break;
        const float os = last ? 1.0f : xs;
        Simple x = {B, hi, hi, step < ORTHO_LO_STEPS ? lo : nullptr, l.m, l.n, l.m, l.ld_a, l.ld_x, 1, l.ld_x, last ? a.ldo : l.ld_x,
                    l.a_stride, l.x_stride, l.x_stride, last ? a.out_stride : l.x_stride, os / (bs * xs), a.a * os / xs,
                    a.a * os / (xs * ORTHO_LO_SCALE), hi2, step + 1 < ORTHO_LO_STEPS ? lo2 : nullptr,
                    last ? static_cast<__nv_bfloat16 *>(a.out) : nullptr, a.rows > a.cols};
        const dim3 gx((unsigned)qesgd_div_up(l.n, 64), (unsigned)qesgd_div_up(l.m, 64), (unsigned)a.batch);
        e = qesgd_launch(qesgd_ortho_product_kernel, gx, dim3(256), stream, x);
        *launched += 3;
    }
    return (int)e;
}
