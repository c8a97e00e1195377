// Newton-Schulz orthogonalisation of a batch of matrices (definition in include/qesgd.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qesgd_mma.cuh"
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

// ------------------------------------------------------------- products ----
// The three products of a step, C = P Q with fp32 sums in tensor memory, by persistent CTAs (or pairs of them) of
// 8 warps: one fills a ring of stages by tiled copies, one thread issues the products, four warps take finished tiles
// out of tensor memory, where the next tile is summed meanwhile.
//   GRAM    A = X X^T: both operands are rows of X.  What is off the diagonal goes to F (fp16), the diagonal to d (fp32).
//   POLY    B = b A + c A A = b (D + F) + c (F F + D F + F D + D D): the product is F F, both operands rows of F (F = F^T).
//   UPDATE  X' = a X + B X: rows of B's part off the diagonal, and X with the contraction across its rows.
// Diagonals stay in fp32 because a matrix with few rows is nearly orthogonal to begin with: then A and B are nearly
// diagonal, and rounding that to fp16 moves all singular values of a row alike (20 x 2000: 2.4e-3 off instead of 1.0e-3,
// before the result's own rounding).  A and B are symmetric: tiles below the diagonal are not computed, the ones above
// are stored twice.
enum Product { GRAM, POLY, UPDATE };

constexpr int WARPS = 8;
constexpr int DEPTH = 64;                     // contraction of a stage: 128 bytes of fp16
constexpr uint32_t OPERAND_BYTES = 128 * 128; // 128 rows (or columns) of a stage

struct ProductArgs {
    uint32_t rows, cols, depth, batch;
    uint32_t tiles_m, tiles_n, tiles;         // tiles of one matrix
    __half *f;                                // GRAM: out, POLY: in
    __half *b;                                // POLY: out
    float *d, *db;                            // diagonals of A and of B
    const __half *hi, *lo;                    // UPDATE: X; lo may be null
    __half *hi_out, *lo_out;                  // UPDATE: X', lo_out may be null
    __nv_bfloat16 *out;                       // UPDATE: the result, of the last step; else null
    uint64_t ld_x, x_stride, ld_a, a_stride, d_stride, ldo, out_stride;
    uint32_t turned, out_vec;
    float ca, cb, cc;
    uint32_t *status;
};

struct Tile {
    uint32_t batch, i, j;
};
template <int MODE>
__device__ __forceinline__ Tile tile_of(uint32_t t, const ProductArgs &a)
{
    Tile x;
    x.batch = t / a.tiles;
    t -= x.batch * a.tiles;
    if (MODE == UPDATE) {
        x.j = t / a.tiles_m;
        x.i = t % a.tiles_m;
    } else {
        x.i = 0;
        while (t >= a.tiles_m - x.i) t -= a.tiles_m - x.i++;
        x.j = x.i + t;
    }
    return x;
}

__device__ __forceinline__ uint32_t half_pair(float a, float b)
{
    const __half2 h = __halves2half2(to_half(a), to_half(b));
    return *reinterpret_cast<const uint32_t *>(&h);
}
// 32 values of a row from column c on; rows are `ld` long, a multiple of 8, and may be written up to there
__device__ __forceinline__ void store_halves(__half *row, uint32_t c, uint64_t ld, const float (&v)[32])
{
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if (c + 8u * g < ld)
            *reinterpret_cast<uint4 *>(row + c + 8 * g) = make_uint4(half_pair(v[8 * g], v[8 * g + 1]), half_pair(v[8 * g + 2], v[8 * g + 3]),
                                                                     half_pair(v[8 * g + 4], v[8 * g + 5]), half_pair(v[8 * g + 6], v[8 * g + 7]));
}

// One row's 32 sums from column c on.
template <int MODE>
__device__ __forceinline__ void finish(float (&v)[32], uint32_t batch, uint32_t row, uint32_t c, bool mirror, const ProductArgs &a)
{
    constexpr float XS = ORTHO_X_SCALE, AS = ORTHO_A_SCALE, BS = ORTHO_B_SCALE;
    if (row >= a.rows || c >= a.cols) return;
    if (MODE == GRAM) {
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            if (c + k == row) {
                a.d[batch * a.d_stride + row] = v[k] * (1.0f / (XS * XS));
                v[k] = 0.0f;
            }
            v[k] *= AS / (XS * XS);
        }
    }
    if (MODE == POLY) {
        const float *const d = a.d + batch * a.d_stride;
        const float di = __ldcg(d + row);
        const __half *const f = a.f + batch * a.a_stride + row * a.ld_a;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (c + 8u * g >= a.ld_a) break;
            const uint4 w = __ldcg(reinterpret_cast<const uint4 *>(f + c) + g);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&u[k / 2]));
                const float fk = (k % 2 ? p.y : p.x) * (1.0f / AS), s = v[8 * g + k] * (1.0f / (AS * AS));
                const uint32_t col = c + 8 * g + k;
                if (col == row) a.db[batch * a.d_stride + row] = a.cb * di + a.cc * (s + di * di);
                v[8 * g + k] = col == row ? 0.0f : BS * (a.cc * (s + (di + __ldcg(d + col)) * fk) + a.cb * fk);
            }
        }
    }
    if (MODE == GRAM || MODE == POLY) {
        __half *const m = (MODE == GRAM ? a.f : a.b) + batch * a.a_stride;
        store_halves(m + row * a.ld_a, c, a.ld_a, v);
        if (mirror)
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (c + k < a.cols) m[(c + k) * a.ld_a + row] = to_half(v[k]);
        return;
    }
    const float linear = (a.ca + __ldcg(a.db + batch * a.d_stride + row)) * (1.0f / XS);
    const uint64_t at = batch * a.x_stride + row * a.ld_x + c;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (c + 8u * g >= a.ld_x) break;
        const uint4 w = __ldcg(reinterpret_cast<const uint4 *>(a.hi + at) + g);
        const uint4 z = a.lo ? __ldcg(reinterpret_cast<const uint4 *>(a.lo + at) + g) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w}, l[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&u[k])), q = __half22float2(*reinterpret_cast<const __half2 *>(&l[k]));
            float &v0 = v[8 * g + 2 * k], &v1 = v[8 * g + 2 * k + 1];
            v0 = linear * (p.x + q.x * (1.0f / ORTHO_LO_SCALE)) + v0 * (1.0f / (BS * XS));
            v1 = linear * (p.y + q.y * (1.0f / ORTHO_LO_SCALE)) + v1 * (1.0f / (BS * XS));
        }
    }
    if (a.out) {
        __nv_bfloat16 *const o = a.out + batch * a.out_stride;
        if (a.turned) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (c + k < a.cols) o[(c + k) * a.ldo + row] = __float2bfloat16_rn(v[k]);
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                __nv_bfloat16 h[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) h[k] = __float2bfloat16_rn(v[8 * g + k]);
                const uint32_t first = c + 8 * g;
                if (a.out_vec && first + 8 <= a.cols) {
                    *reinterpret_cast<uint4 *>(o + row * a.ldo + first) = *reinterpret_cast<const uint4 *>(h);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (first + k < a.cols) o[row * a.ldo + first + k] = h[k];
                }
            }
        }
        return;
    }
    float rest[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        v[k] *= XS;
        rest[k] = (v[k] - __half2float(to_half(v[k]))) * ORTHO_LO_SCALE;
    }
    store_halves(a.hi_out + batch * a.x_stride + row * a.ld_x, c, a.ld_x, v);
    if (a.lo_out) store_halves(a.lo_out + batch * a.x_stride + row * a.ld_x, c, a.ld_x, rest);
}

template <bool PAIR>
struct Shape {
    static constexpr int SIDE = PAIR ? 256 : 128;            // a tile is square
    static constexpr int STAGES = 6;
    static constexpr uint32_t STAGE_BYTES = 2 * OPERAND_BYTES;   // of one CTA: 128 rows of either operand
    static constexpr uint32_t COLUMNS = 2 * SIDE;            // of tensor memory: two tiles
    static constexpr uint32_t SMEM = STAGES * STAGE_BYTES + 1024 + 256;
};

template <int MODE, bool PAIR>
__global__ __launch_bounds__(WARPS * 32, 1) void qesgd_ortho_product_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ CUtensorMap map_p,
                                                                            const __grid_constant__ CUtensorMap map_q)
{
    using S = Shape<PAIR>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    // barriers behind the stages: full[STAGES], empty[STAGES], done[2], free[2]; then the base of the tensor memory
    const uint32_t bars = base + S::STAGES * S::STAGE_BYTES;
    const uint32_t full = bars, empty = bars + 8 * S::STAGES, done = empty + 8 * S::STAGES, free_ = done + 16, slot = free_ + 16;
    volatile uint32_t *const stop = reinterpret_cast<volatile uint32_t *>(raw + (slot + 8 - smem_u32(raw)));
    const uint32_t warp = threadIdx.x / 32u, lane = threadIdx.x % 32u;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const uint32_t group = PAIR ? blockIdx.x / 2u : blockIdx.x, groups = PAIR ? gridDim.x / 2u : gridDim.x;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(full + 8 * s), "r"(1u) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(empty + 8 * s), "r"(1u) : "memory");
        }
        for (int s = 0; s < 2; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(done + 8 * s), "r"(1u) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(free_ + 8 * s), "r"(PAIR ? 8u : 4u) : "memory");
        }
        *stop = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        prefetch_map(&map_p);
        prefetch_map(&map_q);
    }
    if (PAIR) cluster_sync_all();   // both CTAs of the pair are there
    if (warp == 2) tmem_alloc<PAIR>(slot, S::COLUMNS);
    fence_before_sync();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(raw + (slot - smem_u32(raw)));
    const uint32_t all = a.tiles * a.batch, steps = (a.depth + DEPTH - 1) / DEPTH;
    qesgd_wait_for_previous();

    if (warp == 0 && elect_one()) {
        uint32_t n = 0;
        const uint32_t full_lead = PAIR ? map_shared(full, 0) : full;
        for (uint32_t t = group; t < all && !*stop; t += groups) {
            const Tile x = tile_of<MODE>(t, a);
            const uint32_t row = x.i * S::SIDE + rank * 128u, col = x.j * S::SIDE + rank * 128u;
            for (uint32_t k = 0; k < steps; ++k, ++n) {
                const uint32_t s = n % S::STAGES, to = base + s * S::STAGE_BYTES;
                if (n >= S::STAGES && !pipe_wait(empty + 8 * s, (n / S::STAGES - 1u) & 1u, stop)) break;
                if (rank == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full + 8 * s), "r"(S::STAGE_BYTES * (PAIR ? 2u : 1u)) : "memory");
                tma_load_3d<PAIR>(to, &map_p, k * DEPTH, row, x.batch, full_lead + 8 * s);
                if (MODE == UPDATE) {
                    tma_load_3d<PAIR>(to + OPERAND_BYTES, &map_q, col, k * DEPTH, x.batch, full_lead + 8 * s);
                    tma_load_3d<PAIR>(to + OPERAND_BYTES + OPERAND_BYTES / 2, &map_q, col + 64u, k * DEPTH, x.batch, full_lead + 8 * s);
                } else {
                    tma_load_3d<PAIR>(to + OPERAND_BYTES, &map_q, k * DEPTH, col, x.batch, full_lead + 8 * s);
                }
            }
        }
        if (*stop) drain();
    } else if (warp == 1 && rank == 0 && elect_one()) {
        // fp16 operands, fp32 sums, SIDE x SIDE; Q of UPDATE has its contraction across the rows
        constexpr uint32_t INSTRUCTION = 1u << 4 | (MODE == UPDATE ? 1u << 16 : 0u) | (uint32_t)(S::SIDE / 8) << 17 | (uint32_t)(S::SIDE / 16) << 24;
        uint32_t n = 0, done_tiles = 0;
        for (uint32_t t = group; t < all && !*stop; t += groups, ++done_tiles) {
            const uint32_t half = done_tiles & 1u, sums = tmem + half * S::SIDE;
            if (done_tiles >= 2 && !pipe_wait(free_ + 8 * half, (done_tiles / 2 - 1u) & 1u, stop)) break;
            fence_after_sync();
            bool ok = true;
            for (uint32_t k = 0; k < steps; ++k, ++n) {
                const uint32_t s = n % S::STAGES, from = base + s * S::STAGE_BYTES;
                ok = pipe_wait(full + 8 * s, (n / S::STAGES) & 1u, stop);
                if (!ok) break;
                fence_after_sync();
#pragma unroll
                for (uint32_t i = 0; i < DEPTH / 16; ++i) {
                    const uint64_t p = swizzled_matrix(from + i * 32u, 16u, 1024u);
                    const uint64_t q = MODE == UPDATE ? swizzled_matrix(from + OPERAND_BYTES + i * 2048u, OPERAND_BYTES / 2, 1024u)
                                                      : swizzled_matrix(from + OPERAND_BYTES + i * 32u, 16u, 1024u);
                    mma_f16<PAIR>(sums, p, q, INSTRUCTION, k > 0 || i > 0);
                }
                mma_commit<PAIR>(empty + 8 * s);
            }
            if (!ok) break;
            mma_commit<PAIR>(done + 8 * half);
        }
        if (*stop) drain();
    } else if (warp >= 4) {
        const uint32_t quarter = warp % 4u;
        const uint32_t free_lead = PAIR ? map_shared(free_, 0) : free_;
        uint32_t done_tiles = 0;
        for (uint32_t t = group; t < all; t += groups, ++done_tiles) {
            const Tile x = tile_of<MODE>(t, a);
            const uint32_t half = done_tiles & 1u;
            if (!__all_sync(FULL, pipe_wait(done + 8 * half, (done_tiles / 2) & 1u, stop))) break;
            fence_after_sync();
            const uint32_t row = x.i * S::SIDE + rank * 128u + quarter * 32u + lane;
            for (uint32_t c = 0; c < S::SIDE; c += 32) {
                float v[32];
                __syncwarp();
                tmem_load32(tmem + (quarter * 32u << 16) + half * S::SIDE + c, v);
                tmem_wait_load();
                if (c + 32 == S::SIDE) {   // the last of the tile is in registers
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR) mbar_arrive_cluster(free_lead + 8 * half);
                        else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(free_ + 8 * half) : "memory");
                    }
                }
                finish<MODE>(v, x.batch, row, x.j * S::SIDE + c, MODE != UPDATE && x.i != x.j, a);
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && *stop) atomicOr(a.status, QESGD_STATUS_TIMEOUT);
    fence_before_sync();
    if (PAIR) cluster_sync_all();
    fence_after_sync();
    if (warp == 2) tmem_dealloc<PAIR>(tmem, S::COLUMNS);
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

// fp16 matrices [batch][rows][ld] of `cols` columns; a box is 64 columns of `box_rows` rows, 128-byte rows swizzled.
bool half_map(CUtensorMap *map, const void *p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t batch, uint64_t stride, uint32_t box_rows)
{
    const QesgdEncodeTiledFn encode = qesgd_encode_tiled();
    const cuuint64_t dims[3] = {cols, rows, batch}, strides[2] = {ld * 2, stride * 2};
    const cuuint32_t box[3] = {64u, box_rows, 1u}, unit[3] = {1u, 1u, 1u};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3u, const_cast<void *>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, bool PAIR>
cudaError_t launch_product(ProductArgs a, const CUtensorMap &p, const CUtensorMap &q, int sm_count, cudaStream_t stream)
{
    using S = Shape<PAIR>;
    const auto kernel = qesgd_ortho_product_kernel<MODE, PAIR>;
    a.tiles_m = (a.rows + S::SIDE - 1) / S::SIDE;
    a.tiles_n = (a.cols + S::SIDE - 1) / S::SIDE;
    a.tiles = MODE == UPDATE ? a.tiles_m * a.tiles_n : a.tiles_m * (a.tiles_m + 1) / 2;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return e;
    const uint32_t all = a.tiles * a.batch, most = (uint32_t)sm_count / (PAIR ? 2u : 1u);
    return qesgd_launch_cluster(kernel, dim3((all < most ? all : most) * (PAIR ? 2u : 1u)), dim3(WARPS * 32), S::SMEM, PAIR ? 2u : 1u, stream, a, p, q);
}
template <int MODE>
cudaError_t launch_product(const ProductArgs &a, const CUtensorMap &p, const CUtensorMap &q, int sm_count, cudaStream_t stream)
{
    // pairs where they fill most of the SMs
    const uint64_t m = (a.rows + 255) / 256, n = (a.cols + 255) / 256;
    const uint64_t pairs = (MODE == UPDATE ? m * n : m * (m + 1) / 2) * a.batch;
    return pairs * 2 >= (uint64_t)sm_count ? launch_product<MODE, true>(a, p, q, sm_count, stream) : launch_product<MODE, false>(a, p, q, sm_count, stream);
}

}  // namespace

int qesgd_launch_orthogonalize(const OrthoArgs &a, int sm_count, cudaStream_t stream, int *launched)
{
    const OrthoLayout l = qesgd_ortho_layout(a.rows, a.cols, a.batch);
    const auto at = [&](uint64_t off) { return reinterpret_cast<__half *>(a.workspace + off); };
    CUtensorMap rows[2], across[2], f, b;   // X by rows, X across them, F, B
    bool ok = half_map(&f, at(l.off_a), l.m, l.m, l.ld_a, a.batch, l.a_stride, 128) && half_map(&b, at(l.off_b), l.m, l.m, l.ld_a, a.batch, l.a_stride, 128);
    for (int i = 0; i < 2; ++i)
        ok = ok && half_map(&rows[i], at(l.off_hi[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, 128) &&
             half_map(&across[i], at(l.off_hi[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, DEPTH);
    if (!ok) return (int)cudaErrorInvalidValue;
    cudaError_t e = a.dtype == QESGD_F32 ? start<float>(a, l, stream) : a.dtype == QESGD_BF16 ? start<__nv_bfloat16>(a, l, stream) : start<__half>(a, l, stream);
    if (e != cudaSuccess) return (int)e;
    *launched = 2;
    for (uint32_t step = 0; step < a.steps; ++step) {
        const uint32_t now = step % 2, next = 1 - now;
        ProductArgs p = {};
        p.batch = (uint32_t)a.batch;
        p.f = at(l.off_a);
        p.b = at(l.off_b);
        p.d = reinterpret_cast<float *>(a.workspace + l.off_d);
        p.db = p.d + a.batch * l.d_stride;
        p.ld_x = l.ld_x;
        p.x_stride = l.x_stride;
        p.ld_a = l.ld_a;
        p.a_stride = l.a_stride;
        p.d_stride = l.d_stride;
        p.ca = a.a;
        p.cb = a.b;
        p.cc = a.c;
        p.status = a.status;
        p.rows = p.cols = (uint32_t)l.m;
        p.depth = (uint32_t)l.n;
        e = launch_product<GRAM>(p, rows[now], rows[now], sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
        p.depth = (uint32_t)l.m;
        e = launch_product<POLY>(p, f, f, sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
        p.cols = (uint32_t)l.n;
        p.hi = at(l.off_hi[now]);
        p.lo = step < ORTHO_LO_STEPS ? at(l.off_lo[now]) : nullptr;
        p.hi_out = at(l.off_hi[next]);
        p.lo_out = step + 1 < ORTHO_LO_STEPS ? at(l.off_lo[next]) : nullptr;
        if (step + 1 == a.steps) {
            p.out = static_cast<__nv_bfloat16 *>(a.out);
            p.ldo = a.ldo;
            p.out_stride = a.out_stride;
            p.turned = a.rows > a.cols;
            p.out_vec = qesgd_aligned(a.out, 16) && a.ldo % 8 == 0 && a.out_stride % 8 == 0;
        }
        e = launch_product<UPDATE>(p, b, across[now], sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
    }
    return 0;
}
