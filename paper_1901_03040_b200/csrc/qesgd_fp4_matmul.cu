// C = A B^T on microscaled 4-bit operands (layout in include/qesgd.h), on the tensor cores' block-scaled products.
//
// Rows of B lie along the 128 lanes of tensor memory and rows of A along its columns, so that a warp that takes a finished
// tile out holds 32 neighbouring elements of a row of C for each of its registers: stores of 64 or 128 consecutive bytes,
// whatever C's alignment, and a single token fills the lanes with the weight's rows.
//
// A stage is a contraction of 256: 128 bytes of codes of each row, and the tiles of scales as they lie in memory (128 rows by 4
// blocks, 512 bytes), which go on to tensor memory in the same order.  Every stage has columns of its own for its scales, so
// that the thread that issues products need not wait for earlier ones before it copies scales (with two sets in turn, and
// that wait, 8192^3 took 224 us instead of 202).  What lies outside the matrices arrives as zeros.
#include "qesgd_matrix.cuh"
#include "qesgd_mma.cuh"

namespace {

constexpr int TAKERS = 16;                // warps that take tiles out: four for each quarter of tensor memory
constexpr int WARPS = 4 + TAKERS;         // before them: copies, products, tensor memory, one without work
constexpr uint32_t DEPTH = 256;           // contraction of a stage
constexpr uint32_t LANES = 128;           // rows of B of a CTA
constexpr uint32_t SCALE_TILE = 512;

// PAIR: two CTAs on 256 rows of B by 256 of A, one tile in tensor memory at a time (its other half holds scales).
// Else 128 rows of B by 32, 64 or 128 of A, two tiles in tensor memory, and the contraction shared out to a cluster.
template <bool PAIR>
struct Shape {
    static constexpr uint32_t MOST_Q = PAIR ? 256 : 128;      // rows of A of a tile
    static constexpr uint32_t HELD_Q = 128;                   // rows of A in a CTA's shared memory
    static constexpr uint32_t TILES = PAIR ? 1 : 2;           // in tensor memory
    static constexpr int STAGES = PAIR ? 5 : 6;
    static constexpr uint32_t SCALES_P = 2048, SCALES_Q = MOST_Q / 128 * 2048;   // bytes of a stage at most (NV)
    static constexpr uint32_t STAGE_BYTES = LANES * 128 + HELD_Q * 128 + SCALES_P + SCALES_Q;
    static constexpr uint32_t SMEM = STAGES * STAGE_BYTES + 1024 + 256;
    static constexpr uint32_t COLUMNS = 512;
    static constexpr uint32_t SCALE_COLUMN = TILES * MOST_Q;  // a set of scales for each stage behind the tiles
    static constexpr uint32_t SET = 16 + MOST_Q / 128 * 16;
    static_assert(SCALE_COLUMN + STAGES * SET <= COLUMNS, "tensor memory");
};

struct ProductArgs {
    uint32_t M, N, steps, split;              // split: CTAs of a cluster that share the contraction
    uint32_t q;                               // rows of A of a tile
    uint32_t tiles_n, tiles;
    const int32_t *a_exponent, *b_exponent;
    void *c;
    uint64_t ldc;
    uint32_t pairs;                           // rows of 16-bit elements that lie on 4 bytes
    uint32_t *status;
};

// Column n of COUNT rows of C from row m on: what is there, and what comes there.
template <typename T, int COUNT>
__device__ __forceinline__ void load_column(float (&old)[COUNT], uint32_t m, uint32_t n, const ProductArgs &a)
{
    if (n >= a.N || m >= a.M) return;
    const T *c = static_cast<const T *>(a.c) + (m * a.ldc + n);
    if (m + COUNT <= a.M) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k, c += a.ldc) old[k] = to_float(*c);
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k, c += a.ldc) old[k] = m + k < a.M ? to_float(*c) : 0.0f;
    }
}
// Two floats as two 16-bit elements, the first below.
__device__ __forceinline__ uint32_t packed(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t packed(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// For 32 lanes on 32 neighbouring columns, all inside, COUNT rows, all inside, rows on 4 bytes: neighbouring lanes
// exchange an element each, and store two of one row at a time, the even lanes in even rows, the odd ones in odd rows.
template <typename T, int COUNT>
__device__ __forceinline__ void store_column_pairs(const float (&v)[COUNT], T *c, uint32_t lane, const ProductArgs &a)
{
    const bool odd = lane & 1u;
    c += odd ? (int64_t)a.ldc - 1 : 0;
#pragma unroll
    for (int k = 0; k < COUNT; k += 2, c += 2 * a.ldc) {
        const float other = __shfl_xor_sync(0xFFFFFFFFu, odd ? v[k] : v[k + 1], 1);
        *reinterpret_cast<uint32_t *>(c) = odd ? packed(other, v[k + 1], T()) : packed(v[k], other, T());
    }
}
// All lanes of a warp come here; n is the lane's own column.
template <typename T, int COUNT>
__device__ __forceinline__ void store_column(const float (&v)[COUNT], uint32_t m, uint32_t n, const ProductArgs &a)
{
    T *c = static_cast<T *>(a.c) + (m * a.ldc + n);
    if constexpr (sizeof(T) == 2 && COUNT % 2 == 0) {
        const uint32_t lane = threadIdx.x % 32u;
        if (a.pairs && n - lane + 32u <= a.N && m + COUNT <= a.M) {
            store_column_pairs(v, c, lane, a);
            return;
        }
    }
    if (n >= a.N || m >= a.M) return;
    if (m + COUNT <= a.M) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k, c += a.ldc) *c = from_float<T>(v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k, c += a.ldc)
            if (m + k < a.M) *c = from_float<T>(v[k]);
    }
}
// 2^(ta + tb), in two factors where it is no 32-bit number.
struct Power {
    float first, second;
};
__device__ __forceinline__ Power power_of(const ProductArgs &a)
{
    const int ta = a.a_exponent ? min(max(__ldcg(a.a_exponent), -126), 126) : 0, tb = a.b_exponent ? min(max(__ldcg(a.b_exponent), -126), 126) : 0;
    const int t = ta + tb, first = t < -126 ? -126 : t > 126 ? 126 : t;
    return {__uint_as_float((uint32_t)(first + 127) << 23), __uint_as_float((uint32_t)(t - first + 127) << 23)};
}
template <int COUNT>
__device__ __forceinline__ void times(float (&v)[COUNT], const Power &p)
{
#pragma unroll
    for (int k = 0; k < COUNT; ++k) v[k] *= p.first;
    if (p.second != 1.0f)
#pragma unroll
        for (int k = 0; k < COUNT; ++k) v[k] *= p.second;
}

template <typename T, bool PAIR, bool MX, bool ACCUMULATE>
__global__ __launch_bounds__(WARPS * 32, 1) void qesgd_fp4_matmul_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ CUtensorMap map_p,
                                                                         const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_sp,
                                                                         const __grid_constant__ CUtensorMap map_sq)
{
    using S = Shape<PAIR>;
    constexpr uint32_t SCALE_TILES = MX ? 2 : 4;                     // tiles of scales along a stage
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bars = base + S::STAGES * S::STAGE_BYTES;
    const uint32_t full = bars, empty = bars + 8 * S::STAGES, done = empty + 8 * S::STAGES, free_ = done + 16, slot = free_ + 16;
    volatile uint32_t *const stop = reinterpret_cast<volatile uint32_t *>(raw + (slot + 8 - smem_u32(raw)));
    const uint32_t warp = threadIdx.x / 32u, lane = threadIdx.x % 32u;
    const uint32_t share = PAIR ? 2u : a.split;                      // CTAs of a cluster
    const uint32_t rank = share > 1 ? cluster_rank() : 0u;
    const uint32_t group = blockIdx.x / share, groups = gridDim.x / share;
    const uint32_t q_rows = PAIR ? S::MOST_Q : a.q;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(full + 8 * s), "r"(1u) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(empty + 8 * s), "r"(1u) : "memory");
        }
        for (int s = 0; s < 2; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(done + 8 * s), "r"(1u) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(free_ + 8 * s), "r"(PAIR ? 2u * TAKERS : (uint32_t)TAKERS) : "memory");
        }
        *stop = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        prefetch_map(&map_p);
        prefetch_map(&map_q);
        prefetch_map(&map_sp);
        prefetch_map(&map_sq);
    }
    // Both CTAs of a pair are there, and their barriers.  (The first product of a pair waits for copies that its other CTA
    // sets off behind its own part of the allocation.)
    if (PAIR) cluster_sync_all();
    if (warp == 2) tmem_alloc<PAIR>(slot, S::COLUMNS);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(raw + (slot - smem_u32(raw)));
    // this CTA's part of the contraction (of a pair: all of it).  Those who share one leave two stages to what they send
    // one another: each sums up every parts-th row of A, and receives the others' parts of it.
    const uint32_t part = PAIR ? 0u : rank, parts = PAIR ? 1u : share;
    const uint32_t stages = parts > 1 ? S::STAGES - 2u : S::STAGES, received = base + stages * S::STAGE_BYTES;
    const uint32_t every = (q_rows + parts - 1u) / parts;            // rows of A that a CTA sums up, at most
    bool joined = PAIR || parts == 1;                                // has this warp seen that all of the cluster are there?
    if (!joined) cluster_arrive();
    const uint32_t steps = (a.steps - part + parts - 1u) / parts;    // dealt out in turn, so that neighbours read neighbouring bytes
    qesgd_wait_for_previous();

    if (warp == 0 && elect_one()) {
        uint32_t s = 0, turn = 0;   // the stage, and how often all of them have been gone through
        const uint32_t full_lead = PAIR ? map_shared(full, 0) : full;
        const uint32_t bytes = (LANES + (PAIR ? S::HELD_Q : q_rows)) * 128u + SCALE_TILES * SCALE_TILE * (1u + S::MOST_Q / 128u);
        for (uint32_t t = group; t < a.tiles && !*stop; t += groups) {
            const uint32_t p0 = t % a.tiles_n * (PAIR ? 256u : 128u) + (PAIR ? rank * 128u : 0u), q0 = t / a.tiles_n * q_rows;
            for (uint32_t k = part; k < a.steps; k += parts) {
                const uint32_t to = base + s * S::STAGE_BYTES, bar = full_lead + 8 * s;
                if (turn > 0 && !pipe_wait(empty + 8 * s, (turn - 1u) & 1u, stop)) break;
                if (!PAIR || rank == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full + 8 * s), "r"(bytes * (PAIR ? 2u : 1u)) : "memory");
                tma_load_2d<PAIR>(to, &map_p, k * 128u, p0, bar);
                tma_load_2d<PAIR>(to + LANES * 128, &map_q, k * 128u, q0 + (PAIR ? rank * 128u : 0u), bar);
                const uint32_t scales = to + (LANES + S::HELD_Q) * 128;
                // in units of 8 bytes
                tma_load_2d<PAIR>(scales, &map_sp, k * SCALE_TILES * (SCALE_TILE / 8), p0 / 128u, bar);
                tma_load_2d<PAIR>(scales + S::SCALES_P, &map_sq, k * SCALE_TILES * (SCALE_TILE / 8), q0 / 128u, bar);
                if (PAIR) tma_load_2d<PAIR>(scales + S::SCALES_P + 2048, &map_sq, k * SCALE_TILES * (SCALE_TILE / 8), q0 / 128u + 1u, bar);
                if (++s == stages) {
                    s = 0;
                    ++turn;
                }
            }
        }
        if (*stop) drain();
    } else if (warp == 1 && (!PAIR || rank == 0) && elect_one()) {
        // E2M1 operands, fp32 sums; scales E8M0 (MX) or E4M3
        const uint32_t instruction = 1u << 7 | 1u << 10 | (q_rows / 8u) << 17 | (MX ? 1u << 23 : 0u) | (PAIR ? 2u : 1u) << 27;
        uint32_t s = 0, phase = 0, done_tiles = 0;
        for (uint32_t t = group; t < a.tiles && !*stop; t += groups, ++done_tiles) {
            const uint32_t which = done_tiles % S::TILES, turn = done_tiles / S::TILES, sums = tmem + which * S::MOST_Q;
            if (turn >= 1 && !pipe_wait(free_ + 8 * which, (turn - 1u) & 1u, stop)) break;
            fence_after_sync();
            bool ok = true;
            for (uint32_t k = 0; k < steps; ++k) {
                const uint32_t from = base + s * S::STAGE_BYTES;
                ok = pipe_wait(full + 8 * s, phase, stop);
                if (!ok) break;
                fence_after_sync();
                const uint32_t scales = from + (LANES + S::HELD_Q) * 128, sp = tmem + S::SCALE_COLUMN + s * S::SET, sq = sp + 16u;
                // rows 0..127 and 128..255 of A lie side by side for each tile of four blocks
#pragma unroll
                for (uint32_t i = 0; i < SCALE_TILES; ++i) {
                    copy_scales<PAIR>(sp + 4 * i, scales + i * SCALE_TILE);
                    copy_scales<PAIR>(sq + (PAIR ? 8 : 4) * i, scales + S::SCALES_P + i * SCALE_TILE);
                    if (PAIR) copy_scales<PAIR>(sq + 8 * i + 4, scales + S::SCALES_P + 2048 + i * SCALE_TILE);
                }
#pragma unroll
                for (uint32_t i = 0; i < DEPTH / 64; ++i) {
                    const uint64_t p = swizzled_matrix(from + i * 32u, 16u, 1024u), q = swizzled_matrix(from + LANES * 128 + i * 32u, 16u, 1024u);
                    const uint32_t at = MX ? i / 2 : i, half = MX ? i % 2 * 2 : 0u;   // MX: two products share a tile of scales
                    mma_fp4<PAIR, MX>(sums, p, q, instruction | half << 4 | half << 29, sp + 4 * at, sq + (PAIR ? 8 : 4) * at, k > 0 || i > 0);
                }
                mma_commit<PAIR>(empty + 8 * s);
                if (++s == stages) {
                    s = 0;
                    phase ^= 1u;
                }
            }
            if (!ok) break;
            mma_commit<PAIR>(done + 8 * which);
        }
        if (*stop) drain();
    } else if (warp >= 4) {
        const uint32_t quarter = warp % 4u, part_of = (warp - 4u) / 4u;
        const uint32_t free_lead = PAIR ? map_shared(free_, 0) : free_;
        const Power power = power_of(a);
        uint32_t done_tiles = 0;
        for (uint32_t t = group; t < a.tiles; t += groups, ++done_tiles) {
            const uint32_t which = done_tiles % S::TILES, turn = done_tiles / S::TILES;
            const uint32_t n = t % a.tiles_n * (PAIR ? 256u : 128u) + (PAIR ? rank * 128u : 0u) + quarter * 32u + lane, m0 = t / a.tiles_n * q_rows;
            const uint32_t from = tmem + (quarter * 32u << 16) + which * S::MOST_Q;
            const uint32_t rows = min(q_rows, a.M - m0);     // of A in this tile
            const bool ends = ACCUMULATE && parts == 1;
            // 16 rows of A after another: their elements of C are on their way before the sums are there, the next ones' while
            // these are stored (32 at a time did not fit the registers: 1531 x 999 x 2347 13.4 us, and 10.2 with half of them
            // in local memory)
            constexpr uint32_t PARTS = S::MOST_Q / 128 * 2;
            const auto part_at = [&](uint32_t i) { return (4 * (i / 2) + part_of) * 32u + i % 2 * 16u; };
            float old[2][16];
            if (ends) load_column<T>(old[0], m0 + part_at(0), n, a);
            if (!__all_sync(0xFFFFFFFFu, pipe_wait(done + 8 * which, turn & 1u, stop))) break;
            fence_after_sync();
            const auto taken = [&]() {   // the tile is in registers
                tmem_wait_load();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_cluster(free_lead + 8 * which);
                    else mbar_arrive_at(free_ + 8 * which);
                }
            };
            if (ends) {
#pragma unroll
                for (uint32_t i = 0; i < PARTS; ++i) {
                    float v[16];
                    __syncwarp();
                    tmem_load16(from + part_at(i), v);
                    if (i + 1 < PARTS && part_at(i + 1) < rows) load_column<T>(old[(i + 1) % 2], m0 + part_at(i + 1), n, a);
                    if (i + 1 == PARTS) taken();
                    else tmem_wait_load();
                    times(v, power);
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] += old[i % 2][k];
                    if (part_at(i) < rows) store_column<T>(v, m0 + part_at(i), n, a);
                }
            } else {
                float v[S::MOST_Q / 128][32];
#pragma unroll
                for (uint32_t i = 0; i < S::MOST_Q / 128; ++i)
                    if ((4 * i + part_of) * 32u < rows) tmem_load32(from + (4 * i + part_of) * 32u, v[i]);
                taken();
                if (!joined) {
                    cluster_wait();
                    joined = true;
                }
#pragma unroll
                for (uint32_t i = 0; i < S::MOST_Q / 128; ++i) {
                    const uint32_t at = (4 * i + part_of) * 32u;
                    if (at >= rows) break;
                    if (PAIR || parts == 1) {
                        times(v[i], power);
                        store_column<T>(v[i], m0 + at, n, a);
                    } else {
                        // row m of the tile to CTA m % parts, as part `rank` of its row m / parts
                        uint32_t owner = at % parts, to = received + ((rank * every + at / parts) * LANES + quarter * 32u + lane) * 4u;
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            if (at + k < rows) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_shared(to, owner)), "f"(v[i][k]) : "memory");
                            if (++owner == parts) {
                                owner = 0;
                                to += LANES * 4u;
                            }
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    if (!PAIR && parts > 1) {
        if (!joined) cluster_wait();
        __syncwarp();
        cluster_sync_all();
        if (!*stop) {
            const uint32_t n = group % a.tiles_n * 128u + threadIdx.x % LANES, m0 = group / a.tiles_n * q_rows;
            const Power power = power_of(a);
            constexpr uint32_t GROUPS = WARPS * 32 / LANES, ROWS = 4;   // a group of threads takes 4 rows at a time
            const uint32_t rows = min(q_rows, a.M - m0);
            for (uint32_t i0 = threadIdx.x / LANES; i0 * parts + rank < rows; i0 += ROWS * GROUPS) {
                float sum[ROWS][1], old[ROWS][1];
#pragma unroll
                for (uint32_t k = 0; k < ROWS; ++k) {
                    const uint32_t row = (i0 + k * GROUPS) * parts + rank;
                    sum[k][0] = old[k][0] = 0.0f;
                    if (ACCUMULATE && row < rows) load_column<T>(old[k], m0 + row, n, a);
                }
                for (uint32_t r = 0; r < parts; ++r)   // in the order of the CTAs
#pragma unroll
                    for (uint32_t k = 0; k < ROWS; ++k) {
                        const uint32_t i = min(i0 + k * GROUPS, every - 1u);
                        float v;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(received + ((r * every + i) * LANES + threadIdx.x % LANES) * 4u));
                        sum[k][0] += v;
                    }
#pragma unroll
                for (uint32_t k = 0; k < ROWS; ++k) {
                    const uint32_t row = (i0 + k * GROUPS) * parts + rank;
                    times(sum[k], power);
                    sum[k][0] += old[k][0];
                    if (row < rows) store_column<T>(sum[k], m0 + row, n, a);
                }
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *stop) atomicOr(a.status, QESGD_STATUS_TIMEOUT);
    fence_before_sync();
    if (PAIR) cluster_sync_all();
    fence_after_sync();
    if (warp == 2) tmem_dealloc<PAIR>(tmem, S::COLUMNS);
}

// A contraction over nothing.
template <typename T>
__global__ __launch_bounds__(256) void qesgd_fp4_zeros_kernel(T *c, uint64_t M, uint64_t N, uint64_t ldc)
{
    qesgd_wait_for_previous();
    for (uint64_t m = blockIdx.y; m < M; m += gridDim.y)
        for (uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x; n < N; n += (uint64_t)gridDim.x * 256) c[m * ldc + n] = T(0);
}
template <typename T>
cudaError_t launch_zeros(const Fp4MatmulArgs &a, cudaStream_t stream)
{
    const uint64_t x = qesgd_div_up(a.N, 256);
    return qesgd_launch(qesgd_fp4_zeros_kernel<T>, dim3((unsigned)(x < 4096 ? x : 4096), (unsigned)(a.M < 65535 ? a.M : 65535)), dim3(256), stream,
                        static_cast<T *>(a.c), a.M, a.N, a.ldc);
}

// rows of `bytes` bytes; a box is 128 bytes of box_rows rows, swizzled
bool codes_map(CUtensorMap *map, const uint8_t *p, uint64_t rows, uint64_t bytes, uint32_t box_rows)
{
    const cuuint64_t dims[2] = {bytes, rows}, strides[1] = {bytes};
    const cuuint32_t box[2] = {128u, box_rows}, unit[2] = {1u, 1u};
    return qesgd_encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2u, const_cast<uint8_t *>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// the tiles of scales of 128 rows as one row of 8-byte elements; a box is what a stage wants of it
bool scales_map(CUtensorMap *map, const uint8_t *p, uint64_t rows, uint64_t K, bool mx)
{
    const uint64_t tiles = qesgd_div_up(K, mx ? 128 : 64);
    const cuuint64_t dims[2] = {tiles * (SCALE_TILE / 8), qesgd_div_up(rows, 128)}, strides[1] = {tiles * SCALE_TILE};
    const cuuint32_t box[2] = {(mx ? 2u : 4u) * (SCALE_TILE / 8), 1u}, unit[2] = {1u, 1u};
    return qesgd_encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT64, 2u, const_cast<uint8_t *>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, bool PAIR, bool MX, bool ACCUMULATE>
int launch(const Fp4MatmulArgs &f, uint32_t q, uint32_t split, int sm_count, cudaStream_t stream)
{
    using S = Shape<PAIR>;
    const auto kernel = qesgd_fp4_matmul_kernel<T, PAIR, MX, ACCUMULATE>;
    const uint64_t row_bytes = qesgd_div_up(f.K, 32) * 16;
    CUtensorMap p, qm, sp, sq;
    if (!qesgd_encode_tiled() || !codes_map(&p, f.b_codes, f.N, row_bytes, 128) || !codes_map(&qm, f.a_codes, f.M, row_bytes, PAIR ? 128u : q) ||
        !scales_map(&sp, f.b_scales, f.N, f.K, MX) || !scales_map(&sq, f.a_scales, f.M, f.K, MX))
        return (int)cudaErrorInvalidValue;
    ProductArgs a = {};
    a.M = (uint32_t)f.M;
    a.N = (uint32_t)f.N;
    a.steps = (uint32_t)qesgd_div_up(f.K, DEPTH);
    a.split = split;
    a.q = q;
    a.tiles_n = (uint32_t)qesgd_div_up(f.N, PAIR ? 256 : 128);
    const uint64_t tiles = a.tiles_n * qesgd_div_up(f.M, q);
    if (tiles > 0x7FFFFFFF) return (int)cudaErrorInvalidValue;
    a.tiles = (uint32_t)tiles;
    a.a_exponent = f.a_exponent;
    a.b_exponent = f.b_exponent;
    a.c = f.c;
    a.ldc = f.ldc;
    a.pairs = sizeof(T) == 2 && qesgd_aligned(f.c, 4) && f.ldc % 2 == 0;
    a.status = f.status;
    static std::atomic<uint64_t> told{0};
    const cudaError_t e = qesgd_prepare(told, (const void *)kernel, S::SMEM, !PAIR);
    if (e != cudaSuccess) return (int)e;
    const uint32_t most = (uint32_t)sm_count / (PAIR ? 2u : 1u), share = PAIR ? 2u : split;
    const uint32_t groups = split > 1 || a.tiles < most ? a.tiles : most;   // a shared contraction: one tile for each cluster
    return (int)qesgd_launch_cluster(kernel, dim3(groups * share), dim3(WARPS * 32), S::SMEM, share, stream, a, p, qm, sp, sq);
}

template <typename T, bool MX, bool ACCUMULATE>
int launch(const Fp4MatmulArgs &a, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    static QesgdClusters known;
    // By modelled clocks: a stage of a pair takes about 700 to arrive and be multiplied, one of a single CTA 450 where others
    // are few, 600 with all SMs at it.  Too few tiles for the SMs: as many CTAs share a contraction as bring it to an end first;
    // adding the parts up takes 2500 and 100 more for each, and a cluster larger than the device runs of them at once for
    // every tile would wait for a second wave.
    const uint32_t q = a.M <= 32 ? 32 : a.M <= 64 ? 64 : 128;
    const uint64_t sms = (uint64_t)sm_count, pairs = qesgd_div_up(a.M, 256) * qesgd_div_up(a.N, 256);
    const uint64_t tiles = qesgd_div_up(a.M, q) * qesgd_div_up(a.N, 128), steps = qesgd_div_up(a.K, DEPTH);
    const auto stage = [&](uint64_t ctas) { return 450 + 150 * (ctas < sms ? ctas : sms) / sms; };
    const uint64_t by_pairs = qesgd_div_up(pairs, sms / 2) * steps * 700 + 1500;
    const void *const kernel = (const void *)qesgd_fp4_matmul_kernel<T, false, MX, ACCUMULATE>;
    uint32_t split = 1;
    uint64_t best = qesgd_div_up(tiles, sms) * steps * stage(tiles);
    static std::atomic<uint64_t> told{0};
    const cudaError_t e = qesgd_prepare(told, kernel, Shape<false>::SMEM, true);
    if (e != cudaSuccess) return (int)e;
    for (uint32_t s = 2; s <= 16 && s <= steps && tiles * s <= sms; ++s) {
        const uint64_t active = qesgd_active_clusters(known, kernel, WARPS * 32, Shape<false>::SMEM, s);
        const uint64_t t = qesgd_div_up(tiles, active) * qesgd_div_up(steps, s) * stage(tiles * s) + 2500 + 100 * s;
        if (t < best) {
            best = t;
            split = s;
        }
    }
    plan[0] = by_pairs < best ? QESGD_MATRIX_PRODUCT_PAIRS : QESGD_MATRIX_PRODUCT_SINGLES;
    plan[1] = by_pairs < best ? 2 : split;
    plan[2] = by_pairs < best ? 256 : q;
    if (by_pairs < best) return launch<T, true, MX, ACCUMULATE>(a, 256, 1, sm_count, stream);
    return launch<T, false, MX, ACCUMULATE>(a, q, split, sm_count, stream);
}

template <typename T>
int launch(const Fp4MatmulArgs &a, uint32_t format, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    if (format == QESGD_FP4_MX) return a.accumulate ? launch<T, true, true>(a, sm_count, stream, plan) : launch<T, true, false>(a, sm_count, stream, plan);
    return a.accumulate ? launch<T, false, true>(a, sm_count, stream, plan) : launch<T, false, false>(a, sm_count, stream, plan);
}

}  // namespace

int qesgd_launch_fp4_matmul(const Fp4MatmulArgs &a, uint32_t dtype, uint32_t format, int sm_count, cudaStream_t stream, int *launched, uint32_t *plan)
{
    int e;
    if (a.K == 0) e = (int)(dtype == QESGD_F32 ? launch_zeros<uint32_t>(a, stream) : launch_zeros<uint16_t>(a, stream));
    else if (dtype == QESGD_F32) e = launch<float>(a, format, sm_count, stream, plan);
    else if (dtype == QESGD_BF16) e = launch<__nv_bfloat16>(a, format, sm_count, stream, plan);
    else e = launch<__half>(a, format, sm_count, stream, plan);
    *launched = e == 0 ? 1 : 0;
    return e;
}
