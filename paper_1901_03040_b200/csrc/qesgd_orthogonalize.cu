// Newton-Schulz orthogonalisation of a batch of matrices (definition in include/qesgd.h).
#include "qesgd_matrix.cuh"
#include "qesgd_mma.cuh"
#include "qesgd_orthogonalize.h"

namespace {

constexpr int THREADS = 256;
constexpr uint32_t FULL = 0xFFFFFFFFu;

// Sum over a block; every thread calls it, thread 0 has the sum.  The order of the additions is fixed.
template <int SIZE>
__device__ __forceinline__ double block_sum(double sum)
{
    __shared__ double sums[SIZE / 32];
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(FULL, sum, o);
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < SIZE / 32; ++i) sum += sums[i];
    return sum;
}

// Power of two next to the largest of eight magnitudes, as an exponent that keeps 2^-e a normal number.
__device__ __forceinline__ int octet_exponent(const float (&v)[8])
{
    float top = fmaxf(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))),
                      fmaxf(fmaxf(fabsf(v[4]), fabsf(v[5])), fmaxf(fabsf(v[6]), fabsf(v[7]))));
    return min(max((int)(__float_as_uint(top) >> 23) - 127, -120), 120);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// Sum of the squares of eight elements, in 64 bits.  The squares are taken in 32 bits (four times the conversions to 64 would
// take as long as the loads) of elements scaled by a power of two: none is out of range, whatever the elements.
__device__ __forceinline__ double octet_squares(const float (&v)[8])
{
    const int e = octet_exponent(v);
    const float p = power_of_two(-e);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fmaf(v[k] * p, v[k] * p, sum);
    return (double)sum * __longlong_as_double((long long)(2 * e + 1023) << 52);
}
// What an element of G is multiplied by to become one of X as it is kept: f, after p where that is not 1 (a power of two, since
// the quotient may not be a 32-bit number where its product with G's elements is).  f = 0: a matrix of zeros, or not finite.
struct Normalise {
    float f, p;
};
__device__ __forceinline__ Normalise normalise(double squares)
{
    Normalise n = {0.0f, 1.0f};
    if (squares > 0.0 && squares <= 1.7976931348623157e308) {
        double norm = sqrt(squares);
        const int e = (int)(__double_as_longlong(norm) >> 52) - 1023;   // |e| < 200
        if (e < -100 || e > 100) {
            n.p = e < 0 ? 0x1p100f : 0x1p-100f;
            norm *= (double)n.p;
        }
        n.f = (float)((double)ORTHO_X_SCALE / norm);
    }
    return n;
}
__device__ __forceinline__ void times(float (&v)[8], const Normalise &n)
{
    if (n.p != 1.0f)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= n.p;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = n.f == 0.0f ? 0.0f : v[k] * n.f;
}

// Sum of the squares of a part of a matrix.
template <typename T>
__global__ __launch_bounds__(THREADS) void qesgd_ortho_norm_kernel(const T *x, uint32_t rows, uint32_t cols, uint64_t ldx, uint64_t stride, bool vec,
                                                                   double *parts)
{
    qesgd_wait_for_previous();
    const T *const m = x + blockIdx.y * stride;
    const uint32_t octets = (cols + 7) / 8, all = octets * rows;
    double sum = 0.0;
    for (uint32_t n = blockIdx.x * THREADS + threadIdx.x; n < all; n += gridDim.x * THREADS) {
        float v[8];
        values(load_octet(m + n / octets * ldx, n % octets * 8, cols, vec), v);
        sum += octet_squares(v);
    }
    sum = block_sum<THREADS>(sum);
    if (threadIdx.x == 0) parts[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// Two floats as fp16, cut off at its largest number.
__device__ __forceinline__ uint32_t half_pair(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
// The same without the rounding.
__device__ __forceinline__ float cut_off(float v)
{
    float r;
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(65504.0f));
    return r;
}
__device__ __forceinline__ float2 float_pair(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2 *>(&h)); }
// a * b + c on two floats at once
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ void add(float &a, float &b, float c, float d)
{
    asm("{\n.reg .b64 x, y;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nadd.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
// What rounding two floats to the fp16 pair h has left behind.
__device__ __forceinline__ uint32_t rest_pair(float a, float b, uint32_t h)
{
    const float2 kept = float_pair(h);
    const float2 rest = fma2(kept, make_float2(-1.0f, -1.0f), make_float2(a, b));
    return half_pair(rest.x, rest.y);
}
__device__ __forceinline__ void store_terms(const float (&f)[8], __half *hi, __half *lo)
{
    uint32_t h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        h[k] = half_pair(f[2 * k], f[2 * k + 1]);
        l[k] = rest_pair(f[2 * k], f[2 * k + 1], h[k]);
    }
    *reinterpret_cast<uint4 *>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4 *>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}

// X = G / ||G|| in two terms, turned where G has more rows than columns.  Zeros behind the last column, up to the next octet.
template <typename T, bool TURNED>
__global__ __launch_bounds__(THREADS) void qesgd_ortho_start_kernel(const T *x, uint32_t rows, uint32_t cols, uint64_t ldx, uint64_t stride, bool vec,
                                                                    const double *parts, uint32_t nparts, OrthoView v, uint32_t *status)
{
    __shared__ double squares;
    __shared__ float held[TURNED ? 64 * 65 : 1];
    qesgd_wait_for_previous();
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < nparts; i += THREADS) sum += parts[blockIdx.y * nparts + i];
    sum = block_sum<THREADS>(sum);
    if (threadIdx.x == 0) {
        if (!(sum <= 1.7976931348623157e308) && blockIdx.x == 0) atomicOr(status, QESGD_STATUS_NONFINITE);
        squares = sum;
    }
    __syncthreads();
    const Normalise scale = normalise(squares);
    const T *const m = x + blockIdx.y * stride;
    __half *const hi = v.hi + blockIdx.y * v.x_stride, *const lo = v.lo + blockIdx.y * v.x_stride;
    if (!TURNED) {
        const uint32_t octets = (cols + 7) / 8, all = octets * rows;
        for (uint32_t n = blockIdx.x * THREADS + threadIdx.x; n < all; n += gridDim.x * THREADS) {
            const uint32_t at = all - 1 - n, r = at / octets, c = at % octets * 8;
            // from the end, which L2 still holds of the norm's pass (4096 x 8192: 90 MB from memory in place of 134)
            float f[8];
            values(load_octet(m + r * ldx, c, cols, vec), f);
            times(f, scale);
            store_terms(f, hi + r * v.ld + c, lo + r * v.ld + c);
        }
        return;
    }
    const uint32_t across = (cols + 63) / 64, tiles = (rows + 63) / 64 * across;
    for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const uint32_t r0 = t / across * 64, c0 = t % across * 64;
        const uint32_t c = c0 + threadIdx.x % 64u;
#pragma unroll
        for (uint32_t i = threadIdx.x / 64u; i < 64; i += THREADS / 64)
            held[i * 65 + threadIdx.x % 64u] = r0 + i < rows && c < cols ? to_float(m[(uint64_t)(r0 + i) * ldx + c]) : 0.0f;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 64 * 8; i += THREADS) {
            const uint32_t c = c0 + i / 8, r = r0 + i % 8 * 8;
            if (c < cols && r < v.ld) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = held[(i % 8 * 8 + j) * 65 + i / 8];
                times(f, scale);
                store_terms(f, hi + c * v.ld + r, lo + c * v.ld + r);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------- products ----
// The three products of a step, C = P Q with fp32 sums in tensor memory, by persistent CTAs (or pairs of them):
//   GRAM    A = X X^T: both operands are rows of X.  What is off the diagonal goes to F (fp16), the diagonal to d (fp32).
//   POLY    B = b A + c A A = b (D + F) + c (F F + D F + F D + D D): the product is F F, both operands rows of F (F = F^T).
//   UPDATE  X' = a X + B X: rows of B's part off the diagonal, and X with the contraction across its rows (with `terms` = 2
//           once for each of X's terms, one after the other).
// Diagonals stay in fp32 because a matrix with few rows is nearly orthogonal to begin with: then A and B are nearly
// diagonal, and rounding that to fp16 moves all singular values of a row alike (20 x 2000: 2.4e-3 off instead of 1.0e-3,
// before the result's own rounding).  A and B are symmetric: tiles below the diagonal are not computed, the ones above
// are stored twice.
//
// A CTA's warps: 0 fills a ring of stages with operands by tiled copies; one thread of 1 issues the products; 4 to 19 take
// finished tiles out of tensor memory, where the next tile is summed meanwhile, 64 columns at a time.  What a tile's end
// reads (X in two terms, or F) and what it writes pass through a second ring of 128 x 64 boxes: 2 has them filled by tiled
// copies, the sixteen warps replace each element by its result, 3 has them stored by tiled copies.  (With loads and stores
// by the warps themselves, a row for each lane, the update of 12 x 512 x 2048 took 63 us, three times what its products
// take: 32 rows' segments in one instruction are 32 passes through the load-store unit.)
//
// Five steps on 4096 x 8192 take 2.2 ms, 1.1 PFLOP/s: a stage of GRAM or POLY takes 513 clocks of the tensor cores' 512, so
// the clock under the power cap and whole waves of tiles (136 on 74 pairs) bound it.  An update's contraction is as short
// as the smaller side: at 512 its tiles' ends, which move three terms of X, come to as many bytes of shared memory as its
// stages.  With few tiles it is the chain of fifteen launches, some 6 to 8 us each (500 x 500: 127 us, with three updates' contractions
// taken twice, once for each term of X, and 118 without).
enum Product { GRAM, POLY, UPDATE };

constexpr int TAKERS = 16;                    // warps that take tiles out: four for each quarter of tensor memory
constexpr int WARPS = 4 + TAKERS;
constexpr int DEPTH = 64;                     // contraction of a stage: 128 bytes of fp16
constexpr uint32_t OPERAND_BYTES = 128 * 128; // 128 rows (or columns) of a stage; also a box of the second ring
constexpr uint32_t BOX_COLS = 64;

struct ProductArgs {
    uint32_t rows, cols, depth, batch;
    uint32_t tiles_m, tiles;                  // tiles along the rows of one matrix, and of all of it
    __half *mirror;                           // GRAM: F, POLY: B, for the elements below the diagonal
    float *d, *db;                            // diagonals of A and of B
    uint32_t terms;                           // of Q: 2 where UPDATE's product takes X's second one too
    __nv_bfloat16 *out;                       // UPDATE: the result, of the last step; else null
    uint64_t ld_a, a_stride, d_stride, ldo, out_stride;
    uint32_t split;                           // CTAs of a cluster that share a tile's contraction, one tile for each cluster
    uint32_t turned, out_tiled;                // out_tiled: by tiled copies
    float ca, cb, cc;
    uint32_t *status;
};
// P and Q; what the end of a tile reads (F, or X and its second term) and writes
struct ProductMaps {
    CUtensorMap p, q, q_lo, in, in_lo, out, out_lo;
    CUtensorMap q_narrow;   // Q of narrow tiles, for the launch to choose
};

struct Tile {
    uint32_t batch, row, col;   // col: where its columns begin
    bool mirror;                // above the diagonal: stored below it too
};
template <int MODE, uint32_t SIDE, uint32_t WIDTH>
__device__ __forceinline__ Tile tile_of(uint32_t t, const ProductArgs &a)
{
    Tile x;
    x.batch = t / a.tiles;
    t -= x.batch * a.tiles;
    uint32_t i, j;
    if (MODE == UPDATE) {
        j = t / a.tiles_m;
        i = t % a.tiles_m;
        x.col = j * WIDTH;
        x.mirror = false;
    } else {   // squares of SIDE from the diagonal on, in strips of WIDTH
        const uint32_t strip = t % (SIDE / WIDTH);
        t /= SIDE / WIDTH;
        i = 0;
        while (t >= a.tiles_m - i) t -= a.tiles_m - i++;
        j = i + t;
        x.col = j * SIDE + strip * WIDTH;
        x.mirror = i != j;
    }
    x.row = i * SIDE;
    return x;
}

__device__ __forceinline__ uint4 load_shared(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void store_shared(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w));
}
// Octet `o` (16 bytes) of row r of a box, as the tiled copies lay it: swizzled over 8 rows.
__device__ __forceinline__ uint32_t box_octet(uint32_t box, uint32_t r, uint32_t o) { return box + r * 128u + ((o ^ (r & 7u)) << 4); }
template <int N>
__device__ __forceinline__ void halves(const uint4 (&w)[N], float (&v)[8 * N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[k]));
            v[8 * i + 2 * k] = f.x;
            v[8 * i + 2 * k + 1] = f.y;
        }
    }
}

// Element k of v, which stays in registers.
template <int N>
__device__ __forceinline__ float pick(const float (&v)[N], uint32_t k)
{
    if constexpr (N == 1) {
        return v[0];
    } else {
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) half[i] = k & 1u ? v[2 * i + 1] : v[2 * i];
        return pick(half, k / 2u);
    }
}
// The element on the diagonal, kept apart, leaves a zero in row r and column c of a box.
__device__ __forceinline__ void clear_half(uint32_t box, uint32_t r, uint32_t c)
{
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(box_octet(box, r, c / 8u) + c % 8u * 2u), "h"((uint16_t)0) : "memory");
}

constexpr int TAKEN = 64 / (TAKERS / 4);   // columns of a box that a warp takes
constexpr int OCTETS = TAKEN / 8;

// s2 v + (s0 + s1 d) in on two elements
__device__ __forceinline__ void poly(float &v, float &w, float in_v, float in_w, float d_v, float d_w, float s0, float s1, float s2)
{
    const float2 t = fma2(make_float2(d_v, d_w), make_float2(s1, s1), make_float2(s0, s0));
    const float2 p = fma2(t, make_float2(in_v, in_w), fma2(make_float2(v, w), make_float2(s2, s2), make_float2(0.0f, 0.0f)));
    v = p.x;
    w = p.y;
}

// a X + B X as X is kept, from the sums of B X
template <int N>
__device__ __forceinline__ void update(float (&v)[N], const float (&in)[N], float linear)
{
    constexpr float S = 1.0f / ORTHO_B_SCALE;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
        const float2 b = fma2(make_float2(v[k], v[k + 1]), make_float2(S, S), make_float2(0.0f, 0.0f));
        const float2 x = fma2(make_float2(in[k], in[k + 1]), make_float2(linear, linear), b);
        v[k] = x.x;
        v[k + 1] = x.y;
    }
}

// TAKEN neighbouring sums of row `row` (row r of the CTA's boxes) from column c on (octet o of the box) -> what is kept of
// them, in the box at `box` (and a second term in the box behind it).  `linear`: the row's element of D (POLY), a and the
// row's element of B's diagonal (UPDATE); `across`: D from column c on, in shared memory.
template <int MODE>
__device__ __forceinline__ void finish(float (&v)[TAKEN], uint32_t batch, uint32_t row, uint32_t c, uint32_t box, uint32_t r, uint32_t o, float linear,
                                       uint32_t across, bool mirror, const ProductArgs &a)
{
    constexpr float XS = ORTHO_X_SCALE, AS = ORTHO_A_SCALE, BS = ORTHO_B_SCALE;
    const bool diagonal = MODE != UPDATE && row - c < (uint32_t)TAKEN;
    float in[TAKEN];
    if (MODE != GRAM) {
        uint4 w[OCTETS];
#pragma unroll
        for (int i = 0; i < OCTETS; ++i) w[i] = load_shared(box_octet(box, r, o + i));
        halves(w, in);
    }
    if (MODE == GRAM) {
        if (diagonal && row < a.rows) a.d[batch * a.d_stride + row] = pick(v, row - c) * (1.0f / (XS * XS));
#pragma unroll
        for (int k = 0; k < TAKEN; ++k) v[k] *= AS / (XS * XS);
    }
    if (MODE == POLY) {
        const float s2 = a.cc * BS / (AS * AS), s1 = a.cc * BS / AS, s0 = a.cb * BS / AS + s1 * linear;
        if (diagonal && row < a.rows)
            a.db[batch * a.d_stride + row] = a.cb * linear + a.cc * (pick(v, row - c) * (1.0f / (AS * AS)) + linear * linear);
#pragma unroll
        for (int i = 0; i < TAKEN / 4; ++i) {
            const uint4 w = load_shared(across + i * 16);
            const float d[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const int k = 4 * i + j;
                poly(v[k], v[k + 1], in[k], in[k + 1], d[j], d[j + 1], s0, s1, s2);
            }
        }
    }
    if (MODE == UPDATE) {
        uint4 w[OCTETS];
        float rest[TAKEN];
#pragma unroll
        for (int i = 0; i < OCTETS; ++i) w[i] = load_shared(box_octet(box + OPERAND_BYTES, r, o + i));
        halves(w, rest);
#pragma unroll
        for (int k = 0; k < TAKEN; k += 2) add(in[k], in[k + 1], rest[k], rest[k + 1]);
        update(v, in, linear);
        if (a.out) {
            __nv_bfloat162 h[TAKEN / 2];
#pragma unroll
            for (int k = 0; k < TAKEN / 2; ++k) h[k] = __floats2bfloat162_rn(v[2 * k] * (1.0f / XS), v[2 * k + 1] * (1.0f / XS));
            if (a.turned) {
                __nv_bfloat16 *to = a.out + batch * a.out_stride + c * a.ldo + row;
                if (row < a.rows)
#pragma unroll
                    for (int k = 0; k < TAKEN; ++k, to += a.ldo)
                        if (c + k < a.cols) *to = k % 2 ? h[k / 2].y : h[k / 2].x;
            } else {
                const uint32_t *const w = reinterpret_cast<const uint32_t *>(h);
#pragma unroll
                for (int i = 0; i < OCTETS; ++i) store_shared(box_octet(box, r, o + i), make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
            }
            return;
        }
    }
    if (MODE == UPDATE) {   // both terms together are cut off where one alone would be
#pragma unroll
        for (int k = 0; k < TAKEN; ++k) v[k] = cut_off(v[k]);
    }
    uint32_t h[TAKEN / 2];
#pragma unroll
    for (int k = 0; k < TAKEN / 2; ++k) h[k] = half_pair(v[2 * k], v[2 * k + 1]);
#pragma unroll
    for (int i = 0; i < OCTETS; ++i) store_shared(box_octet(box, r, o + i), make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]));
    if (diagonal) clear_half(box, r, o * 8u + row - c);
    if (MODE == UPDATE) {
        uint32_t l[TAKEN / 2];
#pragma unroll
        for (int k = 0; k < TAKEN / 2; ++k) l[k] = rest_pair(v[2 * k], v[2 * k + 1], h[k]);
#pragma unroll
        for (int i = 0; i < OCTETS; ++i)
            store_shared(box_octet(box + OPERAND_BYTES, r, o + i), make_uint4(l[4 * i], l[4 * i + 1], l[4 * i + 2], l[4 * i + 3]));
    }
    if (MODE != UPDATE && mirror && row < a.rows) {
        unsigned short *to = reinterpret_cast<unsigned short *>(a.mirror) + batch * a.a_stride + c * a.ld_a + row;
#pragma unroll
        for (int k = 0; k < TAKEN; ++k, to += a.ld_a)
            if (c + k < a.cols) *to = (unsigned short)(h[k / 2] >> (16 * (k % 2)));
    }
}

// 128 rows from a box of results to rows of `out` that no tiled copy takes, by all threads that take tiles out.
__device__ __forceinline__ void store_rows(uint32_t batch, uint32_t row0, uint32_t c, uint32_t box, uint32_t thread, const ProductArgs &a)
{
    for (uint32_t i = thread; i < 128 * BOX_COLS; i += TAKERS * 32) {
        const uint32_t r = i / BOX_COLS, col = i % BOX_COLS;
        uint16_t h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(box_octet(box, r, col / 8u) + col % 8u * 2u));
        if (row0 + r < a.rows && c + col < a.cols)
            a.out[batch * a.out_stride + (row0 + r) * a.ldo + c + col] = *reinterpret_cast<const __nv_bfloat16 *>(&h);
    }
}

// DEEP: an update whose contraction is long has five stages, and two slots in the second ring, in place of four and three.
// Pairs: 4096 x 8192 2.08 ms in place of 2.16 (five steps), 2048 x 2048 260 us in place of 268; 12 x 512 x 2048 293 in place of 284,
// 4 x 1024 x 4096 398 in place of 394: from contractions of 2048 on.
// NARROW: a single CTA's tile has 64 columns in place of 128.
template <int MODE, bool PAIR, bool DEEP, bool NARROW>
struct Shape {
    static constexpr uint32_t SIDE = PAIR ? 256 : 128;       // rows of a tile
    static constexpr uint32_t WIDTH = NARROW ? 64 : SIDE;    // and columns
    static constexpr uint32_t Q_BYTES = NARROW ? OPERAND_BYTES / 2 : OPERAND_BYTES;
    static constexpr int STAGES = MODE == UPDATE && !DEEP ? 4 : 5;
    static constexpr int SLOTS = MODE == UPDATE && DEEP ? 2 : 3;   // of the second ring
    static constexpr uint32_t STAGE_BYTES = 2 * OPERAND_BYTES;   // of one CTA: 128 rows of either operand
    static constexpr uint32_t SLOT_BYTES = (MODE == UPDATE ? 2 : 1) * OPERAND_BYTES;
    static constexpr uint32_t COLUMNS = 2 * WIDTH;           // of tensor memory: two tiles
    static constexpr uint32_t SMEM = STAGES * STAGE_BYTES + SLOTS * SLOT_BYTES + 1024 + 256 + SIDE * 4;
};

__device__ __forceinline__ void takers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(TAKERS * 32) : "memory"); }

template <int MODE, bool PAIR, bool DEEP, bool NARROW>
__global__ __launch_bounds__(WARPS * 32, 1) void qesgd_ortho_product_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ ProductMaps maps)
{
    using S = Shape<MODE, PAIR, DEEP, NARROW>;
    constexpr uint32_t BOXES = S::WIDTH / BOX_COLS;                   // of a tile, for each CTA
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u, ring = base + S::STAGES * S::STAGE_BYTES;
    const uint32_t bars = ring + S::SLOTS * S::SLOT_BYTES;
    const uint32_t full = bars, empty = full + 8 * S::STAGES, done = empty + 8 * S::STAGES, free_ = done + 16;
    const uint32_t filled = free_ + 16, worked = filled + 8 * S::SLOTS, stored = worked + 8 * S::SLOTS, slot = stored + 8 * S::SLOTS;
    const uint32_t across = bars + 256;                              // D along the columns of a tile (POLY)
    volatile uint32_t *const stop = reinterpret_cast<volatile uint32_t *>(raw + (slot + 8 - smem_u32(raw)));
    const uint32_t warp = threadIdx.x / 32u, lane = threadIdx.x % 32u;
    const uint32_t rank = PAIR || a.split > 1 ? cluster_rank() : 0u;
    // CTAs of a cluster: a pair, or those that share a contraction, of which the first two each finish one box
    const uint32_t share = PAIR ? 2u : a.split, parts = PAIR ? 1u : a.split, part_k = PAIR ? 0u : rank;
    const uint32_t group = blockIdx.x / share, groups = gridDim.x / share;
    const uint32_t own_rows = PAIR ? rank * 128u : 0u;
    const uint32_t box_first = parts > 1 ? rank : 0u, box_end = parts > 1 ? min(rank + 1u, BOXES) : BOXES;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init_at(full + 8 * s, 1u);
            mbar_init_at(empty + 8 * s, 1u);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init_at(done + 8 * s, 1u);
            mbar_init_at(free_ + 8 * s, PAIR ? 2u * TAKERS : TAKERS);
        }
        for (int s = 0; s < S::SLOTS; ++s) {
            mbar_init_at(filled + 8 * s, 1u);
            mbar_init_at(worked + 8 * s, TAKERS);
            mbar_init_at(stored + 8 * s, 1u);
        }
        *stop = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
        prefetch_map(&maps.p);
        prefetch_map(&maps.q);
    }
    // Both CTAs of a pair are there, and their barriers.  (The first product of a pair waits for copies that its other CTA
    // sets off behind its own part of the allocation.)
    if (PAIR) cluster_sync_all();
    if (warp == 2) tmem_alloc<PAIR>(slot, S::COLUMNS);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(raw + (slot - smem_u32(raw)));
    const uint32_t all = a.tiles * a.batch, once = (a.depth + DEPTH - 1) / DEPTH, every = MODE == UPDATE ? once * a.terms : once;
    const uint32_t step0 = every * part_k / parts, steps = every * (part_k + 1) / parts - step0;
    qesgd_wait_for_previous();

    if (warp == 0 && elect_one()) {
        uint32_t n = 0;
        const uint32_t full_lead = PAIR ? map_shared(full, 0) : full;
        for (uint32_t t = group; t < all && !*stop; t += groups) {
            const Tile x = tile_of<MODE, S::SIDE, S::WIDTH>(t, a);
            const uint32_t row = x.row + own_rows, col = x.col + own_rows;
            for (uint32_t k = 0; k < steps; ++k, ++n) {
                const uint32_t s = n % S::STAGES, to = base + s * S::STAGE_BYTES;
                if (n >= S::STAGES && !pipe_wait(empty + 8 * s, (n / S::STAGES - 1u) & 1u, stop)) break;
                const bool second = MODE == UPDATE && step0 + k >= once;   // the contraction over X's second term
                const uint32_t at = (step0 + k - (second ? once : 0u)) * DEPTH;
                const bool own = MODE != UPDATE && !x.mirror;   // a square on the diagonal: Q's rows are among P's
                if (!PAIR || rank == 0) mbar_expect_at(full + 8 * s, (OPERAND_BYTES + (own ? 0u : S::Q_BYTES)) * (PAIR ? 2u : 1u));
                tma_load_3d<PAIR>(to, &maps.p, at, row, x.batch, full_lead + 8 * s);
                if (MODE == UPDATE) {
                    const CUtensorMap *const q = second ? &maps.q_lo : &maps.q;
                    tma_load_3d<PAIR>(to + OPERAND_BYTES, q, col, at, x.batch, full_lead + 8 * s);
                    if (!NARROW) tma_load_3d<PAIR>(to + OPERAND_BYTES + OPERAND_BYTES / 2, q, col + 64u, at, x.batch, full_lead + 8 * s);
                } else if (!own) {
                    tma_load_3d<PAIR>(to + OPERAND_BYTES, &maps.q, at, col, x.batch, full_lead + 8 * s);
                }
            }
        }
        if (*stop) drain();
    } else if (warp == 1 && (!PAIR || rank == 0) && elect_one()) {
        // fp16 operands, fp32 sums, SIDE x WIDTH; Q of UPDATE has its contraction across the rows
        constexpr uint32_t INSTRUCTION = 1u << 4 | (MODE == UPDATE ? 1u << 16 : 0u) | (S::WIDTH / 8) << 17 | (S::SIDE / 16) << 24;
        uint32_t n = 0, done_tiles = 0;
        for (uint32_t t = group; t < all && !*stop; t += groups, ++done_tiles) {
            const uint32_t half = done_tiles & 1u, sums = tmem + half * S::WIDTH;
            const Tile x = tile_of<MODE, S::SIDE, S::WIDTH>(t, a);
            const uint32_t q_at = MODE == UPDATE || x.mirror ? OPERAND_BYTES : (x.col - x.row) * 128u;
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
                                                      : swizzled_matrix(from + q_at + i * 32u, 16u, 1024u);
                    mma_f16<PAIR>(sums, p, q, INSTRUCTION, k > 0 || i > 0);
                }
                mma_commit<PAIR>(empty + 8 * s);
            }
            if (!ok) break;
            mma_commit<PAIR>(done + 8 * half);
        }
        if (*stop) drain();
    } else if (warp == 2 && elect_one()) {
        uint32_t n = 0;
        for (uint32_t t = group; t < all && !*stop; t += groups) {
            const Tile x = tile_of<MODE, S::SIDE, S::WIDTH>(t, a);
            for (uint32_t b = box_first; b < box_end; ++b, ++n) {
                const uint32_t s = n % S::SLOTS, to = ring + s * S::SLOT_BYTES;
                if (n >= S::SLOTS && !pipe_wait(stored + 8 * s, (n / S::SLOTS - 1u) & 1u, stop)) break;
                if (MODE == GRAM) {
                    mbar_arrive_at(filled + 8 * s);
                    continue;
                }
                const uint32_t col = x.col + b * BOX_COLS, row = x.row + own_rows;
                mbar_expect_at(filled + 8 * s, S::SLOT_BYTES);
                tma_load_3d<false>(to, &maps.in, col, row, x.batch, filled + 8 * s);
                if (MODE == UPDATE) tma_load_3d<false>(to + OPERAND_BYTES, &maps.in_lo, col, row, x.batch, filled + 8 * s);
            }
        }
        if (*stop) drain();
    } else if (warp == 3) {
        if (parts > 1) {   // the barriers of the cluster come before the box that this warp stores
            cluster_arrive();
            cluster_wait();
            cluster_arrive();
            cluster_wait();
        }
        if (elect_one()) {
            uint32_t n = 0;
            const bool store = MODE != UPDATE || !a.out || a.out_tiled;
            for (uint32_t t = group; t < all && !*stop; t += groups) {
                const Tile x = tile_of<MODE, S::SIDE, S::WIDTH>(t, a);
                for (uint32_t b = box_first; b < box_end; ++b, ++n) {
                    const uint32_t s = n % S::SLOTS, from = ring + s * S::SLOT_BYTES;
                    if (!pipe_wait(worked + 8 * s, (n / S::SLOTS) & 1u, stop)) break;
                    const uint32_t col = x.col + b * BOX_COLS, row = x.row + own_rows;
                    if (store && col < a.cols && row < a.rows) {
                        tma_store_3d(&maps.out, col, row, x.batch, from);
                        if (MODE == UPDATE && !a.out) tma_store_3d(&maps.out_lo, col, row, x.batch, from + OPERAND_BYTES);
                    }
                    store_commit();
                    store_wait_read<0>();
                    mbar_arrive_at(stored + 8 * s);
                }
            }
            store_wait<0>();
            if (*stop) drain();
        }
    } else if (warp >= 4) {
        const uint32_t quarter = warp % 4u, r = quarter * 32u + lane, part = (warp - 4u) / 4u, thread = threadIdx.x - 128u;
        const uint32_t free_lead = PAIR ? map_shared(free_, 0) : free_;
        uint32_t n = 0, done_tiles = 0;
        // after a wait that ran out the loops are gone through without work: the barriers of these warps stay in step
        bool ok = true;
        for (uint32_t t = group; t < all; t += groups, ++done_tiles) {
            const Tile x = tile_of<MODE, S::SIDE, S::WIDTH>(t, a);
            const uint32_t half = done_tiles & 1u, row0 = x.row + own_rows, row = row0 + r;
            float linear = 0.0f;
            if (MODE != GRAM && row < a.rows) linear = __ldcg((MODE == POLY ? a.d : a.db) + x.batch * a.d_stride + row) + (MODE == UPDATE ? a.ca : 0.0f);
            if (MODE == POLY) {
                takers_sync();   // the last tile's have been read
                if (thread < S::WIDTH) {
                    const uint32_t c = x.col + thread;
                    const float d = c < a.cols ? __ldcg(a.d + x.batch * a.d_stride + c) : 0.0f;
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(across + thread * 4u), "f"(d));
                }
                takers_sync();
            }
            ok = __all_sync(FULL, ok && pipe_wait(done + 8 * half, (done_tiles / 2) & 1u, stop));
            fence_after_sync();
            if (parts > 1) {
                // all of the cluster are through with their stages: the sums of a box go to the CTA that finishes it, by four columns
                __syncwarp();
                cluster_arrive();
                cluster_wait();
                for (uint32_t b = 0; b < BOXES; ++b) {
                    if (b == rank) continue;
                    float v[TAKEN];
                    __syncwarp();
                    tmem_load16(tmem + (quarter * 32u << 16) + b * BOX_COLS + part * TAKEN, v);
                    tmem_wait_load();
                    const uint32_t to = map_shared(base + ((rank * (BOX_COLS / 4) + part * (TAKEN / 4)) * 128u + r) * 16u, b);
#pragma unroll
                    for (int i = 0; i < TAKEN / 4; ++i)
                        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + i * 2048u), "f"(v[4 * i]), "f"(v[4 * i + 1]), "f"(v[4 * i + 2]),
                                     "f"(v[4 * i + 3])
                                     : "memory");
                }
                __syncwarp();
                cluster_arrive();
                cluster_wait();
            }
            for (uint32_t b = box_first; b < box_end; ++b, ++n) {
                const uint32_t s = n % S::SLOTS, box = ring + s * S::SLOT_BYTES, first = b * BOX_COLS + part * TAKEN;
                float v[TAKEN];
                __syncwarp();
                tmem_load16(tmem + (quarter * 32u << 16) + half * S::WIDTH + first, v);
                ok = __all_sync(FULL, ok && pipe_wait(filled + 8 * s, (n / S::SLOTS) & 1u, stop));
                tmem_wait_load();
                if (parts > 1) {
                    float mine[TAKEN];
#pragma unroll
                    for (int k = 0; k < TAKEN; ++k) {
                        mine[k] = v[k];
                        v[k] = 0.0f;
                    }
                    for (uint32_t p = 0; p < parts; ++p) {   // in the order of the contraction
#pragma unroll
                        for (int i = 0; i < TAKEN / 4; ++i) {
                            uint4 f = make_uint4(__float_as_uint(mine[4 * i]), __float_as_uint(mine[4 * i + 1]), __float_as_uint(mine[4 * i + 2]), __float_as_uint(mine[4 * i + 3]));
                            if (p != rank) f = load_shared(base + ((p * (BOX_COLS / 4) + part * (TAKEN / 4) + i) * 128u + r) * 16u);
                            v[4 * i] += __uint_as_float(f.x);
                            v[4 * i + 1] += __uint_as_float(f.y);
                            v[4 * i + 2] += __uint_as_float(f.z);
                            v[4 * i + 3] += __uint_as_float(f.w);
                        }
                    }
                } else if (b + 1 == BOXES) {   // the last of the tile is in registers
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR) mbar_arrive_cluster(free_lead + 8 * half);
                        else mbar_arrive_at(free_ + 8 * half);
                    }
                }
                if (ok) finish<MODE>(v, x.batch, row, x.col + first, box, r, part * OCTETS, linear, across + first * 4u, x.mirror, a);
                if (MODE == UPDATE && a.out && !a.turned && !a.out_tiled) {
                    takers_sync();
                    if (ok) store_rows(x.batch, row0, x.col + b * BOX_COLS, box, thread, a);
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(worked + 8 * s);
            }
        }
    }
    __syncwarp();
    if (parts > 1 && warp < 3) {
        cluster_sync_all();
        cluster_sync_all();
    }
    __syncthreads();
    if (threadIdx.x == 0 && *stop) atomicOr(a.status, QESGD_STATUS_TIMEOUT);
    fence_before_sync();
    if (PAIR) cluster_sync_all();
    fence_after_sync();
    if (warp == 2) tmem_dealloc<PAIR>(tmem, S::COLUMNS);
}

// ---------------------------------------------------- a whole matrix at once ----
// Matrices with up to 128 rows (of the smaller side) and 4096 columns: all steps in one kernel.  A cluster of 1 to 16 CTAs
// has a matrix, each up to 256 of its columns: X stays in registers in 32 bits and in shared memory as one fp16 term, for the
// updates of the first ORTHO_TERMS_STEPS steps as two, where the products read it, beside F, then B in its place; all sums
// stay in tensor memory.  A step exchanges the parts of A among
// the CTAs: each adds up some of its columns, in the order of the CTAs, and writes F's share of them into every CTA.  The
// fifteen products as kernels of their own take 5 us each here, most of it for starting, waiting for the first copies
// and storing what the next one loads.
// 64 x 256 takes 23 us: 3.5 to load and divide by the norm, then 3.7 for each of the first three steps (3.1 with one term of X) and 3.1
// for the others, half of it from a product's first instruction to its sums' arrival (sixteen instructions deep for A), half to take
// the sums out and settle what the next one reads.  128 x 4096 takes 72 us, half of it for the exchange.  With one term of X in all
// steps (21 and 70): X as two terms in shared memory in place of 32 bits 1 us slower, half of the warps idle at the update's end 4 us,
// A begun with the columns that are done, while others are still taken out, 0.5 and 3 us: each part costs one more barrier.
constexpr uint32_t WHOLE_ROWS = 128, WHOLE_COLS = 256, WHOLE_MAX_CLUSTER = 16;
constexpr uint32_t BOX_BYTES = OPERAND_BYTES;              // 128 rows of 64 columns
constexpr uint32_t WHOLE_EXTRA = 1152;                     // diagonals, barrier and the like
constexpr uint32_t WHOLE_THREADS = 512;
constexpr int WHOLE_MOST_SMEM = 10 * BOX_BYTES + WHOLE_EXTRA + 1024 + 128 * 128 * 4;
constexpr uint32_t WHOLE_MIN_SMEM = 120 * 1024;            // one CTA of an SM: CTAs of two clusters must not wait for one another's tensor memory

struct WholeArgs {
    const void *x;
    uint64_t ldx, x_stride, ldo, out_stride;
    uint32_t m, n, width, steps, turned, vec, out_vec;     // width: columns of a CTA
    float ca, cb, cc;
    __nv_bfloat16 *out;
    uint32_t *status;
};

__device__ __forceinline__ void store_remote(uint32_t addr, uint4 v)
{
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ float load_shared_float(uint32_t addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

template <typename T, bool CLUSTER>
__global__ __launch_bounds__(WHOLE_THREADS, 1) void qesgd_ortho_whole_kernel(const __grid_constant__ WholeArgs a)
{
    constexpr float XS = ORTHO_X_SCALE, AS = ORTHO_A_SCALE, BS = ORTHO_B_SCALE;
    constexpr uint32_t A_COLUMN = 0, P_COLUMN = 128, U_COLUMN = 256;   // of tensor memory: sums of GRAM, POLY, UPDATE
    extern __shared__ uint8_t raw[];
    const uint32_t boxes = a.width / BOX_COLS, share = CLUSTER ? (a.n + a.width - 1) / a.width : 1u;
    const uint32_t hi = (smem_u32(raw) + 1023u) & ~1023u, lo = hi + boxes * BOX_BYTES, f = lo + boxes * BOX_BYTES;
    const uint32_t d = f + 2 * BOX_BYTES, db = d + 512, bar = db + 512, slot = bar + 8, norm = bar + 16, parts = f + 2 * BOX_BYTES + WHOLE_EXTRA;
    volatile uint32_t *const stop = reinterpret_cast<volatile uint32_t *>(raw + (slot + 4 - smem_u32(raw)));
    const uint32_t warp = threadIdx.x / 32u, lane = threadIdx.x % 32u, quarter = warp % 4u, part = warp / 4u, r = quarter * 32u + lane;
    const uint32_t rank = CLUSTER ? cluster_rank() : 0u, cluster = CLUSTER ? gridDim.x : 1u;   // gridDim.x: a power of two, `share` or more
    const uint32_t c0 = rank * a.width, slots = 16u / cluster;   // slots: octets of A's columns that a CTA adds up
    if (threadIdx.x == 0) {
        mbar_init_at(bar, 1u);
        *stop = 0u;
        fence_async_shared();
    }
    if (warp == 0) tmem_alloc<false>(slot, 512u);
    qesgd_wait_for_previous();

    // ---- X = G / ||G||: this CTA's columns, every thread eight octets at most (of a row; turned, of a column) ----
    const T *const g = static_cast<const T *>(a.x) + blockIdx.y * a.x_stride;
    float v[8][8];
    double sum = 0.0;
    // rows of X in whole products, columns of A in whole loads; what lies behind them is not looked at
    const uint32_t rows = (a.m + 15u) / 16u * 16u;
    const uint32_t octets = a.turned ? rows / 8 : a.width / 8, all = rows * a.width / 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t n = threadIdx.x + i * WHOLE_THREADS, line = n / octets, first = n % octets * 8;   // line: row of X, or column
        if (i * WHOLE_THREADS >= all) break;
        const bool inside = n < all && (a.turned ? c0 + line < a.n && first < a.m : line < a.m && c0 + first < a.n);
        if (inside) {
            if (a.turned) values(load_octet(g + (c0 + line) * a.ldx, first, a.m, a.vec), v[i]);
            else values(load_octet(g + line * a.ldx, c0 + first, a.n, a.vec), v[i]);
        }
        if (!inside)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = 0.0f;
        sum += octet_squares(v[i]);
    }
    sum = block_sum<WHOLE_THREADS>(sum);
    if (threadIdx.x == 0) *reinterpret_cast<double *>(raw + (norm - smem_u32(raw))) = sum;
    fence_before_sync();
    if (CLUSTER) cluster_sync_all();
    else __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(raw + (slot - smem_u32(raw)));
    sum = 0.0;
    for (uint32_t p = 0; p < cluster; ++p) {
        double other;
        if (CLUSTER) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(other) : "r"(map_shared(norm, p)) : "memory");
        else other = *reinterpret_cast<volatile double *>(raw + (norm - smem_u32(raw)));
        sum += other;
    }
    if (!(sum <= 1.7976931348623157e308) && threadIdx.x == 0 && rank == 0) atomicOr(a.status, QESGD_STATUS_NONFINITE);
    const Normalise scale = normalise(sum);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t n = threadIdx.x + i * WHOLE_THREADS, line = n / octets, first = n % octets * 8;
        if (n >= all) break;
        uint32_t h[4], l[4];
        times(v[i], scale);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            h[k] = half_pair(v[i][2 * k], v[i][2 * k + 1]);
            l[k] = rest_pair(v[i][2 * k], v[i][2 * k + 1], h[k]);
        }
        if (!a.turned) {
            const uint32_t at = first / 64u * BOX_BYTES;
            store_shared(box_octet(hi + at, line, first / 8u % 8u), make_uint4(h[0], h[1], h[2], h[3]));
            store_shared(box_octet(lo + at, line, first / 8u % 8u), make_uint4(l[0], l[1], l[2], l[3]));
        } else {
            const uint32_t at = line / 64u * BOX_BYTES, o = line / 8u % 8u, in = line % 8u * 2u;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(box_octet(hi + at, first + k, o) + in), "h"((uint16_t)(h[k / 2] >> (16 * (k % 2)))));
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(box_octet(lo + at, first + k, o) + in), "h"((uint16_t)(l[k / 2] >> (16 * (k % 2)))));
            }
        }
    }
    fence_async_shared();
    __syncthreads();

    // A finished product is waited for by everybody; a wait that ran out leaves the barriers in step, and the result unsaid.
    uint32_t phase = 0;
    bool ok = true;
    const auto products_done = [&]() {
        ok = pipe_wait(bar, phase, stop) && ok;
        phase ^= 1u;
        __syncwarp();
        fence_after_sync();
    };
    const auto settled = [&]() {   // shared memory written for the next product, tensor memory read
        fence_async_shared();
        fence_before_sync();
        __syncthreads();
        fence_after_sync();
    };
    // Where there are few rows B's are laid down twice or four times, one copy under another: then the update of every row
    // stands in several quarters of tensor memory, and their warps take some of its columns each.
    const uint32_t copies = rows <= 32u ? 4u : rows <= 64u ? 2u : 1u, span = WHOLE_ROWS / copies;
    const uint32_t ur = r % span, ustride = 64u * copies, ufirst = (quarter * 32u / span * 4u + part) * 16u;   // of the update
    const bool uidle = ur / 32u * 32u >= rows;
    const bool idle = quarter * 32u >= rows;
    // and each thread keeps its elements of X in 32 bits: 16 neighbours of its row, up to four times
    float x[4][16];
#pragma unroll
    for (uint32_t n = 0; n < 4; ++n) {
        const uint32_t c = ufirst + n * ustride, at = c / 64u * BOX_BYTES, o = c / 8u % 8u;
        if (c >= a.width || uidle) break;
        float rest[16];
        uint4 q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) q[i] = load_shared(box_octet(hi + at, ur, o + i));
        halves(q, x[n]);
#pragma unroll
        for (int i = 0; i < 2; ++i) q[i] = load_shared(box_octet(lo + at, ur, o + i));
        halves(q, rest);
#pragma unroll
        for (int k = 0; k < 16; k += 2) add(x[n][k], x[n][k + 1], rest[k], rest[k + 1]);
    }
    const uint32_t square = 1u << 4 | (rows / 8) << 17 | (128u / 16) << 24;
    // operands: addresses count in 16 bytes
    const uint64_t hi_rows = swizzled_matrix(hi, 16u, 1024u), f_rows = swizzled_matrix(f, 16u, 1024u);
    const uint64_t hi_columns = swizzled_matrix(hi, BOX_BYTES, 1024u), lo_columns = swizzled_matrix(lo, BOX_BYTES, 1024u);
    for (uint32_t step = 0; step < a.steps; ++step) {
        const bool last = step + 1 == a.steps;
        // ---- A = X X^T ----
        if (warp == 0 && elect_one()) {
#pragma unroll
            for (uint32_t b = 0; b < WHOLE_COLS / BOX_COLS; ++b) {
                if (b >= boxes) break;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    mma_f16<false>(tmem + A_COLUMN, hi_rows + (b * BOX_BYTES + i * 32u) / 16u, hi_rows + (b * BOX_BYTES + i * 32u) / 16u, square, b > 0 || i > 0);
            }
            mma_commit<false>(bar);
        }
        __syncwarp();
        products_done();
#pragma unroll 1
        for (uint32_t c = part * 16u; c < rows && !idle; c += 64u) {
            float w[16];
            __syncwarp();
            tmem_load16(tmem + (quarter * 32u << 16) + A_COLUMN + c, w);
            tmem_wait_load();
            if (CLUSTER) {
                // an octet of columns to the CTA that adds it up: they are dealt out in turn
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t o = c / 8u + i / 2u;
                    store_remote(map_shared(parts + (((rank * slots + o / cluster) * 2u + i % 2u) * 128u + r) * 16u, o % cluster),
                                 make_uint4(__float_as_uint(w[4 * i]), __float_as_uint(w[4 * i + 1]), __float_as_uint(w[4 * i + 2]), __float_as_uint(w[4 * i + 3])));
                }
            } else {
                const bool diagonal = r - c < 16u;
                if (diagonal) asm volatile("st.shared.f32 [%0], %1;" ::"r"(d + r * 4u), "f"(pick(w, r - c) * (1.0f / (XS * XS))));
#pragma unroll
                for (int k = 0; k < 16; ++k) w[k] *= AS / (XS * XS);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    store_shared(box_octet(f + c / 64u * BOX_BYTES, r, c / 8u % 8u + i),
                                 make_uint4(half_pair(w[8 * i], w[8 * i + 1]), half_pair(w[8 * i + 2], w[8 * i + 3]), half_pair(w[8 * i + 4], w[8 * i + 5]),
                                            half_pair(w[8 * i + 6], w[8 * i + 7])));
                if (diagonal) clear_half(f + c / 64u * BOX_BYTES, r, r % 64u);
            }
        }
        if (CLUSTER) {
            __syncwarp();
            cluster_sync_all();
            const uint32_t row = threadIdx.x % 128u;
            for (uint32_t o = rank + cluster * (threadIdx.x / 128u); o < rows / 8u && row < rows; o += cluster * (WHOLE_THREADS / 128u)) {
                float w[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
                for (uint32_t p = 0; p < share; ++p) {   // CTAs behind the last column have nothing to add
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4 q = load_shared(parts + (((p * slots + o / cluster) * 2u + i) * 128u + row) * 16u);
                        w[4 * i] += __uint_as_float(q.x);
                        w[4 * i + 1] += __uint_as_float(q.y);
                        w[4 * i + 2] += __uint_as_float(q.z);
                        w[4 * i + 3] += __uint_as_float(q.w);
                    }
                }
                const float own = pick(w, row % 8u);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = o * 8u + k == row ? 0.0f : w[k] * (AS / (XS * XS));
                const uint4 packed = make_uint4(half_pair(w[0], w[1]), half_pair(w[2], w[3]), half_pair(w[4], w[5]), half_pair(w[6], w[7]));
                for (uint32_t p = 0; p < cluster; ++p) {
                    store_remote(map_shared(box_octet(f + o / 8u * BOX_BYTES, row, o % 8u), p), packed);
                    if (o == row / 8u) store_remote(map_shared(d + row * 4u, p), own * (1.0f / (XS * XS)));
                }
            }
            __syncwarp();
            fence_async();
            fence_before_sync();
            cluster_sync_all();
            fence_async();   // what the others wrote here, for this CTA's product
            __syncthreads();
            fence_after_sync();
        } else {
            settled();
        }
        // ---- B = b A + c A A ----
        if (warp == 0 && elect_one()) {
#pragma unroll
            for (uint32_t i = 0; i < WHOLE_ROWS / 16; ++i) {
                if (i * 16u >= rows) break;
                mma_f16<false>(tmem + P_COLUMN, f_rows + (i / 4 * BOX_BYTES + i % 4 * 32u) / 16u, f_rows + (i / 4 * BOX_BYTES + i % 4 * 32u) / 16u, square, i > 0);
            }
            mma_commit<false>(bar);
        }
        __syncwarp();
        products_done();
        {
            const float dr = load_shared_float(d + r * 4u);
            const float s2 = a.cc * BS / (AS * AS), s1 = a.cc * BS / AS, s0 = a.cb * BS / AS + s1 * dr;
#pragma unroll 1
            for (uint32_t c = part * 16u; c < rows && !idle; c += 64u) {
                float w[16], in[16];
                __syncwarp();
                tmem_load16(tmem + (quarter * 32u << 16) + P_COLUMN + c, w);
                uint4 q[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) q[i] = load_shared(box_octet(f + c / 64u * BOX_BYTES, r, c / 8u % 8u + i));
                halves(q, in);
                tmem_wait_load();
                const bool diagonal = r - c < 16u;
                if (diagonal) asm volatile("st.shared.f32 [%0], %1;" ::"r"(db + r * 4u), "f"(a.cb * dr + a.cc * (pick(w, r - c) * (1.0f / (AS * AS)) + dr * dr)));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 z = load_shared(d + c * 4u + i * 16u);
                    const float dc[4] = {__uint_as_float(z.x), __uint_as_float(z.y), __uint_as_float(z.z), __uint_as_float(z.w)};
#pragma unroll
                    for (int j = 0; j < 4; j += 2) poly(w[4 * i + j], w[4 * i + j + 1], in[4 * i + j], in[4 * i + j + 1], dc[j], dc[j + 1], s0, s1, s2);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 packed = make_uint4(half_pair(w[8 * i], w[8 * i + 1]), half_pair(w[8 * i + 2], w[8 * i + 3]),
                                                    half_pair(w[8 * i + 4], w[8 * i + 5]), half_pair(w[8 * i + 6], w[8 * i + 7]));
                    store_shared(box_octet(f + c / 64u * BOX_BYTES, r, c / 8u % 8u + i), packed);
                    if (copies > 1u)
                        for (uint32_t p = r + span; p < WHOLE_ROWS; p += span) store_shared(box_octet(f + c / 64u * BOX_BYTES, p, c / 8u % 8u + i), packed);
                }
                if (diagonal)
                    for (uint32_t p = r; p < WHOLE_ROWS; p += span) clear_half(f + c / 64u * BOX_BYTES, p, r % 64u);
            }
        }
        settled();
        // ---- X' = a X + B X ----
        if (warp == 0 && elect_one()) {
            const uint32_t instruction = 1u << 4 | 1u << 16 | (a.width / 8) << 17 | (128u / 16) << 24;
#pragma unroll
            for (uint32_t i = 0; i < WHOLE_ROWS / 16; ++i) {
                if (i * 16u >= rows) break;
                mma_f16<false>(tmem + U_COLUMN, f_rows + (i / 4 * BOX_BYTES + i % 4 * 32u) / 16u, hi_columns + i * 2048u / 16u, instruction, i > 0);
            }
#pragma unroll
            for (uint32_t i = 0; i < WHOLE_ROWS / 16; ++i) {
                if (i * 16u >= rows || step >= ORTHO_TERMS_STEPS) break;
                mma_f16<false>(tmem + U_COLUMN, f_rows + (i / 4 * BOX_BYTES + i % 4 * 32u) / 16u, lo_columns + i * 2048u / 16u, instruction, true);
            }
            mma_commit<false>(bar);
        }
        __syncwarp();
        products_done();
        const float linear = a.ca + load_shared_float(db + ur * 4u);
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            const uint32_t c = ufirst + n * ustride, at = c / 64u * BOX_BYTES, o = c / 8u % 8u;
            if (c >= a.width || uidle) break;
            float w[16];
            __syncwarp();
            tmem_load16(tmem + (quarter * 32u << 16) + U_COLUMN + c, w);
            tmem_wait_load();
            update(w, x[n], linear);
            uint32_t h[8];
            if (!last) {
#pragma unroll
                for (int k = 0; k < 16; ++k) x[n][k] = cut_off(w[k]);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[k] = half_pair(w[2 * k], w[2 * k + 1]);
                if (step + 1 < ORTHO_TERMS_STEPS) {
                    uint32_t l[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) l[k] = rest_pair(x[n][2 * k], x[n][2 * k + 1], h[k]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) store_shared(box_octet(lo + at, ur, o + i), make_uint4(l[4 * i], l[4 * i + 1], l[4 * i + 2], l[4 * i + 3]));
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(w[2 * k] * (1.0f / XS), w[2 * k + 1] * (1.0f / XS));
                    h[k] = *reinterpret_cast<const uint32_t *>(&p);
                }
                if (a.turned) {
                    __nv_bfloat16 *to = a.out + blockIdx.y * a.out_stride + (c0 + c) * a.ldo + ur;
                    if (ur < a.m && ok)
#pragma unroll
                        for (int k = 0; k < 16; ++k, to += a.ldo)
                            if (c0 + c + k < a.n) {
                                const uint16_t e = (uint16_t)(h[k / 2] >> (16 * (k % 2)));
                                *to = *reinterpret_cast<const __nv_bfloat16 *>(&e);
                            }
                    continue;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) store_shared(box_octet(hi + at, ur, o + i), make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]));
        }
        __syncwarp();
        settled();
    }
    // ---- the result, row by row ----
    if (!a.turned && ok) {
        __nv_bfloat16 *const out = a.out + blockIdx.y * a.out_stride;
        for (uint32_t n = threadIdx.x; n < a.m * (a.width / 8); n += WHOLE_THREADS) {
            const uint32_t row = n / (a.width / 8), o = n % (a.width / 8), c = c0 + o * 8;
            if (c >= a.n) continue;
            const uint4 w = load_shared(box_octet(hi + o / 8 * BOX_BYTES, row, o % 8));
            __nv_bfloat16 *const to = out + row * a.ldo + c;
            if (a.out_vec && c + 8 <= a.n) {
                *reinterpret_cast<uint4 *>(to) = w;
            } else {
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint16_t e = (uint16_t)(u[k / 2] >> (16 * (k % 2)));
                    if (c + k < a.n) to[k] = *reinterpret_cast<const __nv_bfloat16 *>(&e);
                }
            }
        }
    }
    __syncwarp();
    if (threadIdx.x == 0 && *stop) {
        drain();
        atomicOr(a.status, QESGD_STATUS_TIMEOUT);
    }
    fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc<false>(tmem, 512u);
}

uint32_t whole_cluster(uint64_t n)
{
    uint32_t cluster = 1;
    while (cluster * WHOLE_COLS < n) cluster *= 2;
    return cluster;
}
// Large clusters come one after another where a batch has many (7 of 16 CTAs run at once): 16 matrices of 128 x 4096 take
// 224 us, and 176 as fifteen products.
bool takes_whole(uint64_t m, uint64_t n, uint64_t batch)
{
    if (m > WHOLE_ROWS || n > WHOLE_COLS * WHOLE_MAX_CLUSTER) return false;
    const uint32_t cluster = whole_cluster(n);
    if (cluster < 8) return true;
    static QesgdClusters known;
    static std::atomic<uint64_t> told{0};
    const void *const kernel = (const void *)qesgd_ortho_whole_kernel<float, true>;
    if (qesgd_prepare(told, kernel, WHOLE_MOST_SMEM, true) != cudaSuccess) return false;
    return batch <= 2 * qesgd_active_clusters(known, kernel, WHOLE_THREADS, WHOLE_MOST_SMEM, cluster);
}
template <typename T>
cudaError_t launch_whole(const OrthoArgs &o, cudaStream_t stream, int *launched, uint32_t *plan)
{
    WholeArgs a = {};
    a.x = o.x;
    a.ldx = o.ldx;
    a.x_stride = o.x_stride;
    a.ldo = o.ldo;
    a.out_stride = o.out_stride;
    a.m = (uint32_t)(o.rows < o.cols ? o.rows : o.cols);
    a.n = (uint32_t)(o.rows < o.cols ? o.cols : o.rows);
    a.turned = o.rows > o.cols;
    a.steps = o.steps;
    a.vec = qesgd_aligned(o.x, 16) && o.ldx * sizeof(T) % 16 == 0 && o.x_stride * sizeof(T) % 16 == 0;
    a.out_vec = qesgd_aligned(o.out, 16) && o.ldo % 8 == 0 && o.out_stride % 8 == 0;
    a.ca = o.a;
    a.cb = o.b;
    a.cc = o.c;
    a.out = static_cast<__nv_bfloat16 *>(o.out);
    a.status = o.status;
    const uint32_t cluster = whole_cluster(a.n);
    a.width = (a.n + cluster - 1) / cluster;
    a.width = (a.width + BOX_COLS - 1) / BOX_COLS * BOX_COLS;
    uint32_t smem = (2 * a.width / BOX_COLS + 2) * BOX_BYTES + WHOLE_EXTRA + 1024 + (cluster > 1 ? 128 * 128 * 4 : 0);
    if (smem < WHOLE_MIN_SMEM) smem = WHOLE_MIN_SMEM;
    const auto kernel = cluster > 1 ? qesgd_ortho_whole_kernel<T, true> : qesgd_ortho_whole_kernel<T, false>;
    static std::atomic<uint64_t> told[2];
    cudaError_t e = qesgd_prepare(told[cluster > 1], (const void *)kernel, WHOLE_MOST_SMEM, cluster > 1);
    if (e != cudaSuccess) return e;
    e = qesgd_launch_cluster(kernel, dim3(cluster, (unsigned)o.batch), dim3(WHOLE_THREADS), smem, cluster, stream, a);
    if (e == cudaSuccess) *launched = 1;
    plan[0] = QESGD_MATRIX_ORTHO_WHOLE;
    plan[1] = cluster;
    return e;
}

template <typename T>
cudaError_t start(const OrthoArgs &a, const OrthoLayout &l, cudaStream_t stream, int *launched)
{
    const T *const x = static_cast<const T *>(a.x);
    const bool vec = qesgd_aligned(x, 16) && a.ldx * sizeof(T) % 16 == 0 && a.x_stride * sizeof(T) % 16 == 0;
    const dim3 grid(l.parts, (unsigned)a.batch);
    const uint32_t rows = (uint32_t)a.rows, cols = (uint32_t)a.cols;
    double *const parts = reinterpret_cast<double *>(a.workspace);
    cudaError_t e = qesgd_launch(qesgd_ortho_norm_kernel<T>, grid, dim3(THREADS), stream, x, rows, cols, a.ldx, a.x_stride, vec, parts);
    if (e != cudaSuccess) return e;
    *launched += 1;
    const OrthoView v = {reinterpret_cast<__half *>(a.workspace + l.off_hi[0]), reinterpret_cast<__half *>(a.workspace + l.off_lo[0]), l.ld_x, l.x_stride};
    const dim3 squares((unsigned)(qesgd_div_up(rows, 64) * qesgd_div_up(cols, 64)), (unsigned)a.batch);
    e = qesgd_launch(rows > cols ? qesgd_ortho_start_kernel<T, true> : qesgd_ortho_start_kernel<T, false>, rows > cols ? squares : grid, dim3(THREADS), stream, x, rows, cols,
                     a.ldx, a.x_stride, vec, (const double *)parts, l.parts, v, a.status);
    if (e == cudaSuccess) *launched += 1;
    return e;
}

// 16-bit matrices [batch][rows][ld] of `cols` columns; a box is 64 columns of `box_rows` rows, 128-byte rows swizzled.
bool half_map(CUtensorMap *map, const void *p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t batch, uint64_t stride, uint32_t box_rows,
              CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_FLOAT16)
{
    const QesgdEncodeTiledFn encode = qesgd_encode_tiled();
    const cuuint64_t dims[3] = {cols, rows, batch}, strides[2] = {ld * 2, stride * 2};
    const cuuint32_t box[3] = {64u, box_rows, 1u}, unit[3] = {1u, 1u, 1u};
    return encode && encode(map, type, 3u, const_cast<void *>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product is launched: by single CTAs, of which 1, 2 or 4 share a contraction, by ones with narrow tiles, by pairs, or by pairs with
// the deep ring.  (qesgd_debug_matrix_plan tells.)
enum ProductShape : uint32_t { SINGLES = 1, SHARED_BY_2 = 2, SHARED_BY_4 = 4, NARROW_TILES = 8, PAIRS = 16, DEEP_PAIRS = 17 };

// f with the kernel of a shape, as an instance of Kernel.
template <int MODE_, bool PAIR_, bool DEEP_, bool NARROW_>
struct Kernel {
    static constexpr int MODE = MODE_;
    static constexpr bool PAIR = PAIR_, DEEP = DEEP_, NARROW = NARROW_;
};
template <int MODE, typename F>
cudaError_t with_kernel(uint32_t shape, const F &f)
{
    if (shape == NARROW_TILES) return f(Kernel<MODE, false, false, true>());
    if (shape == PAIRS) return f(Kernel<MODE, true, false, false>());
    if (shape == DEEP_PAIRS) return f(Kernel<MODE, true, MODE == UPDATE, false>());
    return f(Kernel<MODE, false, false, false>());
}
// Chooses the shape by modelled time, and tells its kernel what it needs.  Nothing is enqueued.
template <int MODE>
cudaError_t plan_product(const ProductArgs &a, int sm_count, uint32_t &shape)
{
    const auto tiles = [&](uint64_t side) {
        const uint64_t m = (a.rows + side - 1) / side, n = (a.cols + side - 1) / side;
        return (MODE == UPDATE ? m * n : m * (m + 1) / 2) * a.batch;
    };
    const double steps = (a.depth + DEPTH - 1) / DEPTH * a.terms, sms = sm_count;
    const double singles = (double)tiles(128), pairs = (double)tiles(256);
    // clocks: a stage of one CTA takes 450 (few CTAs) to 650 (all SMs) to arrive, one of a pair 512 to 690
    const auto stage = [&](double ctas, double few, double many) { return few + (many - few) * (ctas < sms ? ctas / sms : 1.0); };
    const auto waves = [&](double n, double most) { return (double)(uint64_t)((n + most - 1) / most); };
    double best = waves(pairs, (double)(sm_count / 2)) * steps * stage(2 * pairs, 512, 690) + 5000;
    shape = MODE == UPDATE && a.depth >= 2048 ? DEEP_PAIRS : PAIRS;
    for (uint32_t s = 1; s <= 4; s *= 2) {
        if (s > 1 && (singles * s > sms || steps < 4 * s)) break;
        static QesgdClusters known;
        static std::atomic<uint64_t> told{0};
        const void *const kernel = (const void *)qesgd_ortho_product_kernel<MODE, false, false, false>;
        const uint32_t smem = Shape<MODE, false, false, false>::SMEM;
        if (s > 1 && qesgd_prepare(told, kernel, (int)smem, false) != cudaSuccess) break;
        const double active = s > 1 ? (double)qesgd_active_clusters(known, kernel, WARPS * 32, smem, s) : sms;
        const double t = waves(singles, active) * (double)(uint64_t)((steps + s - 1) / s) * stage(singles * s, 450, 650) + 2500 + (s > 1 ? 2000 : 0);
        if (t < best) {
            best = t;
            shape = s;
        }
    }
    // narrow tiles: 350 to 500 clocks a stage, and 1200 less at the end
    const double strips = MODE == UPDATE ? (double)(((uint64_t)a.rows + 127) / 128 * ((a.cols + 63) / 64) * a.batch) : 2 * singles;
    if (waves(strips, sms) * steps * stage(strips, 350, 500) + 1300 < best) shape = NARROW_TILES;
    return with_kernel<MODE>(shape, [](auto k) {
        using K = decltype(k);
        static std::atomic<uint64_t> told{0};
        return qesgd_prepare(told, (const void *)qesgd_ortho_product_kernel<MODE, K::PAIR, K::DEEP, K::NARROW>, Shape<MODE, K::PAIR, K::DEEP, K::NARROW>::SMEM, false);
    });
}
template <int MODE>
cudaError_t launch_product(ProductArgs a, ProductMaps maps, uint32_t shape, int sm_count, cudaStream_t stream)
{
    return with_kernel<MODE>(shape, [&](auto k) {
        using K = decltype(k);
        using S = Shape<MODE, K::PAIR, K::DEEP, K::NARROW>;
        if (K::NARROW && MODE != UPDATE) maps.q = maps.q_narrow;
        a.tiles_m = (a.rows + S::SIDE - 1) / S::SIDE;
        a.tiles = MODE == UPDATE ? a.tiles_m * ((a.cols + S::WIDTH - 1) / S::WIDTH) : a.tiles_m * (a.tiles_m + 1) / 2 * (S::SIDE / S::WIDTH);
        a.split = K::PAIR || K::NARROW ? 1u : shape;
        const uint32_t share = K::PAIR ? 2u : a.split, all = a.tiles * a.batch, most = (uint32_t)sm_count / share;
        return qesgd_launch_cluster(qesgd_ortho_product_kernel<MODE, K::PAIR, K::DEEP, K::NARROW>, dim3((a.split > 1 || all < most ? all : most) * share), dim3(WARPS * 32),
                                    S::SMEM, share, stream, a, maps);
    });
}

}  // namespace

int qesgd_launch_orthogonalize(const OrthoArgs &a, int sm_count, cudaStream_t stream, int *launched, uint32_t *plan)
{
    *launched = 0;
    if (takes_whole(a.rows < a.cols ? a.rows : a.cols, a.rows < a.cols ? a.cols : a.rows, a.batch))
        return (int)(a.dtype == QESGD_F32    ? launch_whole<float>(a, stream, launched, plan)
                     : a.dtype == QESGD_BF16 ? launch_whole<__nv_bfloat16>(a, stream, launched, plan)
                                             : launch_whole<__half>(a, stream, launched, plan));
    const OrthoLayout l = qesgd_ortho_layout(a.rows, a.cols, a.batch);
    const auto at = [&](uint64_t off) { return reinterpret_cast<__half *>(a.workspace + off); };
    CUtensorMap hi[2], lo[2], across[2], across_lo[2], f, b, hi_64[2], f_64;   // X's terms by rows, and across them, F, B; 64 rows of them
    bool ok = half_map(&f, at(l.off_a), l.m, l.m, l.ld_a, a.batch, l.a_stride, 128) && half_map(&b, at(l.off_b), l.m, l.m, l.ld_a, a.batch, l.a_stride, 128) &&
              half_map(&f_64, at(l.off_a), l.m, l.m, l.ld_a, a.batch, l.a_stride, 64);
    for (int i = 0; i < 2; ++i)
        ok = ok && half_map(&hi[i], at(l.off_hi[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, 128) &&
             half_map(&hi_64[i], at(l.off_hi[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, 64) &&
             half_map(&lo[i], at(l.off_lo[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, 128) &&
             half_map(&across[i], at(l.off_hi[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, DEPTH) &&
             half_map(&across_lo[i], at(l.off_lo[i]), l.m, l.n, l.ld_x, a.batch, l.x_stride, DEPTH);
    if (!ok) return (int)cudaErrorInvalidValue;
    ProductArgs gram = {};
    gram.batch = (uint32_t)a.batch;
    gram.d = reinterpret_cast<float *>(a.workspace + l.off_d);
    gram.db = gram.d + a.batch * l.d_stride;
    gram.ld_a = l.ld_a;
    gram.a_stride = l.a_stride;
    gram.d_stride = l.d_stride;
    gram.ca = a.a;
    gram.cb = a.b;
    gram.cc = a.c;
    gram.status = a.status;
    gram.rows = gram.cols = (uint32_t)l.m;
    gram.depth = (uint32_t)l.n;
    gram.terms = 1;
    gram.mirror = at(l.off_a);
    ProductArgs poly = gram, update[2];   // an update of one term of X, and of both
    poly.depth = (uint32_t)l.m;
    poly.mirror = at(l.off_b);
    update[0] = poly;
    update[0].cols = (uint32_t)l.n;
    update[1] = update[0];
    update[1].terms = 2;
    const uint32_t both = l.m < ORTHO_TERMS_SIDE ? ORTHO_TERMS_STEPS : 0;   // steps whose update takes both
    uint32_t by_gram, by_poly, by_update[2] = {0, 0};
    cudaError_t e = plan_product<GRAM>(gram, sm_count, by_gram);
    if (e == cudaSuccess) e = plan_product<POLY>(poly, sm_count, by_poly);
    if (e == cudaSuccess && both < a.steps) e = plan_product<UPDATE>(update[0], sm_count, by_update[0]);
    if (e == cudaSuccess && both > 0) e = plan_product<UPDATE>(update[1], sm_count, by_update[1]);
    if (e != cudaSuccess) return (int)e;
    plan[0] = QESGD_MATRIX_ORTHO_PRODUCTS;
    plan[1] = by_gram;
    plan[2] = by_poly;
    plan[3] = by_update[1];
    plan[4] = by_update[0];

    e = a.dtype == QESGD_F32 ? start<float>(a, l, stream, launched) : a.dtype == QESGD_BF16 ? start<__nv_bfloat16>(a, l, stream, launched) : start<__half>(a, l, stream, launched);
    if (e != cudaSuccess) return (int)e;
    for (uint32_t step = 0; step < a.steps; ++step) {
        const uint32_t now = step % 2, next = 1 - now;
        e = launch_product<GRAM>(gram, {hi[now], hi[now], hi[now], f, f, f, f, hi_64[now]}, by_gram, sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
        e = launch_product<POLY>(poly, {f, f, f, f, f, b, b, f_64}, by_poly, sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
        ProductArgs p = update[step < both];
        if (step + 1 == a.steps) {
            p.out = static_cast<__nv_bfloat16 *>(a.out);
            p.ldo = a.ldo;
            p.out_stride = a.out_stride;
            p.turned = a.rows > a.cols;
            // a batch of one matrix has no stride of its own
            const uint64_t stride = a.batch > 1 ? a.out_stride : (a.rows * a.ldo + 7) / 8 * 8;
            p.out_tiled = !p.turned && qesgd_aligned(a.out, 16) && a.ldo % 8 == 0 && stride % 8 == 0 &&
                          half_map(&hi[next], a.out, l.m, l.n, a.ldo, a.batch, stride, 128, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16);
        }
        e = launch_product<UPDATE>(p, {b, across[now], across_lo[now], hi[now], lo[now], hi[next], lo[next], across[now]}, by_update[step < both], sm_count, stream);
        if (e != cudaSuccess) return (int)e;
        *launched += 1;
    }
    return 0;
}
