// Microscaled 4-bit floats: a matrix quantised with blocks along its rows, along its columns (the transpose), or
// both in one read; the way back; and the exponent of a whole tensor.  Definitions are stated in include/qesgd.h.
//
// This file must be compiled with -fmad=false: the choice of a level is a sequence of single IEEE operations.
//
// A lane has 16 consecutive elements of a row, two octets: 32 or 64 bytes of input, two Philox4x32-10 blocks of 8 draws
// each, two 32-bit words of codes.  A block of 16 is in one lane, one of 32 in two neighbours, so its largest magnitude
// takes no shuffle or one.
//
// Memory is the floor, and nothing else is full either.  4096 x 4096 fp32 with draws takes 26 instructions an element (5 of them
// Philox's): while an SM is at work it issues in 71 % of its slots (integer pipe 62 %, DRAM 37 %), in the rest none of its 27
// warps has its data, and 1024 tiles on 592 that run at once leave SMs without work for 21 % of the time.  8192 x 8192 bf16 along
// both axes, 20 instructions an element for both: 72 %, 66 % and 37 %, without work 9 %.  With the ways back to bf16 27 and 116 us,
// where the bytes take 18 and 85.
#include <type_traits>

#include "qesgd_matrix.cuh"

namespace {

constexpr uint32_t FULL = 0xFFFFFFFFu;
constexpr int THREADS = 256;
constexpr int TILE_ROWS = 128;       // rows of a tile of scales
constexpr int SCALE_TILE = 512;      // bytes of it: 128 rows by 4 blocks

template <int FORMAT>
struct Format;
template <>
struct Format<QESGD_FP4_MX> {
    static constexpr int BLOCK = 32;
};
template <>
struct Format<QESGD_FP4_NV> {
    static constexpr int BLOCK = 16;
};

// The eight 16-bit draws of octet `n` (Philox4x32 with 10 rounds, round keys prepared on the host), as in the encode
// kernel: draw j is half j % 2 of word j / 2.
__device__ __forceinline__ void draws_of(uint64_t n, const Fp4QuantizeArgs &a, uint32_t (&x)[4])
{
    x[0] = (uint32_t)n;
    x[1] = (uint32_t)(n >> 32);
    x[2] = a.worker;
    x[3] = a.epoch;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * x[0];
        const uint64_t p1 = (uint64_t)0xCD9E8D57u * x[2];
        const uint32_t n0 = (uint32_t)(p1 >> 32) ^ x[1] ^ a.round_key[r][0];
        const uint32_t n2 = (uint32_t)(p0 >> 32) ^ x[3] ^ a.round_key[r][1];
        x[1] = (uint32_t)p1;
        x[3] = (uint32_t)p0;
        x[0] = n0;
        x[2] = n2;
    }
}

__device__ __forceinline__ int clamp_exponent(int t) { return min(max(t, -126), 126); }
__device__ __forceinline__ int tensor_exponent(const int32_t *p) { return p ? clamp_exponent(__ldg(p)) : 0; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// A block's scale, from the bits of its largest magnitude: the byte that is kept, and what its elements are multiplied by
// (and, NV, by the reciprocal of s).
struct Scale {
    uint32_t byte;
    float mul;    // 2^-e (MX), 2^-t (NV)
    float2 inv;   // 1 / s in two terms (NV), 0 for s = 0
    bool bad;     // something in the block is not finite
};
__device__ __forceinline__ float e4m3(uint32_t code, float factor) { return __fmul_rn(__uint_as_float(code << 20), factor); }   // factor: a power of two or 6 of them, times 2^120
// inverse: 1 / s of every E4M3 number, in shared memory (__frcp_rn of each block's takes ten instructions)
template <int FORMAT, bool SCALED>
__device__ __forceinline__ Scale block_scale(uint32_t top, float to_tensor, const float2 *inverse)
{
    Scale s;
    s.bad = top >= 0x7F800000u;
    if (FORMAT == QESGD_FP4_MX) {
        // top = 1.f * 2^(E - 127) is at most 6 * 2^e = 1.5 * 2^(e + 2) from e = E - 129 on, one later where 1.f > 1.5: where the
        // mantissa carries
        s.byte = s.bad ? 0u : (uint32_t)max((int)((top + 0x3FFFFFu) >> 23) - 2, 0);
        s.mul = __uint_as_float((254u - s.byte) << 23);
        s.inv = make_float2(1.0f, 0.0f);
    } else {
        // The bits of an E4M3 number are bits 20..26 of the float 2^-120 times it, subnormals included.  A quotient by 6 that is
        // rounded down, and then up to such bits, is right or one number short; 6 s is exact.
        float v = __uint_as_float(s.bad ? 0u : top);
        if (SCALED) v = __fmul_rn(v, to_tensor);
        uint32_t code = min((__float_as_uint(__fmul_rd(v, 0x1.555554p-123f)) + 0xFFFFFu) >> 20, 126u);
        code = min(code + (e4m3(code, 6.0f * 0x1p120f) < v ? 1u : 0u), 126u);
        if (SCALED) code = max(code, s.bad || top == 0u ? 0u : 1u);   // top * 2^-t may be 0
        s.byte = code;
        s.inv = inverse[code];
        s.mul = to_tensor;
    }
    return s;
}
__device__ __forceinline__ void fill_inverse(float2 *inverse)
{
    if (threadIdx.x >= 128) return;
    const float s = e4m3(threadIdx.x, 0x1p120f), r = threadIdx.x ? __frcp_rn(s) : 0.0f;
    inverse[threadIdx.x] = make_float2(r, __fmul_rn(__fmaf_rn(-r, s, 1.0f), r));
}
// x over the block's scale, correctly rounded.  NV: x times 1 / s in two terms is 2^-47 off the quotient at most; s has 4
// significant bits, so a quotient lies on a rounding border or at least 2^-5 units in the last place from it.  (One
// term is not enough for 16-bit x either: 1.25 times 1.875 times fl32(1 / 1.875) passes the tie at 1.25.)  SCALED: there is
// a tensor exponent, and x * 2^-t may leave the float range: it is clipped to 6 either way.
template <int FORMAT, bool SCALED>
__device__ __forceinline__ float over_scale(float x, const Scale &s)
{
    if (FORMAT == QESGD_FP4_MX) return __fmul_rn(x, s.mul);
    const float y = SCALED ? fminf(fmaxf(__fmul_rn(x, s.mul), -3.402823466e38f), 3.402823466e38f) : x;
    return __fmaf_rn(y, s.inv.x, __fmul_rn(y, s.inv.y));
}

// The same for two elements at once (sm_100 multiplies and adds pairs of floats in one instruction: 8192 x 8192 along both
// axes and back 118 -> 116 us).
template <int FORMAT, bool SCALED>
__device__ __forceinline__ void over_scale(float &a, float &b, const Scale &s)
{
    if (SCALED) {
        a = over_scale<FORMAT, SCALED>(a, s);
        b = over_scale<FORMAT, SCALED>(b, s);
    } else if (FORMAT == QESGD_FP4_MX) {
        asm("{\n.reg .b64 x, m;\nmov.b64 x, {%0, %1};\nmov.b64 m, {%2, %2};\nmul.rn.f32x2 x, x, m;\nmov.b64 {%0, %1}, x;\n}" : "+f"(a), "+f"(b) : "f"(s.mul));
    } else {
        asm("{\n.reg .b64 x, h, l;\nmov.b64 x, {%0, %1};\nmov.b64 h, {%2, %2};\nmov.b64 l, {%3, %3};\nmul.rn.f32x2 l, x, l;\nfma.rn.f32x2 x, x, h, l;\nmov.b64 {%0, %1}, x;\n}"
            : "+f"(a), "+f"(b)
            : "f"(s.inv.x), "f"(s.inv.y));
    }
}

// Eight elements of one block -> their codes.
template <int FORMAT, bool SCALED, bool STOCHASTIC>
__device__ __forceinline__ uint32_t quantize_octet(const float (&v)[8], const Scale &s, const uint32_t (&draw)[4])
{
    uint32_t w = 0u;
    if (!STOCHASTIC) {
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = v[j];
#pragma unroll
        for (int j = 0; j < 8; j += 2) over_scale<FORMAT, SCALED>(q[j], q[j + 1], s);
        asm("{\n"
            ".reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3};\n"
            "}\n"
            : "=r"(w)
            : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    } else {
        // Behind q2 = max(q + 1, 2 q) (the first below 1, the second above) the grid is that of floats with one bit of mantissa,
        // from 1.0 on: the level is what bits 22 and up of q2 count, and one more where the bits below, R / 2^22 of a step, are
        // more than the draw's u = (2 k + 1) / 2^17: where R + 2^22 - 1 - 32 (2 k + 1) carries.  Both are integers, and q + 1,
        // rounded upwards, compares with them as the exact sum does.  Times 64 the level stands in the top four bits (and a
        // bit of the exponent with it), from which funnel shifts collect the word; 254 counts up to 1.0.
        uint32_t signs = 0u;
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            const float x = fabsf(over_scale<FORMAT, SCALED>(v[j], s));
            const float q = FORMAT == QESGD_FP4_MX ? x : fminf(x, 6.0f);   // MX: never above 6
            const float q2 = fmaxf(__fadd_ru(q, 1.0f), __fadd_rn(q, q));
            const uint32_t k = j % 2 ? draw[j / 2] >> 16 : draw[j / 2] & 0xFFFFu;
            const uint32_t t = __float_as_uint(q2) * 64u + ((((1u << 22) - 33u) - (254u << 22)) * 64u - k * 4096u);
            w = __funnelshift_l(t, w, 4);
            signs = __funnelshift_l(__float_as_uint(v[j]), signs, 4);
        }
        w = (w & 0x77777777u) | (signs & 0x88888888u);
    }
    // a zero has no sign: the top bit of a half stays where its level is 1 at least
    w &= 0x77777777u | ((w & 0x77777777u) + 0x77777777u);
    return s.bad ? 0u : w;
}

// Byte of (row, block) within the tiles that a CTA keeps in shared memory, one after another along the blocks.
__device__ __forceinline__ uint32_t scale_slot(uint32_t row, uint32_t block)
{
    return block / 4u * SCALE_TILE + (row % 32u) * 16u + (row / 32u) * 4u + block % 4u;
}

// The largest magnitude of a block, of which a lane has one whole (NV) or its neighbour the other half (MX).
template <int FORMAT>
__device__ __forceinline__ uint32_t over_block(uint32_t top)
{
    return FORMAT == QESGD_FP4_MX ? max(top, __shfl_xor_sync(FULL, top, 1)) : top;
}
// Two octets of a row -> two words of codes, and their block's scale.
template <typename T, int FORMAT, bool SCALED, bool STOCHASTIC>
__device__ __forceinline__ uint2 quantize_span(const Octet<T> (&x)[2], uint64_t n, float to_tensor, const float2 *inverse, const Fp4QuantizeArgs &a, Scale &s)
{
    s = block_scale<FORMAT, SCALED>(over_block<FORMAT>(max(top_of(x[0]), top_of(x[1]))), to_tensor, inverse);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t draw[4] = {0u, 0u, 0u, 0u};
        if (STOCHASTIC) draws_of(n + i, a, draw);
        float v[8];
        values(x[i], v);
        w[i] = quantize_octet<FORMAT, SCALED, STOCHASTIC>(v, s, draw);
    }
    return make_uint2(w[0], w[1]);
}

// ------------------------------------------------------- blocks along rows ----
// A CTA's tile: 64 rows (or 32), part of a tile of scales, by 256 columns, 16 for each lane, two rows for a warp at a time.
constexpr int ROW_COLS = 256;

template <typename T, int FORMAT, bool SCALED, bool STOCHASTIC, int ROWS>
__global__ __launch_bounds__(THREADS, 4) void qesgd_fp4_quantize_rows_kernel(const __grid_constant__ Fp4QuantizeArgs a)
{
    constexpr int BLOCK = Format<FORMAT>::BLOCK;
    constexpr int TILES = ROW_COLS / BLOCK / 4;        // of scales
    constexpr int UNROLL = sizeof(T) == 4 ? 1 : 2;
    __shared__ __align__(16) uint8_t scales[TILES * SCALE_TILE];   // the first 8 (or 4) of every 16 bytes
    __shared__ float2 inverse[128];
    if (FORMAT == QESGD_FP4_NV) fill_inverse(inverse);
    qesgd_wait_for_previous();
    const uint32_t o = threadIdx.x % 16u, line = threadIdx.x / 16u;
    const uint32_t col_tiles = (uint32_t)((a.cols + ROW_COLS - 1) / ROW_COLS);
    const uint64_t tiles = (uint64_t)col_tiles * ((a.rows + TILE_ROWS - 1) / TILE_ROWS * (TILE_ROWS / ROWS));
    const uint64_t padded = (a.cols + 31) / 32 * 32;
    const uint64_t scale_tiles = (a.cols + 4 * BLOCK - 1) / (4 * BLOCK);
    const float to_tensor = SCALED ? power_of_two(-tensor_exponent(a.tensor_exponent)) : 1.0f;
    bool bad = false;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t row0 = tile / col_tiles * ROWS;
        const uint32_t col0 = (uint32_t)(tile % col_tiles) * ROW_COLS;
        const uint32_t rows = row0 < a.rows ? (uint32_t)min((uint64_t)ROWS, a.rows - row0) : 0u;
        if (rows < ROWS)
            for (uint32_t i = threadIdx.x; i < sizeof(scales) / 4; i += THREADS) reinterpret_cast<uint32_t *>(scales)[i] = 0u;
        __syncthreads();
        const uint64_t c = col0 + o * 16u;
        const T *from = static_cast<const T *>(a.x) + (row0 + line) * a.ldx;
        uint64_t n = ((row0 + line) * padded + c) / 8;
        const auto load = [&](Octet<T> (&x)[UNROLL][2], uint32_t r0) {
#pragma unroll
            for (int i = 0; i < UNROLL; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    x[i][k] = r0 + i * (THREADS / 16) < rows ? load_octet(from + i * (THREADS / 16) * a.ldx, c + 8 * k, a.cols, a.vec) : no_octet<T>();
            from += UNROLL * (THREADS / 16) * a.ldx;
        };
        Octet<T> next[UNROLL][2];
        load(next, line);
#pragma unroll 1
        for (uint32_t r0 = line; r0 < (rows + 1u) / 2u * 2u; r0 += THREADS / 16 * UNROLL) {   // both halves of a warp stay together
            Octet<T> x[UNROLL][2];
#pragma unroll
            for (int i = 0; i < UNROLL; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) x[i][k] = next[i][k];
            load(next, r0 + THREADS / 16 * UNROLL);
#pragma unroll
            for (int i = 0; i < UNROLL; ++i, n += (THREADS / 16) * (padded / 8)) {
                const uint32_t r = r0 + i * (THREADS / 16);
                Scale s;
                const uint2 w = quantize_span<T, FORMAT, SCALED, STOCHASTIC>(x[i], n, to_tensor, inverse, a, s);
                if (r >= rows) continue;
                bad |= s.bad;
                if (c < padded) *reinterpret_cast<uint2 *>(a.codes + n * 4) = w;
                const uint32_t block = o * 16u / BLOCK;
                if (o * 16u % BLOCK == 0u) scales[block / 4u * SCALE_TILE + r % 32u * 16u + r / 32u * 4u + block % 4u] = (uint8_t)s.byte;
            }
            __syncwarp();
        }
        __syncthreads();
        const uint64_t at = col0 / (4 * BLOCK);
        const uint32_t have = (uint32_t)min((uint64_t)TILES, scale_tiles - at);
        uint8_t *const out = a.scales + (row0 / TILE_ROWS * scale_tiles + at) * SCALE_TILE + row0 / 32 % 4 * 4;
        using Rows = std::conditional_t<ROWS == 64, uint2, uint32_t>;   // rows 32 apart are neighbours
        for (uint32_t i = threadIdx.x; i < have * (SCALE_TILE / 16); i += THREADS)
            *reinterpret_cast<Rows *>(out + i * 16u) = *reinterpret_cast<const Rows *>(scales + i * 16u);
        __syncthreads();
    }
    if (bad) atomicOr(a.status, QESGD_STATUS_NONFINITE);
}

// ------------------------------- blocks along columns, or along both axes ----
constexpr int SIDE = 128;   // a CTA's tile: whole tiles of scales for either axis

// Where element (r, c) of the tile lies in shared memory: rows one after another, the 16-byte lines of each turned by one
// more for every eight of them, so that eight lanes meet eight different banks when they store two or four lines apart
// and when they load neighbouring ones.
template <typename T>
__device__ __forceinline__ uint32_t held_at(uint32_t r, uint32_t c)
{
    const uint32_t at = c * sizeof(T), line = at / 16u;
    return r * (SIDE * sizeof(T)) + (line & ~7u) * 16u + ((line + line / 8u) & 7u) * 16u + at % 16u;
}

// The tile goes through shared memory as it is.  Then a thread takes two neighbouring columns of 32 rows: one load for both
// where elements have 16 bits, whole blocks without an exchange, and 16 bytes of codes for each column.
template <typename T, int FORMAT, bool SCALED, bool STOCHASTIC>
__global__ __launch_bounds__(THREADS) void qesgd_fp4_quantize_columns_kernel(const __grid_constant__ Fp4QuantizeArgs a)
{
    constexpr int BLOCK = Format<FORMAT>::BLOCK;
    constexpr int BLOCKS = SIDE / BLOCK;
    extern __shared__ __align__(16) uint8_t held[];
    __shared__ __align__(16) uint8_t scales[2][SIDE * BLOCKS];
    __shared__ float2 inverse[128];
    if (FORMAT == QESGD_FP4_NV) fill_inverse(inverse);
    __syncthreads();
    qesgd_wait_for_previous();
    const uint32_t col_tiles = (uint32_t)((a.cols + SIDE - 1) / SIDE);
    const uint64_t tiles = (uint64_t)col_tiles * ((a.rows + SIDE - 1) / SIDE);
    const uint64_t padded = (a.cols + 31) / 32 * 32, padded_t = (a.rows + 31) / 32 * 32;
    const uint64_t scale_tiles = (a.cols + 4 * BLOCK - 1) / (4 * BLOCK), scale_tiles_t = (a.rows + 4 * BLOCK - 1) / (4 * BLOCK);
    const float to_tensor = SCALED ? power_of_two(-tensor_exponent(a.tensor_exponent)) : 1.0f;
    bool bad = false;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t row0 = tile / col_tiles * SIDE, col0 = tile % col_tiles * SIDE;
        {
            // every row and column of the tile goes the whole way, as zeros past the matrix's edge: then padding bytes are zeros
            constexpr int UNROLL = sizeof(T) == 4 ? 1 : 2;
            const uint32_t o = threadIdx.x % 8u, line = threadIdx.x / 8u;
            const uint64_t c = col0 + o * 16u;
            const T *from = static_cast<const T *>(a.x) + (row0 + line) * a.ldx;
            uint64_t n = ((row0 + line) * padded + c) / 8;
#pragma unroll 1
            for (uint32_t i0 = line; i0 < SIDE; i0 += THREADS / 8 * UNROLL) {
                Octet<T> x[UNROLL][2];
#pragma unroll
                for (int i = 0; i < UNROLL; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        x[i][k] = row0 + i0 + i * (THREADS / 8) < a.rows ? load_octet(from + i * (THREADS / 8) * a.ldx, c + 8 * k, a.cols, a.vec) : no_octet<T>();
                from += UNROLL * (THREADS / 8) * a.ldx;
#pragma unroll
                for (int i = 0; i < UNROLL; ++i, n += (THREADS / 8) * (padded / 8)) {
                    const uint32_t r = i0 + i * (THREADS / 8);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int q = 0; q < Octet<T>::WORDS / 4; ++q)
                            *reinterpret_cast<uint4 *>(held + held_at<T>(r, o * 16u + k * 8u + q * (16 / sizeof(T)))) = *reinterpret_cast<const uint4 *>(&x[i][k].w[4 * q]);
                    if (a.codes) {
                        Scale s;
                        const uint2 w = quantize_span<T, FORMAT, SCALED, STOCHASTIC>(x[i], n, to_tensor, inverse, a, s);
                        bad |= s.bad;
                        if (row0 + r < a.rows && c < padded) *reinterpret_cast<uint2 *>(a.codes + n * 4) = w;
                        if (o * 16u % BLOCK == 0u) scales[0][scale_slot(r, o * 16u / BLOCK)] = (uint8_t)s.byte;
                    }
                }
            }
        }
        __syncthreads();
        {
            const uint32_t k = threadIdx.x % (SIDE / 2) * 2u, i0 = threadIdx.x / (SIDE / 2) * 32u;
            uint32_t words[2][4];
#pragma unroll
            for (int g = 0; g < 32 / BLOCK; ++g) {
                float v[2][BLOCK];
                uint32_t top[2] = {0u, 0u}, both = 0u;
#pragma unroll
                for (int j = 0; j < BLOCK; ++j) {
                    const uint8_t *const p = held + held_at<T>(i0 + g * BLOCK + j, k);
                    if constexpr (sizeof(T) == 4) {
                        const uint2 w = *reinterpret_cast<const uint2 *>(p);
                        v[0][j] = __uint_as_float(w.x);
                        v[1][j] = __uint_as_float(w.y);
                        top[0] = max(top[0], w.x & 0x7FFFFFFFu);
                        top[1] = max(top[1], w.y & 0x7FFFFFFFu);
                    } else {
                        const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
                        const float2 f = pair_of(w, T());
                        v[0][j] = f.x;
                        v[1][j] = f.y;
                        both = __vmaxu2(both, w & 0x7FFF7FFFu);
                    }
                }
                if constexpr (sizeof(T) == 2) {
                    top[0] = top16<T>(both & 0xFFFFu);
                    top[1] = top16<T>(both >> 16);
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint64_t c = col0 + k + n;
                    const Scale s = block_scale<FORMAT, SCALED>(top[n], to_tensor, inverse);
                    bad |= s.bad;
#pragma unroll
                    for (int o = 0; o < BLOCK / 8; ++o) {
                        uint32_t draw[4] = {0u, 0u, 0u, 0u};
                        if (STOCHASTIC) draws_of((c * padded_t + row0 + i0 + g * BLOCK + o * 8) / 8, a, draw);
                        float e[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] = v[n][o * 8 + j];
                        words[n][g * (BLOCK / 8) + o] = quantize_octet<FORMAT, SCALED, STOCHASTIC>(e, s, draw);
                    }
                    scales[1][scale_slot(k + n, (i0 + g * BLOCK) / BLOCK)] = (uint8_t)s.byte;
                }
            }
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint64_t c = col0 + k + n;
                if (c < a.cols && row0 + i0 < padded_t)
                    *reinterpret_cast<uint4 *>(a.codes_t + (c * padded_t + row0 + i0) / 2) = make_uint4(words[n][0], words[n][1], words[n][2], words[n][3]);
            }
        }
        __syncthreads();
        for (int side = a.codes ? 0 : 1; side < 2; ++side) {
            const uint64_t all = side ? scale_tiles_t : scale_tiles;
            const uint64_t at = (side ? row0 : col0) / (4 * BLOCK), line = (side ? col0 : row0) / TILE_ROWS;
            const uint32_t have = (uint32_t)min((uint64_t)(BLOCKS / 4), all - at);
            uint4 *out = reinterpret_cast<uint4 *>((side ? a.scales_t : a.scales) + (line * all + at) * SCALE_TILE);
            for (uint32_t i = threadIdx.x; i < have * (SCALE_TILE / 16); i += THREADS) out[i] = reinterpret_cast<const uint4 *>(scales[side])[i];
        }
        __syncthreads();
    }
    if (bad) atomicOr(a.status, QESGD_STATUS_NONFINITE);
}

// --------------------------------------------------------------- way back ----
// grid values of the two codes of a byte
__device__ __forceinline__ float2 values_of(uint32_t byte)
{
    uint32_t h;
    asm("{\n"
        ".reg .b8 b;\n"
        ".reg .b16 w;\n"
        "cvt.u16.u32 w, %1;\n"
        "cvt.u8.u16 b, w;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b;\n"
        "}\n" : "=r"(h) : "r"(byte));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
template <int FORMAT>
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    // 2^(byte - 127), 2^-127 being a subnormal float; or the E4M3 number of these bits
    if (FORMAT == QESGD_FP4_MX) return byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
    return __fmul_rn(__uint_as_float((byte & 0x7Fu) << 20), 0x1p120f);
}

// A warp takes 256 columns of a row at a time, an octet for each lane.  Where rows of `out` lie on 16 bytes the octet is
// stored as it is; else it goes through shared memory, so that neighbouring lanes store neighbouring elements (two at a
// time where a row of 16-bit elements begins on 4 bytes).
constexpr int BACK_ROWS = 32, BACK_COLS = 256;

template <typename T, int FORMAT, bool VEC>
__global__ __launch_bounds__(THREADS) void qesgd_fp4_dequantize_kernel(const __grid_constant__ Fp4DequantizeArgs a)
{
    constexpr int BLOCK = Format<FORMAT>::BLOCK;
    constexpr int UNROLL = BACK_ROWS / (THREADS / 32);
    __shared__ __align__(16) T turned[VEC ? 8 : THREADS / 32 * BACK_COLS];
    qesgd_wait_for_previous();
    const uint32_t lane = threadIdx.x % 32u, warp = threadIdx.x / 32u;
    T *const mine = turned + (VEC ? 0 : warp * BACK_COLS);
    const uint64_t padded = (a.cols + 31) / 32 * 32, scale_tiles = (a.cols + 4 * BLOCK - 1) / (4 * BLOCK);
    const uint32_t col_tiles = (uint32_t)((a.cols + BACK_COLS - 1) / BACK_COLS);
    const uint64_t tiles = (uint64_t)col_tiles * ((a.rows + BACK_ROWS - 1) / BACK_ROWS);
    // far exponents take two factors: their product with a scale may not be a 32-bit number
    const int t = tensor_exponent(a.tensor_exponent);
    const float near = t >= -100 && t <= 100 ? power_of_two(t) : 1.0f, far = t >= -100 && t <= 100 ? 1.0f : power_of_two(t);
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t row0 = tile / col_tiles * BACK_ROWS;
        const uint32_t col0 = (uint32_t)(tile % col_tiles) * BACK_COLS;
        // within a tile of scales: 32 rows lie 16 bytes apart, then the next quarter begins
        static_assert(BACK_ROWS == 32, "a quarter of a tile of scales");
        const uint8_t *const scales = a.scales + row0 / 128 * scale_tiles * SCALE_TILE + row0 / 32 % 4 * 4;
        const uint32_t rows = (uint32_t)min((uint64_t)BACK_ROWS, a.rows - row0);
        const uint32_t cols = (uint32_t)min((uint64_t)BACK_COLS, a.cols - col0);   // of this tile
        const uint32_t c = lane * 8u, block = c / BLOCK;                           // col0 begins a tile of scales
        const uint8_t *const at = scales + (uint64_t)(col0 / (4u * BLOCK) + block / 4u) * SCALE_TILE + block % 4u + warp * 16u;
        const uint8_t *const codes = a.codes + ((row0 + warp) * padded + col0 + c) / 2;
        T *out = static_cast<T *>(a.out) + (row0 + warp) * a.ldo + col0;
        uint32_t w[UNROLL], byte[UNROLL];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            const bool inside = warp + i * (THREADS / 32) < rows && c < cols;
            byte[i] = inside ? at[i * (THREADS / 32) * 16] : 0u;
            w[i] = inside ? *reinterpret_cast<const uint32_t *>(codes + i * (THREADS / 64) * padded) : 0u;
        }
#pragma unroll
        for (int i = 0; i < UNROLL; ++i, out += (THREADS / 32) * a.ldo) {
            if (warp + i * (THREADS / 32) >= rows) break;
            const float scale = __fmul_rn(scale_value<FORMAT>(byte[i]), near);
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 p = values_of((w[i] >> (8 * j)) & 0xFFu);
                f[2 * j] = __fmul_rn(p.x, scale);
                f[2 * j + 1] = __fmul_rn(p.y, scale);
            }
            if (far != 1.0f)
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = __fmul_rn(f[j], far);
            __align__(16) T v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = from_float<T>(f[j]);
            if (VEC) {
                if (c + 8 <= cols) {
#pragma unroll
                    for (int n = 0; n < (int)sizeof(T) / 2; ++n) reinterpret_cast<uint4 *>(out + c)[n] = reinterpret_cast<const uint4 *>(v)[n];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < cols) out[c + j] = v[j];
                }
                continue;
            }
            __syncwarp();
#pragma unroll
            for (int n = 0; n < (int)sizeof(T) / 2; ++n) reinterpret_cast<uint4 *>(mine + c)[n] = reinterpret_cast<const uint4 *>(v)[n];
            __syncwarp();
            if (sizeof(T) == 2 && reinterpret_cast<uintptr_t>(out) % 4 == 0) {
#pragma unroll
                for (uint32_t j = 0; j < BACK_COLS / 64; ++j) {
                    const uint32_t n = j * 64u + lane * 2u;
                    if (n + 2 <= cols) *reinterpret_cast<uint32_t *>(out + n) = *reinterpret_cast<const uint32_t *>(mine + n);
                    else if (n < cols) out[n] = mine[n];
                }
            } else {
#pragma unroll
                for (uint32_t j = 0; j < BACK_COLS / 32; ++j)
                    if (j * 32u + lane < cols) out[j * 32u + lane] = mine[j * 32u + lane];
            }
        }
    }
}

// ------------------------------------------------ exponent of a tensor ----
// Every CTA raises the result, which starts below any exponent, to that of its own largest magnitude: a maximum of
// integers, the same whatever the order.
constexpr uint32_t TOP_COLS = 2048;
template <typename T>
__global__ __launch_bounds__(THREADS) void qesgd_fp4_tensor_exponent_kernel(const T *x, uint64_t rows, uint64_t cols, uint64_t ldx, bool vec,
                                                                            int32_t *out, uint32_t *status)
{
    __shared__ uint32_t tops[THREADS / 32];
    qesgd_wait_for_previous();
    // a warp takes a row's 2048 columns, 256 at a time
    const uint32_t lane = threadIdx.x % 32u, warp = threadIdx.x / 32u;
    const uint32_t spans = (uint32_t)((cols + TOP_COLS - 1) / TOP_COLS);
    const uint64_t tiles = (uint64_t)spans * ((rows + THREADS / 32 - 1) / (THREADS / 32));
    uint32_t top = 0u;
    bool bad = false;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t r = tile / spans * (THREADS / 32) + warp;
        if (r >= rows) continue;
        const uint64_t first = tile % spans * TOP_COLS;
        const T *const row = x + r * ldx;
#pragma unroll 1
        for (uint32_t i = 0; i < TOP_COLS / 256; i += 4) {
            Octet<T> o[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                const uint64_t c = first + (i + k) * 256u + lane * 8u;
                o[k] = c < cols ? load_octet(row, c, cols, vec) : no_octet<T>();
            }
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                const uint32_t m = top_of(o[k]);
                if (m < 0x7F800000u) {
                    top = max(top, m);
                } else {   // something is not finite: the rest counts
                    float v[8];
                    values(o[k], v);
                    bad = true;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t e = __float_as_uint(v[j]) & 0x7FFFFFFFu;
                        top = max(top, e >= 0x7F800000u ? 0u : e);
                    }
                }
            }
        }
    }
    top = __reduce_max_sync(FULL, top);
    if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < THREADS / 32; ++i) top = max(top, tops[i]);
        // top = 1.f * 2^(E - 127) is at most 2688 * 2^t = 1.3125 * 2^(t + 11) from t = E - 138 on, one later where 1.f > 1.3125
        const int t = (int)(top >> 23) - 138 + ((top & 0x7FFFFFu) > 0x280000u ? 1 : 0);
        atomicMax(out, top == 0u ? -126 : clamp_exponent(t));
    }
    if (bad) atomicOr(status, QESGD_STATUS_NONFINITE);
}

template <typename T, int FORMAT, bool SCALED, bool STOCHASTIC>
cudaError_t launch_quantize(const Fp4QuantizeArgs &a, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    const auto grid_of = [](uint64_t tiles) { return dim3((unsigned)(tiles < 0x7FFFFFFF ? tiles : 0x7FFFFFFF)); };
    if (!a.codes_t) {
        // Tiles of 32 rows where those of 64 would all run at once (four to an SM), so that they spread evenly: 64 x 65536
        // fp32 with draws and back 10.2 us in place of 12.5, 512 x 4096 6.6 in place of 7.0, but 4096 x 4096 28.7 in place of 27.1.
        const uint64_t halves = qesgd_div_up(a.rows, TILE_ROWS) * 2 * qesgd_div_up(a.cols, ROW_COLS);
        plan[0] = QESGD_MATRIX_QUANTIZE_ROWS;
        plan[1] = halves <= 4 * (uint64_t)sm_count ? 32 : 64;
        return plan[1] == 32
                   ? qesgd_launch(qesgd_fp4_quantize_rows_kernel<T, FORMAT, SCALED, STOCHASTIC, 32>, grid_of(2 * halves), dim3(THREADS), stream, a)
                   : qesgd_launch(qesgd_fp4_quantize_rows_kernel<T, FORMAT, SCALED, STOCHASTIC, 64>, grid_of(halves), dim3(THREADS), stream, a);
    }
    plan[0] = QESGD_MATRIX_QUANTIZE_COLUMNS;
    const dim3 grid = grid_of(qesgd_div_up(a.rows, TILE_ROWS) * qesgd_div_up(a.cols, SIDE));
    const auto kernel = qesgd_fp4_quantize_columns_kernel<T, FORMAT, SCALED, STOCHASTIC>;
    const int smem = SIDE * SIDE * (int)sizeof(T);
    static std::atomic<uint64_t> told{0};
    const cudaError_t e = qesgd_prepare(told, (const void *)kernel, smem, false);
    return e != cudaSuccess ? e : qesgd_launch_smem(kernel, grid, dim3(THREADS), smem, stream, a);
}
template <typename T, bool STOCHASTIC>
cudaError_t launch_quantize(const Fp4QuantizeArgs &a, uint32_t format, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    if (format == QESGD_FP4_MX) return launch_quantize<T, QESGD_FP4_MX, false, STOCHASTIC>(a, sm_count, stream, plan);
    return a.tensor_exponent ? launch_quantize<T, QESGD_FP4_NV, true, STOCHASTIC>(a, sm_count, stream, plan) : launch_quantize<T, QESGD_FP4_NV, false, STOCHASTIC>(a, sm_count, stream, plan);
}
template <typename T>
cudaError_t launch_quantize(const Fp4QuantizeArgs &a, uint32_t format, bool stochastic, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    return stochastic ? launch_quantize<T, true>(a, format, sm_count, stream, plan) : launch_quantize<T, false>(a, format, sm_count, stream, plan);
}
template <typename T, int FORMAT>
cudaError_t launch_dequantize(const Fp4DequantizeArgs &a, cudaStream_t stream)
{
    const uint64_t tiles = qesgd_div_up(a.cols, BACK_COLS) * qesgd_div_up(a.rows, BACK_ROWS);
    const dim3 grid((unsigned)(tiles < 0x7FFFFFFF ? tiles : 0x7FFFFFFF));
    return a.vec ? qesgd_launch(qesgd_fp4_dequantize_kernel<T, FORMAT, true>, grid, dim3(THREADS), stream, a)
                 : qesgd_launch(qesgd_fp4_dequantize_kernel<T, FORMAT, false>, grid, dim3(THREADS), stream, a);
}
template <typename T>
cudaError_t launch_dequantize(const Fp4DequantizeArgs &a, uint32_t format, cudaStream_t stream)
{
    return format == QESGD_FP4_MX ? launch_dequantize<T, QESGD_FP4_MX>(a, stream) : launch_dequantize<T, QESGD_FP4_NV>(a, stream);
}
template <typename T>
cudaError_t launch_exponent(const void *x, uint64_t rows, uint64_t cols, uint64_t ldx, bool vec, int32_t *out, uint32_t *status,
                            int sm_count, cudaStream_t stream)
{
    const uint64_t ctas = qesgd_div_up(cols, TOP_COLS) * qesgd_div_up(rows, THREADS / 32), most = (uint64_t)sm_count * 8;
    return qesgd_launch(qesgd_fp4_tensor_exponent_kernel<T>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(THREADS), stream,
                        static_cast<const T *>(x), rows, cols, ldx, vec, out, status);
}

}  // namespace

int qesgd_launch_fp4_quantize(const Fp4QuantizeArgs &a, uint32_t dtype, uint32_t format, bool stochastic, int sm_count, cudaStream_t stream, uint32_t *plan)
{
    switch (dtype) {
        case QESGD_F32: return (int)launch_quantize<float>(a, format, stochastic, sm_count, stream, plan);
        case QESGD_BF16: return (int)launch_quantize<__nv_bfloat16>(a, format, stochastic, sm_count, stream, plan);
        default: return (int)launch_quantize<__half>(a, format, stochastic, sm_count, stream, plan);
    }
}
int qesgd_launch_fp4_dequantize(const Fp4DequantizeArgs &a, uint32_t dtype, uint32_t format, cudaStream_t stream)
{
    switch (dtype) {
        case QESGD_F32: return (int)launch_dequantize<float>(a, format, stream);
        case QESGD_BF16: return (int)launch_dequantize<__nv_bfloat16>(a, format, stream);
        default: return (int)launch_dequantize<__half>(a, format, stream);
    }
}
int qesgd_launch_fp4_tensor_exponent(const void *x, uint32_t dtype, uint64_t rows, uint64_t cols, uint64_t ldx, bool vec,
                                     int32_t *out, uint32_t *status, int sm_count, cudaStream_t stream)
{
    const cudaError_t e = cudaMemsetAsync(out, 0x80, sizeof(int32_t), stream);   // below every exponent
    if (e != cudaSuccess) return (int)e;
    switch (dtype) {
        case QESGD_F32: return (int)launch_exponent<float>(x, rows, cols, ldx, vec, out, status, sm_count, stream);
        case QESGD_BF16: return (int)launch_exponent<__nv_bfloat16>(x, rows, cols, ldx, vec, out, status, sm_count, stream);
        default: return (int)launch_exponent<__half>(x, rows, cols, ldx, vec, out, status, sm_count, stream);
    }
}
