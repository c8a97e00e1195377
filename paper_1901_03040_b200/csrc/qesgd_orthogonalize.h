// Workspace of qesgd_orthogonalize, and the scales at which its intermediates are kept.
#pragma once

#include <cuda_fp16.h>

#include "qesgd_internal.h"

// X, A = X X^T and B = b A + c A A are kept in fp16, times powers of two.  With X = G / ||G||_F elements of an n x n matrix
// start near 1 / n and end near 1 / sqrt(n), those of A near n^-1.5: unscaled they would fall below fp16's normal
// numbers (6e-5) from n = 128 on.  In magnitude X may reach 255, A 15, B 63.
constexpr float ORTHO_X_SCALE = 256.0f, ORTHO_A_SCALE = 4096.0f, ORTHO_B_SCALE = 1024.0f;
// What rounding X to fp16 leaves behind is kept beside X, in fp16 too, for the term a X of every step: the rounding errors of
// strong directions are as large as weak ones and grow with them.  512 x 512, 16 directions over 10^-4 of them, five steps:
// 4.4e-2 off without (before the result's rounding), 1.1e-2 with it in two steps, 2.7e-3 in three, 1.2e-3 in four, 8.5e-4 in all.
// Where singular values lie far apart, B X takes both terms of X in the first steps.  What rounding X to one term leaves
// behind are new directions, as large as weak ones: |b s^2 + c s^4| = 2.8 times them enters X', and each later step enlarges
// it by 3.4.  (B's own rounding only mixes the rows that X has: a second term of B changes nothing.)  Five steps, worst of 1 to
// 64 strong directions 10 to 10^5 times the rest, before the result's rounding: 8 x 8 4e-2 off with one term, 8e-3 with two
// in the first step, 3e-3 in two steps, 1e-3 in three; 64 x 1000 8e-3, 4e-3, 3e-3, 1e-3; 128 x 128 4e-3, 2e-3, 2e-3, 1e-3.
// Both terms in all steps gain nothing on three.
constexpr uint32_t ORTHO_TERMS_STEPS = 3;
// Products of their own (more than 128 rows) take one term where the smaller side has at least this many: the errors fall
// with its square root, 4e-3 at 129, 3e-3 at 256, 1.9e-3 at 512, 1.4e-3 at 1024, against 1e-3 to 1.3e-3 with both terms, and a second
// term doubles an update's contraction.
constexpr uint32_t ORTHO_TERMS_SIDE = 512;

struct OrthoView {
    __half *hi, *lo;
    uint64_t ld, x_stride;
};

// m = the smaller side, n = the larger: X is m x n whichever way the matrix lies.
struct OrthoLayout {
    uint64_t m, n, ld_x, ld_a, x_stride, a_stride;   // elements
    uint32_t parts;                                  // partial sums of a matrix's norm
    uint64_t d_stride;                               // floats: a diagonal, up to whole tiles
    uint64_t off_hi[2], off_lo[2], off_a, off_b, off_d, bytes;
};
inline OrthoLayout qesgd_ortho_layout(uint64_t rows, uint64_t cols, uint64_t batch)
{
    OrthoLayout l;
    l.m = rows < cols ? rows : cols;
    l.n = rows < cols ? cols : rows;
    l.ld_x = (l.n + 7) / 8 * 8;      // rows begin on 16 bytes
    l.ld_a = (l.m + 7) / 8 * 8;
    l.x_stride = (l.m * l.ld_x + 63) / 64 * 64;
    l.a_stride = (l.m * l.ld_a + 63) / 64 * 64;
    const uint64_t parts = qesgd_div_up(l.m * l.n, 4096);
    // as many CTAs as run at once: norm and start of 12 x 512 x 2048 took 28 us with three times as many, and 22 so
    const uint64_t most = batch < 64 ? 1024 / batch : 16;
    l.parts = (uint32_t)(parts < most ? parts : most);
    uint64_t at = (batch * l.parts * sizeof(double) + 255) / 256 * 256;
    const uint64_t x = (batch * l.x_stride * 2 + 255) / 256 * 256, a = (batch * l.a_stride * 2 + 255) / 256 * 256;
    for (int i = 0; i < 2; ++i) {
        l.off_hi[i] = at;
        l.off_lo[i] = at + x;
        at += 2 * x;
    }
    l.off_a = at;
    l.off_b = at + a;
    l.d_stride = (l.m + 255) / 256 * 256;
    l.off_d = at + 2 * a;
    l.bytes = l.off_d + 2 * batch * l.d_stride * sizeof(float);
    return l;
}
