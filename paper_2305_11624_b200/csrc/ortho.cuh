// Orthogonal updates by Newton-Schulz products: how matrices lie in the workspace and what a launch is told of them.
//
//     X = G / (|G| + eps)        steps times:  A = X X^T,  X <- a X + (b A + c A A) X
//
// (a matrix with more rows than columns: A = X^T X and X <- a X + X (b A + c A A), without a transposed copy).  A has the shorter side m.
//
// Numbers are pairs of halves, hi + lo with lo = fl(v - hi): 22 significant bits, so that a product of matrices is three tensor-core
// products, hi hi + hi lo + lo hi, and what is left out is 2^-22 of it.  One bf16 or half product (2^-9, 2^-11) is not enough: the five
// steps lift a small singular value by up to 3.4445^5 = 485, and with it the rounding of X beside large ones.  Stored values are 2^10 times
// the numbers (singular values stay below 1.21, so nothing passes 2^14, and lo is a normal half for numbers down to 2^-13).
//
// A matrix lies in tiles of 128 rows x 64 columns, 16 KB, in the very form that the MMAs read from shared memory (128-byte swizzle): a
// tile is brought by a copy of consecutive bytes, without a tensor map.  Read along its rows it is a K-major operand of 64 k; half a tile,
// read down its rows, is an MN-major one of 64 k x 64.  Of A and its like, which are symmetric, tiles of the lower half exist; the upper half is
// read from the lower one in the other form.
#pragma once

#include "kernels.h"

namespace convbn {

constexpr uint32_t kOrthoTile = 16384;
constexpr float kOrthoScale = 1024.f;
constexpr float kOrthoCoefA = 3.4445f, kOrthoCoefB = -4.7750f, kOrthoCoefC = 2.0315f;

// Offset of the 16-byte chunk of 8 columns `chunk` of row `row` in a tile.
__host__ __device__ __forceinline__ uint32_t ortho_chunk(uint32_t row, uint32_t chunk) { return row * 128u + ((chunk ^ (row & 7u)) << 4); }

// 2^10 / (|G| + eps) as a power of two, in two factors, and a fraction of 48 bits: a product in 64 bits is two conversions an element, of
// which an SM does sixteen a clock (a quarter of the time of putting a matrix into tiles).
struct OrthoScaling {
    float two_a, two_b, hi, lo;
    // (a zero matrix has no quotient where eps is none either: zeros stay zeros; a sum that is no number passes through)
    __device__ __forceinline__ static OrthoScaling of(double squares, double eps) {
        if (squares == 0.) return {1.f, 1.f, 0.f, 0.f};
        int power;
        const double part = frexp((double)kOrthoScale / (sqrt(squares) + eps), &power);
        OrthoScaling s;
        s.two_a = ldexpf(1.f, power / 2);
        s.two_b = ldexpf(1.f, power - power / 2);
        s.hi = (float)part;
        s.lo = (float)(part - (double)s.hi);
        return s;
    }
    __device__ __forceinline__ float operator()(float g) const {
        const float u = g * two_a * two_b;
        return fmaf(u, hi, u * lo);
    }
};

// The products.  All steps of X at a time, direct:
//     A = X X^T        R = b A + c A A        X <- a X + R X
// or, where X is long, on m x m matrices, all polynomials of one A, which commute and are symmetric: k steps are X <- Q X with
//     A = X X^T;   k times:  R = b A + c A A;   Q <- (a + R) Q  (from 1);   B = (a + R) A;   A <- (a + R) B        then X <- Q X
// For k = 3 and 2 five steps are 6 m^2 n + 14 m^3 operations (symmetric products half) where the direct ones are 15 m^2 n + 5 m^3, and two
// sums over all of X's columns where they are five.  The price is precision: A's rounding, which belongs to all singular values alike, grows
// by 3.4445^2 a step for the small ones.  After three steps X is formed and A from it anew; so the results are as near to the formula as fp32
// products bring them (with stages of 2 and 3 steps it is twice to four times as far, with one of five ten times).
enum {
    kOrthoGram = 0,                // A = X X^T
    kOrthoSquare = 1,              // R = b A + c A A
    kOrthoSquareQ = 2,             // the same, and Q = a + R
    kOrthoB = 3,                   // B = a A + R A
    kOrthoBQ = 4,                  // the same, and Q' = a Q + R Q
    kOrthoA = 5,                   // A = a B + R B
    kOrthoQ = 6,                   // Q' = a Q + R Q
    kOrthoUpdate = 7,              // X' = a X + R X
    kOrthoUpdateQ = 8,             // X' = Q X
    kOrthoOpMask = 15, kOrthoX = 16, kOrthoQSource = 32, kOrthoLast = 64       // X, Q in their second places; the last product
};
constexpr float kOrthoQScale = 256.f;             // Q's numbers are up to 3.4445^3

}  // namespace convbn
