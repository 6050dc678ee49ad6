// Orthogonal updates by Newton-Schulz products: how matrices lie in the workspace and what a launch is told of them.
//
//     X = G / (|G| + eps)        steps times:  A = X X^T,  P = b A + c A A,  X <- a X + P X
//
// (a matrix with more rows than columns: A = X^T X and X <- a X + X P, without a transposed copy).  A and P have the shorter side m.
//
// Numbers are pairs of halves, hi + lo with lo = fl(v - hi): 22 significant bits, so that a product of matrices is three tensor-core
// products, hi hi + hi lo + lo hi, and what is left out is 2^-22 of it.  One bf16 or half product (2^-9, 2^-11) is not enough: the five
// steps lift a small singular value by up to 3.4445^5 = 485, and with it the rounding of X beside large ones.  Stored values are 2^10 times
// the numbers (singular values stay below 1.21, so nothing passes 2^14, and lo is a normal half for numbers down to 2^-13).
//
// A matrix lies in tiles of 128 rows x 64 columns, 16 KB, in the very form that the MMAs read from shared memory (128-byte swizzle): a
// tile is brought by a copy of consecutive bytes, without a tensor map.  Read along its rows it is a K-major operand of 64 k; half a tile,
// read down its rows, is an MN-major one of 64 k x 64.  Of A and P, which are symmetric, tiles of the lower half exist; the upper half is
// read from the lower one in the other form.
#pragma once

#include "kernels.h"

namespace convbn {

constexpr uint32_t kOrthoTile = 16384;
constexpr float kOrthoScale = 1024.f;
constexpr float kOrthoA = 3.4445f, kOrthoB = -4.7750f, kOrthoC = 2.0315f;
constexpr int kOrthoChunk = 16384;                // elements that a block sums the squares of

// Offset of the 16-byte chunk of 8 columns `chunk` of row `row` in a tile.
__host__ __device__ __forceinline__ uint32_t ortho_chunk(uint32_t row, uint32_t chunk) { return row * 128u + ((chunk ^ (row & 7u)) << 4); }

enum { kOrthoGram = 0, kOrthoSquare = 1, kOrthoUpdate = 2 };

}  // namespace convbn
