// The 8-bit form of an activation (convbn_pack): consecutive groups of 32 elements, a signed code per element, a byte per group
// that names the group's step 2^(byte - 127).  An element stands for code * step, which is exact in all three storage types.
#pragma once

#include "common.cuh"
#include "packed_f32.cuh"

namespace convbn {

constexpr int kPackGroup = 32;
constexpr uint32_t kPackBad = 255;       // a group with an infinity or a NaN

__device__ __forceinline__ float pack_step(uint32_t byte) {      // NaN for a group that held no number
    return byte == kPackBad ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}
// Codes 0 .. 3 of a word times their step (in both halves): a byte q + 128 in the low mantissa bits of 2^23 is 2^23 + 128 + q.  (One
// fused multiply-add per value instead of a sum and a product would want (2^23 + 128) step finite, which it is not for the largest
// steps; with a branch for those it was slower, 3x3 64 -> 64 at 56 x 56, N = 32 43.9 -> 48.3 us.)
__device__ __forceinline__ void restore4(uint32_t word, f32x2 step, f32x2 (&f)[2]) {
    const uint32_t u = word ^ 0x80808080u;
    const f32x2 a = pair(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540u)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7541u)));
    const f32x2 b = pair(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7542u)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7543u)));
    const f32x2 one = pair(1.f, 1.f), off = pair(-8388736.f, -8388736.f), none = pair(-0.f, -0.f);
    f[0] = fma2(fma2(a, one, off), step, none);
    f[1] = fma2(fma2(b, one, off), step, none);
}

}  // namespace convbn
