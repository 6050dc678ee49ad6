// The 8-bit form of an activation (convbn_pack): consecutive groups of 32 elements, a signed code per element, a byte per group
// that names the group's step 2^(byte - 127).  An element stands for code * step, which is exact in all three storage types.
#pragma once

#include "common.cuh"

namespace convbn {

constexpr int kPackGroup = 32;
constexpr uint32_t kPackBad = 255;       // a group with an infinity or a NaN

__device__ __forceinline__ float pack_step(uint32_t byte) {      // NaN for a group that held no number
    return byte == kPackBad ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}
// Codes 0 .. 3 of a word as floats: a byte b + 128 in the low mantissa bits of 2^23 is 2^23 + 128 + b.
__device__ __forceinline__ void codes_to_f32(uint32_t word, float (&f)[4]) {
    const uint32_t u = word ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540u + (uint32_t)i)) - 8388736.f;
}

}  // namespace convbn
