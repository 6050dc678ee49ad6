// What the kernels of the deployed 8-bit product share: rows to codes, sums to results.
#pragma once

#include "common.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

// Largest magnitudes below this count as zero: 127 / a would not be finite.
constexpr float kQuantTiny = 7.8886091e-31f;      // 2^-100

struct RowScale { float inv, scale; };            // 127 / a, a / 127
__device__ __forceinline__ RowScale row_scale(uint32_t top) {      // bits of the largest magnitude as fp32
    const float a = __uint_as_float(top);
    if (top >= 0x7F800000u) return {0.f, __uint_as_float(0x7FC00000u)};     // (codes 0, scale NaN: so is every result)
    if (a < kQuantTiny) return {0.f, 0.f};
    return {__fdiv_rn(127.f, a), __fdiv_rn(a, 127.f)};
}
// 1.5 2^23 + code: the code is the low byte.  |x inv| <= 127 (1 + 2^-24), so no clamp; the product is exact inside the fma.
__device__ __forceinline__ uint32_t code_bits(float x, float inv) { return __float_as_uint(fmaf(x, inv, 12582912.f)); }
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// Eight elements of a row as loaded, and what is asked of them.
template <class T>
struct Eight {
    static constexpr int kWords = 8 * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void load(const T *p) {            // 16-byte aligned
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            const uint4 q = __ldg((const uint4 *)p + i);
            w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
        }
    }
    __device__ __forceinline__ void load_shared(uint32_t at) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at + 4u * i) : "memory");
    }
    __device__ __forceinline__ void load_some(const T *p, int count) {      // any alignment, the rest zero
        zero();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= count) break;
            if constexpr (sizeof(T) == 2) w[i / 2] |= (uint32_t)__ldg((const unsigned short *)p + i) << (16 * (i & 1));
            else w[i] = __ldg((const unsigned int *)p + i);
        }
    }
    // Largest magnitude as bits (16-bit types: the same in both halves); a NaN stays, and lies above every number.
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (sizeof(T) == 2) {
            uint32_t m = w[0];
#pragma unroll
            for (int i = 1; i < kWords; ++i) m = larger(m, w[i]);
            return merge(m);
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kWords; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
            return m;
        }
    }
    // of the larger magnitudes of two words' halves (16-bit types; the signs are any)
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        if constexpr (__is_same(T, __half)) asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t merge(uint32_t m) {
        return larger(m, __byte_perm(m, m, 0x1032)) & 0x7FFF7FFFu;
    }
    // of a largest magnitude as bits, that number's bits as fp32
    static __device__ __forceinline__ uint32_t top_f32(uint32_t m) {
        if constexpr (sizeof(T) == 4) return m;
        else if constexpr (__is_same(T, __half)) return __float_as_uint(unpack_h16((uint16_t)m, 1));
        else return m & 0xFFFF0000u;
    }
    // (inv = 0: codes 0, but of an infinity or a NaN, whose row's scale is NaN)
    __device__ __forceinline__ uint2 codes(float inv) const {
        const f32x2 by = pair(inv, inv), magic = pair(12582912.f, 12582912.f);
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            f32x2 v;
            if constexpr (sizeof(T) == 2) v = widen_t<__is_same(T, __half)>(w[i / 2]);
            else v = pair(__uint_as_float(w[i]), __uint_as_float(w[i + 1]));
            v = fma2(v, by, magic);
            t[i] = (uint32_t)v;
            t[i + 1] = (uint32_t)(v >> 32);
        }
        return make_uint2(pack_bytes(t[0], t[1], t[2], t[3]), pack_bytes(t[4], t[5], t[6], t[7]));
    }
};

// Input row (output pixel p): its channels lie side by side.
struct RowMap {
    long long step;            // elements from one row to the next, where every pixel is read
    int strided;
    long long pixel, line, image;      // strided: elements from an output pixel to the next of its row, to the next row, image
    FastDiv by_w, by_h;
    __device__ __forceinline__ long long at(uint32_t p) const {
        if (!strided) return (long long)p * step;
        const uint32_t t = by_w.div(p), img = by_h.div(t);
        return (long long)img * image + (long long)(t - img * by_h.d) * line + (long long)(p - t * by_w.d) * pixel;
    }
};

}  // namespace convbn
