// What the kernels of the deployed 8-bit product share: rows to codes, sums to results.
#pragma once

#include "common.cuh"
#include "mma_sync.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

// Largest magnitudes below this count as zero: 127 / a would not be finite.
constexpr float kQuantTiny = 7.8886091e-31f;      // 2^-100

// The factor is 127 times the rounded reciprocal (two roundings, and part of the definition: x times it may lie on a half), the
// scale a times the rounded 1 / 127.
struct RowScale { float inv, scale; };            // 127 / a, a / 127
__device__ __forceinline__ RowScale row_scale(uint32_t top) {      // bits of the largest magnitude as fp32
    const float a = __uint_as_float(top);
    if (top >= 0x7F800000u) return {0.f, __uint_as_float(0x7FC00000u)};     // (codes 0, scale NaN: so is every result)
    if (a < kQuantTiny) return {0.f, 0.f};
    return {__fmul_rn(__frcp_rn(a), 127.f), __fmul_rn(a, 1.f / 127.f)};
}
// 1.5 2^23 + code: the code is the low byte; the product is exact inside the fma.  No clamp: |x inv| is at most 127 (1 + 2^-23), and
// 127 (1 + 2^-21) for maxima above 2^126, whose reciprocals are subnormal (they must not be flushed) and have 21 bits or more; from 127.5
// on it would be 128.
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
    // from shared memory; the second 16 bytes of fp32 lie in the neighbouring chunk of a swizzled row
    __device__ __forceinline__ void load_shared(uint32_t at) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at ^ (uint32_t)(4 * i)) : "memory");
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
    // The same in steps: of these eight (16-bit types: of the even and the odd ones), of two such, as top() has it.
    __device__ __forceinline__ uint32_t part() const {
        uint32_t m = sizeof(T) == 2 ? w[0] : w[0] & 0x7FFFFFFFu;
#pragma unroll
        for (int i = 1; i < kWords; ++i) m = sizeof(T) == 2 ? larger(m, w[i]) : max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
    static __device__ __forceinline__ uint32_t of_two(uint32_t a, uint32_t b) { return sizeof(T) == 2 ? larger(a, b) : max(a, b); }
    static __device__ __forceinline__ uint32_t whole(uint32_t m) { return sizeof(T) == 2 ? merge(m) : m; }
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

RowMap quant_row_map(const Problem &pb);      // (quant_fused.cu)

// mbar_wait_bounded whose attempts may last up to 4 us each: a waiting warp leaves the issue slots to those that convert.
template <class Bar>
__device__ __forceinline__ bool mbar_wait_parked(Bar bar, uint32_t parity, volatile int *abort_flag, uint64_t limit_ns = 2000000000ull) {
    auto attempt = [&]() {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(ptx::smem_u32(bar)), "r"(parity), "r"(4000u) : "memory");
        return ok != 0;
    };
    if (attempt()) return true;
    const uint64_t t0 = ptx::globaltimer_ns();
    while (true) {
        if (attempt()) return true;
        if (abort_flag && *abort_flag) return false;
        if (ptx::globaltimer_ns() - t0 > limit_ns) return false;
    }
}

// ---- tensor-core product of codes ---------------------------------------------------------------------------------------
// tcgen05.mma instruction descriptor of kind::i8: bits 4-5 D format (2 = s32), 7-9 and 10-12 operand formats (1 = s8), 17-22 N >> 3,
// 24-28 M >> 4.
__host__ __device__ constexpr uint32_t idesc_s8(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CTAS = 1>
__device__ __forceinline__ void umma_s8(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::%7.kind::i8 [%0], da, db, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "n"(CTAS)
        : "memory");
}

// What an epilogue warp does with 32 rows and 128 bytes of columns of Z: sums times the row's and the channel's scale, shift,
// addend, ReLU, into its box (which holds the addend's) or, where rows of Z do not start on 16-byte boundaries, straight into Z.
template <class T>
struct QuantOut {
    T *z;
    const T *add;
    uint32_t p;
    int n, dense, relu;        // dense: boxes
};
// xs2: scales of rows lane / 4 + 8 k (16-bit boxes), otherwise of row `lane`.  SMALL: |sums| below 2^22: added to the bits of 1.5 2^23
// they are its low bits, and the conversion unit, a quarter as fast, is left alone.
template <class T, bool SMALL>
__device__ __forceinline__ void quant_chunk(const QuantOut<T> &o, uint8_t *buf, bool boxed, uint32_t t_row, const float *ws_c, const float *b_c,
                                            const f32x2 (&xs2)[4], uint32_t row, int col0, int cols, int lane) {
    constexpr int CH = 128 / sizeof(T), PER = 16 / sizeof(T);
    const f32x2 one = pair(1.f, 1.f), away = pair(-12582912.f, -12582912.f), none = pair(-0.f, -0.f);
    auto scaled = [&](uint32_t a, uint32_t b, f32x2 xs) {
        if constexpr (SMALL)
            return fma2(fma2(pair(__uint_as_float(a + 0x4B400000u), __uint_as_float(b + 0x4B400000u)), one, away), xs, none);
        else
            return fma2(pair((float)(int)a, (float)(int)b), xs, none);
    };
    if constexpr (sizeof(T) == 2) {
        if (o.dense) {
            // the accumulator as matrix fragments: see umma_conv.cu
            constexpr bool H = __is_same(T, __half);
            const uint32_t ws_at = ptx::smem_u32(ws_c) + (uint32_t)(lane & 3) * 8u, b_at = ptx::smem_u32(b_c) + (uint32_t)(lane & 3) * 8u;
            const uint32_t frag = ptx::smem_u32(buf) + (uint32_t)((lane & 7) + (lane & 8)) * 128u;
            const uint32_t frag_chunk = (uint32_t)(((lane >> 4) ^ (lane & 7)) << 4);
            auto rows16 = [&](auto add_tag, auto relu_tag) {
                constexpr bool ADD = decltype(add_tag)::value, RELU = decltype(relu_tag)::value;
#pragma unroll
                for (int c = 0; c < 64; c += 32) {     // 32 columns of all rows at a time: their parameters are read once
                    uint32_t v[2][16];
                    ptx::tmem_ld_16x32(t_row + (uint32_t)c, v[0]);
                    ptx::tmem_ld_16x32(t_row + (16u << 16) + (uint32_t)c, v[1]);
                    f32x2 sc[4], sh[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        sc[q] = lds_f32x2(ws_at + (uint32_t)(c + 8 * q) * 4u);
                        sh[q] = lds_f32x2(b_at + (uint32_t)(c + 8 * q) * 4u);
                    }
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 4; q += 2)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t r[4], a[4];       // columns c + 8 q and the next 8: rows 0-7, 8-15 of each
                            const uint32_t at16 = (uint32_t)h * 2048u + (((uint32_t)(c / 8 + q) << 4) ^ frag_chunk);
                            if constexpr (ADD) ldmatrix_x4(a[0], a[1], a[2], a[3], frag + at16);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t *s = &v[h][(q + (e >> 1)) * 4 + (e & 1) * 2];
                                f32x2 f = fma2(scaled(s[0], s[1], xs2[2 * h + (e & 1)]), sc[q + (e >> 1)], sh[q + (e >> 1)]);
                                if constexpr (ADD) f = fma2(f, one, widen_t<H>(a[e]));
                                r[e] = narrow_t<H>(f);
                                if constexpr (RELU) r[e] = post_pair<H>(r[e], false, 0u, true, false, 0u);
                            }
                            stmatrix_x4(frag + at16, r[0], r[1], r[2], r[3]);
                        }
                }
            };
            if (boxed) { if (o.relu) rows16(std::true_type(), std::true_type()); else rows16(std::true_type(), std::false_type()); }
            else { if (o.relu) rows16(std::false_type(), std::true_type()); else rows16(std::false_type(), std::false_type()); }
            return;
        }
    }
#pragma unroll 1
    for (int h = 0; h < CH; h += 32) {
        uint32_t v[32];
        ptx::tmem_ld_32x32(t_row + (uint32_t)h, v);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const f32x2 f = fma2(scaled(v[j], v[j + 1], xs2[0]), *(const f32x2 *)(ws_c + h + j), *(const f32x2 *)(b_c + h + j));
            v[j] = (uint32_t)f;
            v[j + 1] = (uint32_t)(f >> 32);
        }
        if (sizeof(T) == 4 && o.dense) {
#pragma unroll
            for (int j = 0; j < 32; j += PER) {
                uint4 *at = (uint4 *)(buf + lane * 128 + ((((j / PER) ^ lane) & 7) << 4));
                uint4 q = boxed ? *at : make_uint4(0u, 0u, 0u, 0u);
                uint32_t *w = (uint32_t *)&q;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f = __uint_as_float(v[j + e]);
                    if (boxed) f += __uint_as_float(w[e]);
                    w[e] = __float_as_uint(o.relu ? fmaxf(f, 0.f) : f);
                }
                *at = q;
            }
        } else if (row < o.p) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                if (h + j >= cols) continue;
                const size_t at = (size_t)row * o.n + col0 + h + j;
                float f = __uint_as_float(v[j]);
                if (o.add) f += to_f32(o.add[at]);
                o.z[at] = from_f32<T>(o.relu ? fmaxf(f, 0.f) : f);
            }
        }
    }
}

}  // namespace convbn
