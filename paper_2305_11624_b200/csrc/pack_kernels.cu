// Activations in 8 bits between forward and backward (convbn_pack, convbn_unpack).
//
// Group of 32 consecutive elements, a = max |x|:  e = the smallest integer with rne(a 2^-e) <= 127, within the storage type's
// bounds;  q = rne(x 2^-e), and the sign of x where that is 0 but x is not, so that the codes keep the decisions of a ReLU
// exactly (x > 0 <=> q > 0).  q 2^e has at most 7 significant bits: restoring it rounds nothing, and neither does a product of it
// with another stored tensor that is accumulated in fp32.  A power of two costs up to one bit of the step against a / 127; with it
// the weight gradient's operand is exact in the storage type.
// Bounds of e: -126 to 121 for bf16 and fp32 (127 * 2^121 is finite), -24 to 9 for half (2^-24 is its smallest number).
//
// Both kernels are one pass over memory: a thread takes 16 elements (32 or 64 bytes) and one 16-byte store of codes, two
// neighbouring lanes share a group.
#include "kernels.h"
#include "pack8.cuh"

namespace convbn {

namespace {

constexpr int kPer = 16;                 // elements of a thread and turn: half a group

template <class T> struct PackBounds { static constexpr int lo = -126, hi = 121; };
template <> struct PackBounds<__half> { static constexpr int lo = -24, hi = 9; };

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <class T>
__device__ __forceinline__ void load16(const T *p, float (&f)[kPer]) {
    constexpr int W = kPer * sizeof(T) / 16;
    uint4 q[W];
#pragma unroll
    for (int i = 0; i < W; ++i) q[i] = __ldg((const uint4 *)p + i);
    const uint32_t *w = (const uint32_t *)q;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < kPer / 2; ++i) unpack2_t<!__is_same(T, __nv_bfloat16)>(w[i], f[2 * i], f[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) f[i] = __uint_as_float(w[i]);
    }
}

// (A chunk a thread and no loop: 1.25 GB there and back 220 us; in a loop of 16 blocks per SM 237, two chunks requested at once 230.)
template <class T>
__global__ void __launch_bounds__(256) pack_kernel(const T *__restrict__ x, uint8_t *__restrict__ codes, uint8_t *__restrict__ steps,
                                                   long long count) {
    pdl_wait();
    pdl_launch_dependents();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, at = i * kPer;
    const bool whole = at + kPer <= count;
    float f[kPer];
    if (whole) load16(x + at, f);
    else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) f[k] = at + k < count ? to_f32(x[at + k]) : 0.f;
    }
    float a = fabsf(f[0]);
#pragma unroll
    for (int k = 1; k < kPer; ++k) a = max_nan(a, fabsf(f[k]));
    a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, 1));
    const uint32_t bits = __float_as_uint(a);
    const bool bad = bits >= 0x7F800000u;
    // (the carry of 0x10000 into the exponent: from 127.5 2^(k - 6) on, which would round to 128)
    int e = (int)((bits + 0x10000u) >> 23) - 133;
    e = max(PackBounds<T>::lo, min(PackBounds<T>::hi, e));
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[kPer / 4];
#pragma unroll
    for (int k = 0; k < kPer; k += 4) {
        uint32_t t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = f[k + j], m = fminf(fmaxf(fabsf(v) * inv, 1.f), 127.f);
            // 1.5 2^23 + q: the code is the low byte
            t[j] = __float_as_uint((v == 0.f ? 0.f : copysignf(m, v)) + 12582912.f);
        }
        w[k / 4] = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
        if (bad) w[k / 4] = 0u;
    }
    if (whole) *(uint4 *)(codes + at) = make_uint4(w[0], w[1], w[2], w[3]);
    else {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (at + k < count) codes[at + k] = (uint8_t)(w[k / 4] >> (8 * (k & 3)));
    }
    if ((i & 1) == 0 && at < count) steps[i >> 1] = (uint8_t)(bad ? kPackBad : (uint32_t)(e + 127));
}

template <class T>
__global__ void __launch_bounds__(256) unpack_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ steps,
                                                     T *__restrict__ out, long long count) {
    pdl_wait();
    pdl_launch_dependents();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, at = i * kPer;
    if (at >= count) return;
    const float step = pack_step(__ldg(steps + (i >> 1)));
    if (at + kPer <= count) {
        const f32x2 by = pair(step, step);
        const uint4 q = __ldg((const uint4 *)(codes + at));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        uint4 o[kPer * sizeof(T) / 16];
        uint32_t *r = (uint32_t *)o;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f32x2 f[2];
            restore4(w[k], by, f);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if constexpr (sizeof(T) == 2) r[2 * k + j] = narrow_t<!__is_same(T, __nv_bfloat16)>(f[j]);
                else { r[4 * k + 2 * j] = (uint32_t)f[j]; r[4 * k + 2 * j + 1] = (uint32_t)(f[j] >> 32); }
            }
        }
#pragma unroll
        for (int k = 0; k < (int)(kPer * sizeof(T) / 16); ++k) ((uint4 *)(out + at))[k] = o[k];
    } else {
        for (int k = 0; at + k < count; ++k) out[at + k] = from_f32<T>((float)(int8_t)codes[at + k] * step);
    }
}

unsigned pack_blocks(long long count) { return (unsigned)((count + 256 * kPer - 1) / (256 * kPer)); }

}  // namespace

cudaError_t launch_pack(int dtype, const void *x, void *codes, void *steps, long long count, cudaStream_t st) {
    auto go = [&](auto tag) {
        using T = decltype(tag);
        return launch_pdl(pack_kernel<T>, dim3(pack_blocks(count)), dim3(256), 0, st, (const T *)x, (uint8_t *)codes, (uint8_t *)steps, count);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

cudaError_t launch_unpack(int dtype, const void *codes, const void *steps, void *out, long long count, cudaStream_t st) {
    auto go = [&](auto tag) {
        using T = decltype(tag);
        return launch_pdl(unpack_kernel<T>, dim3(pack_blocks(count)), dim3(256), 0, st, (const uint8_t *)codes, (const uint8_t *)steps,
                          (T *)out, count);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

}  // namespace convbn
