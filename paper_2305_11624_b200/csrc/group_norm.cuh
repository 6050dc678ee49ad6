// Group norm with an activation, channels last: what its kernels share.
//
//     mean, var over the M = H W C/G values of a group of a sample      r = 1 / sqrt(var + eps)
//     y = gamma (x - mean) r + beta        z = act(y)
//     dy = dz act'(y)     dbeta = sum dy     dgamma = sum dy xhat     dx = r (gamma dy - E[gamma dy] - xhat E[gamma dy xhat])
//
// Arithmetic is fp32, two values an instruction.  The kernels are bound by memory only as long as an element takes some twenty
// instructions: with single fp32 operations the same passes took 18 (forward) and 40 (backward) and half the time again.
#pragma once

#include "kernels.h"
#include "packed_f32.cuh"

namespace convbn {

__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float2 split2(f32x2 p) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }

// V elements of T, moved as one access of V sizeof(T) bytes; as (V + 1) / 2 pairs (V = 1: the second of the pair is zero).
template <class T, int V>
struct NormVec {
    static constexpr int kBytes = V * (int)sizeof(T), kPairs = (V + 1) / 2;
    static constexpr bool kHalf = std::is_same<T, __half>::value;
    using Word = typename std::conditional<kBytes == 16, uint4, typename std::conditional<kBytes == 8, uint2,
                 typename std::conditional<kBytes == 4, uint32_t, uint16_t>::type>::type>::type;
    Word w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const Word *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<Word *>(p) = w; }
    // the same for data that nothing reads again
    __device__ __forceinline__ void store_last(T *p) const {
        if constexpr (kBytes == 2) __stcs(reinterpret_cast<unsigned short *>(p), w);
        else __stcs(reinterpret_cast<Word *>(p), w);
    }
    __device__ __forceinline__ f32x2 get(int i) const {
        if constexpr (sizeof(T) == 4) {
            const float *f = reinterpret_cast<const float *>(&w);
            if constexpr (V == 1) return pair(f[0], 0.f);
            else return pair(f[2 * i], f[2 * i + 1]);
        } else if constexpr (V == 1) {
            return widen_t<kHalf>((uint32_t)w);
        } else {
            return widen_t<kHalf>(reinterpret_cast<const uint32_t *>(&w)[i]);
        }
    }
    __device__ __forceinline__ void put(int i, f32x2 v) {
        if constexpr (sizeof(T) == 4) {
            float *f = reinterpret_cast<float *>(&w);
            const float2 s = split2(v);
            f[2 * i] = s.x;
            if constexpr (V > 1) f[2 * i + 1] = s.y;
        } else if constexpr (V == 1) {
            w = (uint16_t)narrow_t<kHalf>(v);
        } else {
            reinterpret_cast<uint32_t *>(&w)[i] = narrow_t<kHalf>(v);
        }
    }
    // max(., 0); not-a-number becomes 0
    __device__ __forceinline__ void relu() {
        if constexpr (sizeof(T) == 4) {
            float *f = reinterpret_cast<float *>(&w);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = fmaxf(f[i], 0.f);
        } else if constexpr (V == 1) {
            w = (uint16_t)post_pair<kHalf>(w, false, 0u, true, false, 0u);
        } else {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                uint32_t &u = reinterpret_cast<uint32_t *>(&w)[i];
                u = post_pair<kHalf>(u, false, 0u, true, false, 0u);
            }
        }
    }
    // pair i zero where y is negative (y is no zero and a number)
    __device__ __forceinline__ void keep_positive(int i, f32x2 y) {
        const float2 s = split2(y);
        if constexpr (sizeof(T) == 4) {
            uint32_t *u = reinterpret_cast<uint32_t *>(&w);
            u[2 * i] &= ~(uint32_t)((int)__float_as_uint(s.x) >> 31);
            if constexpr (V > 1) u[2 * i + 1] &= ~(uint32_t)((int)__float_as_uint(s.y) >> 31);
        } else {
            uint32_t sign;                                       // of y's two values, sixteen bits each
            asm("prmt.b32 %0, %1, %2, 0xFFBB;" : "=r"(sign) : "r"(__float_as_uint(s.x)), "r"(__float_as_uint(s.y)));
            if constexpr (V == 1) w &= (uint16_t)~sign;
            else reinterpret_cast<uint32_t *>(&w)[i] &= ~sign;
        }
    }
    __device__ __forceinline__ void clear(int e) { reinterpret_cast<T *>(&w)[e] = from_f32<T>(0.f); }
    __device__ __forceinline__ float value(int e) const { return to_f32(reinterpret_cast<const T *>(&w)[e]); }
};

// The smaller magnitude of three, not-a-number if one is.
__device__ __forceinline__ float least3(float m, f32x2 y) {
    const float2 s = split2(y);
    float a;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(fabsf(s.x)), "f"(fabsf(s.y)));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(a));
    return m;
}

// What a thread knows of its V channels.
template <int V, bool ONE>
struct NormChannels {
    static constexpr int P = (V + 1) / 2, W = ONE ? 1 : P;
    f32x2 minus_mean[W], scale[P], beta[P];                      // scale = gamma r
    __device__ __forceinline__ f32x2 centred(f32x2 x, int i) const { return add2(x, minus_mean[ONE ? 0 : i]); }
    __device__ __forceinline__ f32x2 y(f32x2 xc, int i) const { return fma2(xc, scale[i], beta[i]); }
};

// 1 / (1 + exp(-y)); exp(-y) = infinity gives 0.  The exponent is rounded once (|y| 2^-24 of the exponential), ex2.approx and rcp.approx add 2^-22
// and 2^-23: for y = -20 1.5e-6 of the result, which is 2e-9 there; fp32 tensors have the same.
__device__ __forceinline__ f32x2 sigmoid2(f32x2 y) {
    const float2 t = split2(mul2(y, both(-1.44269504f)));
    float e0, e1, r0, r1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t.y));
    const float2 d = split2(add2(pair(e0, e1), both(1.f)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(d.y));
    return pair(r0, r1);
}

template <class T, int V, int ACT, bool ONE>
__device__ __forceinline__ NormVec<T, V> norm_forward(const NormVec<T, V> &x, const NormChannels<V, ONE> &k) {
    NormVec<T, V> z;
#pragma unroll
    for (int i = 0; i < NormVec<T, V>::kPairs; ++i) {
        f32x2 y = k.y(k.centred(x.get(i), i), i);
        if constexpr (ACT == CONVBN_ACT_SILU) y = mul2(y, sigmoid2(y));
        z.put(i, y);
    }
    if constexpr (ACT == CONVBN_ACT_RELU) z.relu();
    return z;
}

// ReLU: dz where y > 0.  The sign of y decides a whole gradient.  (The forward call's max(y, 0) has nothing to decide: next to zero it is off by y's
// own rounding, on either side.)  x - mean and gamma r are each off by half a step, so y in fp32 by less than
// 4 * 2^-24 of gamma r (x - mean), which is next to |beta| where y is next to zero: if one of the V values is within `near` = 2^-20 max |beta|
// (or no number), each sign is taken in 64 bits.
template <class T, int V>
__device__ __noinline__ NormVec<T, V> relu_grad_near_zero(NormVec<T, V> dz, NormVec<T, V> x, const float *mean, const float *rstd, const float *gamma,
                                                          const float *beta, int channel, int cg) {
    for (int i = 0; i < V; ++i) {
        const int c = channel + i, g = c / cg;
        const float m = mean[g], v = x.value(i);
        const bool on = v == m && rstd[g] < __int_as_float(0x7f800000) ? beta[c] > 0.f : ((double)v - m) * rstd[g] * gamma[c] + beta[c] > 0.;
        if (!on) dz.clear(i);
    }
    return dz;
}

// dy = dz act'(y) as pairs, and x - mean.  mean .. beta, channel: for the values next to zero (mean, rstd from the sample's first group on,
// gamma, beta and channel from the tensor's first channel on).
struct NormExact {
    const float *mean, *rstd, *gamma, *beta;
    int channel, cg;
    float near;
};
template <class T, int V, int ACT, bool ONE>
__device__ __forceinline__ void norm_grad(const NormVec<T, V> &x, NormVec<T, V> dz, const NormChannels<V, ONE> &k, const NormExact &e,
                                          f32x2 (&xc)[(V + 1) / 2], f32x2 (&dy)[(V + 1) / 2]) {
    constexpr int P = (V + 1) / 2;
#pragma unroll
    for (int i = 0; i < P; ++i) xc[i] = k.centred(x.get(i), i);
    if constexpr (ACT == CONVBN_ACT_RELU) {
        float least = __int_as_float(0x7f800000);
        const NormVec<T, V> given = dz;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            f32x2 y = k.y(xc[i], i);
            if constexpr (V == 1) y = both(split2(y).x);
            least = least3(least, y);
            dz.keep_positive(i, y);
        }
        if (!(least > e.near)) dz = relu_grad_near_zero<T, V>(given, x, e.mean, e.rstd, e.gamma, e.beta, e.channel, e.cg);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        dy[i] = dz.get(i);
        if constexpr (ACT == CONVBN_ACT_SILU) {
            const f32x2 y = k.y(xc[i], i), gate = sigmoid2(y);
            dy[i] = mul2(mul2(dy[i], gate), fma2(y, fma2(gate, both(-1.f), both(1.f)), both(1.f)));
        }
    }
}

}  // namespace convbn
