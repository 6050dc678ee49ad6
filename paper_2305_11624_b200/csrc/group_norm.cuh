// Group norm with an activation, channels last: what its kernels share.
//
//     mean, var over the M = H W C/G values of a group of a sample      r = 1 / sqrt(var + eps)
//     y = gamma (x - mean) r + beta        z = act(y)
//     dy = dz act'(y)     dbeta = sum dy     dgamma = sum dy xhat     dx = r (gamma dy - E[gamma dy] - xhat E[gamma dy xhat])
#pragma once

#include "kernels.h"

namespace convbn {

// V elements of T, moved as one access of V sizeof(T) bytes.
template <class T, int V>
struct NormVec {
    static constexpr int kBytes = V * (int)sizeof(T);
    using Word = typename std::conditional<kBytes == 16, uint4, typename std::conditional<kBytes == 8, uint2,
                 typename std::conditional<kBytes == 4, uint32_t, uint16_t>::type>::type>::type;
    Word w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const Word *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<Word *>(p) = w; }
    // the same for data that nothing reads again
    __device__ __forceinline__ void load_last(const T *p) {
        if constexpr (kBytes == 2) w = __ldcs(reinterpret_cast<const unsigned short *>(p));
        else w = __ldcs(reinterpret_cast<const Word *>(p));
    }
    __device__ __forceinline__ void store_last(T *p) const {
        if constexpr (kBytes == 2) __stcs(reinterpret_cast<unsigned short *>(p), w);
        else __stcs(reinterpret_cast<Word *>(p), w);
    }
    __device__ __forceinline__ void get(float (&f)[V]) const {
        const T *t = reinterpret_cast<const T *>(&w);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_f32(t[i]);
    }
    __device__ __forceinline__ void put(const float (&f)[V]) {
        T *t = reinterpret_cast<T *>(&w);
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] = from_f32<T>(f[i]);
    }
};

template <int ACT>
__device__ __forceinline__ float norm_act(float y) {
    if constexpr (ACT == CONVBN_ACT_RELU) return fmaxf(y, 0.f);
    if constexpr (ACT == CONVBN_ACT_SILU) return __fdividef(y, 1.f + __expf(-y));
    return y;
}

// dz act'(y) with y = gamma (x - mean) r + beta, given xc = x - mean and scale = gamma r in fp32.
// ReLU: the sign of y decides a whole gradient.  xc and scale are each off by half a step, so y in fp32 by less than
// 4 * 2^-24 |xc scale|, which is next to |beta| where y is next to zero; there the sign is taken in 64 bits.
template <int ACT>
__device__ __forceinline__ float norm_act_grad(float dz, float xc, float x, float mean, float r, float gamma, float scale, float beta) {
    if constexpr (ACT == CONVBN_ACT_RELU) {
        const float y = fmaf(xc, scale, beta);
        bool on = y > 0.f;
        if (fabsf(y) <= 1e-6f * fabsf(beta)) on = ((double)x - mean) * r * gamma + beta > 0.;
        return on ? dz : 0.f;
    }
    if constexpr (ACT == CONVBN_ACT_SILU) {
        const float y = fmaf(xc, scale, beta);
        const float gate = __fdividef(1.f, 1.f + __expf(-y));
        return dz * gate * fmaf(y, 1.f - gate, 1.f);
    }
    return dz;
}

}  // namespace convbn
