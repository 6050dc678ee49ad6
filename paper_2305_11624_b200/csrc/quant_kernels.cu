// Deploy mode in 8-bit integers, for 1x1 and Linear-BN blocks (convbn_deploy_prepare_quant, convbn_deploy_fwd_quant).
//
//     wq[co] = rne(omega[co] 127 / a_co),  a_co = max |omega[co]|          ws[co] = s[co] a_co / 127      (once)
//     xq[p]  = rne(x[p] 127 / a_p),        a_p  = max |x[p]|               xs[p]  = a_p / 127             (every call)
//     z[p][co] = (sum_k xq wq) xs[p] ws[co] + b'[co]
//
// The BatchNorm scale s goes into the channel scale, so the weights' codes are those of omega itself and no folded weight is
// rounded.  The sum is exact in 32 bits up to C_in = 131072; a code is the rounding of the exact product of x
// and fl(127 fl(1 / a)), formed by one fused multiply-add, so it does not depend on how a compiler or a library rounds in between.
#include "kernels.h"
#include "quant8.cuh"

namespace convbn {

namespace {

// |x| as bits: the largest one is the largest magnitude, and an infinity or a NaN is above every number.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t code_of(float x, float inv) { return inv == 0.f ? 0u : code_bits(x, inv) & 0xFFu; }

template <class T>
__global__ void __launch_bounds__(256) quant_weights_kernel(int c_in, int pitch, const T *__restrict__ w, const float *__restrict__ b,
                                                            const float *__restrict__ gamma, const float *__restrict__ beta,
                                                            const float *__restrict__ mean, const float *__restrict__ var, float eps,
                                                            int8_t *__restrict__ codes, float *__restrict__ scale,
                                                            float *__restrict__ shift) {
    __shared__ uint32_t part[8];
    pdl_wait();
    pdl_launch_dependents();
    const int co = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T *row = w + (size_t)co * c_in;
    uint32_t top = 0;
    for (int k = threadIdx.x; k < c_in; k += 256) top = max(top, magnitude(to_f32(row[k])));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) part[warp] = top;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, part[lane & 7]);
    const RowScale rs = row_scale(top);
    for (int k = threadIdx.x; k < pitch; k += 256)
        codes[(size_t)co * pitch + k] = k < c_in ? (int8_t)code_of(to_f32(row[k]), rs.inv) : (int8_t)0;
    if (threadIdx.x == 0) {
        const float r = __frcp_rn(__fsqrt_rn(var[co] + eps)), s = gamma[co] * r;
        scale[co] = s * rs.scale;
        shift[co] = ((b ? b[co] : 0.f) - mean[co]) * s + beta[co];
    }
}

}  // namespace

bool quant_eligible(const Problem &pb) {
    return pb.groups == 1 && pb.kh == 1 && pb.kw == 1 && pb.pad_h == 0 && pb.pad_w == 0 && pb.c_in <= 131072 &&
           pb.p < (1LL << 31) - 256;
}

size_t quant_codes_bytes(const Problem &pb) { return (size_t)pb.p * quant_pitch(pb); }

cudaError_t launch_quant_weights(const Problem &pb, int dtype, const void *w, const float *b, const float *gamma, const float *beta,
                                 const float *mean, const float *var, void *codes, float *scale, float *shift, cudaStream_t st) {
    auto go = [&](auto tag) {
        using T = decltype(tag);
        return launch_pdl(quant_weights_kernel<T>, dim3(pb.c_out), dim3(256), 0, st, pb.c_in, quant_pitch(pb), (const T *)w, b, gamma,
                          beta, mean, var, pb.eps, (int8_t *)codes, scale, shift);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

}  // namespace convbn
