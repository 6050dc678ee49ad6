// Deploy mode in 8-bit integers, for 1x1 and Linear-BN blocks (convbn_deploy_prepare_quant, convbn_deploy_fwd_quant).
//
//     wq[co] = rne(omega[co] 127 / a_co),  a_co = max |omega[co]|          ws[co] = s[co] a_co / 127      (once)
//     xq[p]  = rne(x[p] 127 / a_p),        a_p  = max |x[p]|               xs[p]  = a_p / 127             (every call)
//     z[p][co] = (sum_k xq wq) xs[p] ws[co] + b'[co]
//
// The BatchNorm scale s goes into the channel scale, so the weights' codes are those of omega itself and no folded weight is
// rounded.  The sum is exact in 32 bits up to C_in = 131072; a code is the rounding of the exact product x * fl(127 / a), formed
// by one fused multiply-add, so it does not depend on how a compiler or a library rounds in between.
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

// A warp per row (output pixel) of X.
template <class T>
__global__ void __launch_bounds__(256) quant_rows_kernel(const Problem pb, int pitch, const T *__restrict__ x, uint8_t *__restrict__ codes,
                                                         float *__restrict__ scale) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    for (long long p = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); p < pb.p; p += (long long)gridDim.x * 8) {
        const int wo = (int)(p % pb.w_out);
        const long long t = p / pb.w_out, img = t / pb.h_out;
        const int ho = (int)(t - img * pb.h_out);
        const T *row = x + ((img * pb.h_in + (long long)ho * pb.stride_h) * pb.w_in + (long long)wo * pb.stride_w) * pb.c_in;
        uint32_t top = 0;
        for (int k = lane; k < pb.c_in; k += 32) top = max(top, magnitude(to_f32(row[k])));
        const RowScale rs = row_scale(__reduce_max_sync(0xffffffffu, top));
        for (int k = lane; k < pitch; k += 32)
            codes[(size_t)p * pitch + k] = k < pb.c_in ? (uint8_t)code_of(to_f32(row[k]), rs.inv) : (uint8_t)0;
        if (lane == 0) scale[p] = rs.scale;
    }
}

template <class T>
__device__ __forceinline__ T finish(int acc, float xs, float ws, float b, const T *add, size_t at, int relu) {
    float z = fmaf((float)acc * xs, ws, b);
    if (add) z += to_f32(add[at]);
    return from_f32<T>(relu ? fmaxf(z, 0.f) : z);
}

// 64 rows x 64 channels a block, 64 bytes of K a turn, 4 x 4 sums a thread.
template <class T>
__global__ void __launch_bounds__(256) quant_product_kernel(long long rows, int c_out, int pitch, const uint8_t *__restrict__ xq,
                                                            const float *__restrict__ xs, const int8_t *__restrict__ wq,
                                                            const float *__restrict__ ws, const float *__restrict__ shift,
                                                            const T *__restrict__ add, int relu, T *__restrict__ z) {
    __shared__ int a[64][17], b[64][17];
    pdl_wait();
    pdl_launch_dependents();
    const long long p0 = (long long)blockIdx.x * 64;
    const int c0 = blockIdx.y * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < pitch; k0 += 64) {
        for (int i = threadIdx.x; i < 64 * 16; i += 256) {
            const int r = i >> 4, q = i & 15, k = k0 + 4 * q;
            a[r][q] = p0 + r < rows && k < pitch ? *(const int *)(xq + (size_t)(p0 + r) * pitch + k) : 0;
            b[r][q] = c0 + r < c_out && k < pitch ? *(const int *)(wq + (size_t)(c0 + r) * pitch + k) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(a[ty * 4 + i][q], b[tx + 16 * j][q], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const long long p = p0 + ty * 4 + i;
        if (p >= rows) break;
        for (int j = 0; j < 4; ++j) {
            const int co = c0 + tx + 16 * j;
            if (co >= c_out) break;
            const size_t at = (size_t)p * c_out + co;
            z[at] = finish<T>(acc[i][j], xs[p], ws[co], shift[co], add, at, relu);
        }
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

cudaError_t launch_quant_rows(const Problem &pb, int dtype, const void *x, void *codes, float *scale, cudaStream_t st) {
    const long long cap = (long long)device_sm_count() * 8, blocks = (pb.p + 7) / 8;
    auto go = [&](auto tag) {
        using T = decltype(tag);
        return launch_pdl(quant_rows_kernel<T>, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(256), 0, st, pb, quant_pitch(pb),
                          (const T *)x, (uint8_t *)codes, scale);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

cudaError_t launch_quant_product(const Problem &pb, int dtype, const void *xq, const float *xs, const void *wq, const float *ws,
                                 const float *shift, const void *add, int relu, void *z, cudaStream_t st) {
    const dim3 grid((unsigned)((pb.p + 63) / 64), (unsigned)((pb.c_out + 63) / 64));
    if (grid.y > 65535u) return cudaErrorInvalidValue;
    auto go = [&](auto tag) {
        using T = decltype(tag);
        return launch_pdl(quant_product_kernel<T>, grid, dim3(256), 0, st, pb.p, pb.c_out, quant_pitch(pb), (const uint8_t *)xq, xs,
                          (const int8_t *)wq, ws, shift, (const T *)add, relu, (T *)z);
    };
    return dtype == CONVBN_F32 ? go(float()) : (dtype == CONVBN_F16 ? go(__half()) : go(__nv_bfloat16()));
}

}  // namespace convbn
