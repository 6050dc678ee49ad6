// The deployed 8-bit product for few rows (a token, an image's last layer), in one launch: a block makes codes of its 16 rows in
// shared memory and multiplies them with the codes of a few channels, which its warps read from memory once, 16 bytes a lane, straight
// into the fragments of warp-level MMAs (m16n8k32, 8-bit integers).  Within a step of 64 the positions of K are taken in the order in
// which four lanes' 16 bytes give them: the sum does not depend on it, both operands use the same.
// Bound by latency: launch, rows, scales, weights, one after the other.  K is cut among the warps of a block, whose integer sums meet
// in shared memory (exact, in any order).
#include "kernels.h"
#include "quant8.cuh"

namespace convbn {

namespace {

constexpr int kSRows = 16, kSMaxK = 4096;

__device__ __forceinline__ void mma_16x8x32_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// KS of the eight warps share eight channels; a lane keeps KEEP chunks of eight elements of each of its two rows.
template <class T, int KS, int KEEP>
__global__ void __launch_bounds__(256) quant_small_kernel(const RowMap rows, uint32_t p, int k, int pitch, int n, int vec, int relu,
                                                          const T *__restrict__ x, const int8_t *__restrict__ wq,
                                                          const float *__restrict__ ws, const float *__restrict__ shift,
                                                          const T *__restrict__ add, T *__restrict__ z) {
    constexpr int NG = 8 / KS;                                // groups of eight channels
    extern __shared__ uint8_t codes[];                        // [16][kp + 16]
    __shared__ float xs[kSRows];
    __shared__ int sums[KS > 1 ? NG * KS : 1][32][4];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int ks = warp % KS, ng = warp / KS, kp = (k + 63) / 64 * 64, row_bytes = kp + 16;      // (16: rows start in other banks)
    const uint32_t row0 = blockIdx.x * kSRows;
    const int n0 = (blockIdx.y * NG + ng) * 8;
    // the first weights are requested before the rows: they depend on nothing
    const int8_t *wrow = wq + (size_t)min(n0 + g, n - 1) * pitch + 16 * t;
    const int steps = kp / 64;
    constexpr int AHEAD = 4;
    uint4 w[AHEAD];
    auto weights = [&](int s) { return s < steps && 64 * s + 16 * t < pitch ? __ldg((const uint4 *)(wrow + 64 * s)) : make_uint4(0u, 0u, 0u, 0u); };
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) w[a] = weights(ks + a * KS);
    // rows 2 warp and 2 warp + 1
    {
        const T *src[2];
        Eight<T> kept[2][KEEP];
        auto read = [&](Eight<T> &v, const T *row, int at) {
            if (at >= k) v.zero();
            else if (vec) v.load(row + at);
            else v.load_some(row + at, k - at);
        };
        bool there[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            there[h] = row0 + 2 * warp + h < p;
            src[h] = x + (there[h] ? rows.at(row0 + 2 * warp + h) : 0);
#pragma unroll
            for (int c = 0; c < KEEP; ++c)
                if (there[h]) read(kept[h][c], src[h], (c * 32 + lane) * 8);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!there[h]) break;
            const int r = 2 * warp + h;
            uint32_t top = kept[h][0].top();
#pragma unroll
            for (int c = 1; c < KEEP; ++c) top = max(top, kept[h][c].top());
            for (int at = (KEEP * 32 + lane) * 8; at < k; at += 256) {
                Eight<T> v;
                read(v, src[h], at);
                top = max(top, v.top());
            }
            const RowScale rs = row_scale(Eight<T>::top_f32(__reduce_max_sync(0xffffffffu, top)));
#pragma unroll
            for (int c = 0; c < KEEP; ++c)
                if ((c * 32 + lane) * 8 < kp) *(uint2 *)(codes + r * row_bytes + (c * 32 + lane) * 8) = kept[h][c].codes(rs.inv);
            for (int at = (KEEP * 32 + lane) * 8; at < kp; at += 256) {
                Eight<T> v;
                read(v, src[h], at);
                *(uint2 *)(codes + r * row_bytes + at) = v.codes(rs.inv);
            }
            if (lane == 0) xs[r] = rs.scale;
        }
    }
    __syncthreads();
    int acc[4] = {0, 0, 0, 0};
    const uint8_t *a_lo = codes + g * row_bytes + 16 * t, *a_hi = a_lo + 8 * row_bytes;
    for (int s0 = ks; s0 < steps; s0 += AHEAD * KS) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int s = s0 + a * KS;
            const uint4 b = w[a];
            w[a] = weights(s + AHEAD * KS);
            if (s >= steps) continue;
            const uint4 lo = *(const uint4 *)(a_lo + 64 * s), hi = *(const uint4 *)(a_hi + 64 * s);
            mma_16x8x32_s8(acc, lo.x, hi.x, lo.y, hi.y, b.x, b.y);
            mma_16x8x32_s8(acc, lo.z, hi.z, lo.w, hi.w, b.z, b.w);
        }
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[warp][lane][e] = acc[e];
        __syncthreads();
        if (ks != 0) return;
#pragma unroll
        for (int o = 1; o < KS; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += sums[warp + o][lane][e];
    }
    // rows g and g + 8, channels 2 t and 2 t + 1
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int r = g + (e >> 1) * 8, col = n0 + 2 * t + (e & 1);
        if (row0 + r >= p || col >= n) continue;
        const size_t at = (size_t)(row0 + r) * n + col;
        float f = fmaf((float)acc[e] * xs[r], __ldg(ws + col), __ldg(shift + col));
        if (add) f += to_f32(add[at]);
        z[at] = from_f32<T>(relu ? fmaxf(f, 0.f) : f);
    }
}

}  // namespace

// This kernel and the two of quant_gemm.cu, us: one row 64 -> 64 2.1 and 4.4, 2048 -> 1000 4.2 and 7.0; 16 rows 2048 -> 2048 5.7 and
// 7.2; 64 rows 512 -> 2048 4.4 and 5.2; 256 rows 512 -> 1024 4.7 and 5.4; 4000 rows 256 -> 64 3.6 and 6.0.  Every block reads all
// codes of its channels, and results leave one by one: it pays up to 2^27 products and 2^19 results (256 rows 512 -> 2048 7.5 and 5.4,
// 4000 rows 64 -> 512 11.9 and 5.9), beyond 1024 channels up to 16 rows (64 rows 2048 -> 1000 8.8 and 7.0).
bool quant_small_eligible(const Problem &pb) {
    return pb.c_in <= kSMaxK && (pb.c_in <= 1024 || pb.p <= kSRows) && pb.p * pb.c_out <= (1LL << 19) &&
           pb.p * pb.c_out <= (1LL << 27) / pb.c_in;
}

cudaError_t launch_quant_small(const Problem &pb, int dtype, const void *x, const void *wq, const float *ws, const float *shift,
                               const void *add, int relu, void *z, cudaStream_t st) {
    const int es = dtype == CONVBN_F32 ? 4 : 2, kp = (pb.c_in + 63) / 64 * 64;
    const RowMap rows = quant_row_map(pb);
    const int vec = pb.c_in % 8 == 0 && (size_t)pb.c_in * es % 16 == 0;
    const int blocks = (int)((pb.p + kSRows - 1) / kSRows), groups = (pb.c_out + 7) / 8;
    auto sized = [&](auto tag, auto ks, auto keep) {
        using T = decltype(tag);
        constexpr int KS = decltype(ks)::value, KEEP = decltype(keep)::value;
        static PerDevice attr;
        auto kernel = quant_small_kernel<T, KS, KEEP>;
        if (cudaError_t e = max_dynamic_smem_once(kernel, kSRows * (kSMaxK + 16), &attr); e != cudaSuccess) return e;
        return launch_pdl(kernel, dim3((unsigned)blocks, (unsigned)((groups + 8 / KS - 1) / (8 / KS))), dim3(256), (size_t)kSRows * (kp + 16), st,
                          rows, (uint32_t)pb.p, pb.c_in, quant_pitch(pb), pb.c_out, vec, relu, (const T *)x, (const int8_t *)wq, ws, shift,
                          (const T *)add, (T *)z);
    };
    auto go = [&](auto tag, auto ks) {
        using std::integral_constant;
        return pb.c_in <= 512 ? sized(tag, ks, integral_constant<int, 2>()) : sized(tag, ks, integral_constant<int, 8>());
    };
    // K cut as far as blocks are missing to give every SM one, and as there are steps of 64 for the warps
    auto typed = [&](auto tag) {
        using std::integral_constant;
        const long long warps = (long long)blocks * groups, sms = device_sm_count();
        if (warps <= 2 * sms && kp >= 512) return go(tag, integral_constant<int, 8>());
        if (warps <= 4 * sms && kp >= 256) return go(tag, integral_constant<int, 4>());
        if (warps <= 8 * sms && kp >= 128) return go(tag, integral_constant<int, 2>());
        return go(tag, integral_constant<int, 1>());
    };
    return dtype == CONVBN_F32 ? typed(float()) : (dtype == CONVBN_F16 ? typed(__half()) : typed(__nv_bfloat16()));
}

}  // namespace convbn
