// Orthogonal updates (formulas, pairs of halves, tiles: ortho.cuh): the matrices' norms, their way into tiles, and the products.
#include "ortho.cuh"
#include "sm100_ptx.cuh"

namespace convbn {

using namespace ptx;

namespace {

// Places in a matrix's part of the workspace.
struct OrthoPlace {
    long long x_bytes, s_bytes;                // of X's hi (or lo) tiles; of a symmetric matrix's
    __host__ __device__ OrthoPlace(int rt, int ct) {
        const int d = rt < ct ? rt : ct;
        x_bytes = (long long)rt * ct * 2 * kOrthoTile;
        s_bytes = (long long)d * d * 2 * kOrthoTile;
    }
    __host__ __device__ long long x(int which) const { return which * 2 * x_bytes; }        // X before and after a step, in turn
    __host__ __device__ long long a() const { return 4 * x_bytes; }
    __host__ __device__ long long p() const { return 4 * x_bytes + 2 * s_bytes; }
    __host__ __device__ long long sums() const { return 4 * x_bytes + 4 * s_bytes; }
};
__host__ __device__ inline int ortho_chunks(const OrthoItem &it) { return (int)(((long long)it.rows * it.cols + kOrthoChunk - 1) / kOrthoChunk); }

// The item that task `t` belongs to; `first` picks the member that holds the tasks before it.
template <class F>
__device__ __forceinline__ int find_item(const OrthoTable &tab, int t, F &&first) {
    int lo = 0, hi = tab.items - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(tab.item[mid]) <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ float ortho_read(const OrthoTable &tab, const OrthoItem &it, long long at) {
    if (tab.muon) {
        const float v = it.momentum[at];          // (the new one)
        return tab.nesterov ? fmaf(tab.momentum, v, ((const float *)it.g)[at]) : v;
    }
    return to_f32(((const T *)it.g)[at]);
}

// Sums of squares of a chunk of a matrix's elements, in 64 bits (a gradient's squares leave fp32's range); muon: the momentum's step on the way.
template <class T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws) {
    __shared__ double part[8];
    pdl_wait();
    pdl_launch_dependents();
    const int task = blockIdx.x;
    const OrthoItem &it = tab.item[find_item(tab, task, [](const OrthoItem &i) { return i.first_sum; })];
    const int chunks = ortho_chunks(it), local = task - it.first_sum, copy = local / chunks, chunk = local % chunks;
    const long long size = (long long)it.rows * it.cols, from = (long long)chunk * kOrthoChunk;
    const int n = (int)min((long long)kOrthoChunk, size - from);
    const long long base = copy * size + from;
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += 256) {
        if (tab.muon) it.momentum[base + i] = fmaf(tab.momentum, it.momentum[base + i], ((const float *)it.g)[base + i]);
        const double u = ortho_read<T>(tab, it, base + i);
        s += u * u;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += part[i];
        ((double *)(ws + it.base + copy * it.bytes + OrthoPlace(it.rt, it.ct).sums()))[chunk] = s;
    }
}

// A tile of X = G / (|G| + eps), zeros beyond the matrix.
template <class T>
__global__ void __launch_bounds__(256) ortho_tile_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws) {
    __shared__ double part[8];
    pdl_wait();
    pdl_launch_dependents();
    const int task = blockIdx.x;
    const OrthoItem &it = tab.item[find_item(tab, task, [](const OrthoItem &i) { return i.first_tile; })];
    const int per = it.rt * it.ct * 2, local = task - it.first_tile, copy = local / per, tile = local % per;
    const OrthoPlace place(it.rt, it.ct);
    uint8_t *m = ws + it.base + copy * it.bytes;
    const double *sums = (const double *)(m + place.sums());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double s = 0.;
    for (int i = threadIdx.x; i < ortho_chunks(it); i += 256) s += sums[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) part[warp] = s;
    __syncthreads();
    s = part[0];
    for (int i = 1; i < 8; ++i) s += part[i];
    const double inv = (double)kOrthoScale / (sqrt(s) + tab.eps);
    const int row0 = tile / (2 * it.ct) * 128, col0 = tile % (2 * it.ct) * 64;
    uint8_t *hi = m + place.x(0) + (long long)tile * kOrthoTile, *lo = hi + place.x_bytes;
    const long long base = copy * ((long long)it.rows * it.cols);
#pragma unroll 4
    for (int k = 0; k < 32; ++k) {
        const int r = warp + 8 * (k >> 1), c = lane + 32 * (k & 1);
        float v = 0.f;
        if (row0 + r < it.rows && col0 + c < it.cols)
            v = (float)(ortho_read<T>(tab, it, base + (long long)(row0 + r) * it.cols + col0 + c) * inv);
        const __half h = __float2half_rn(v);
        const uint32_t at = ortho_chunk(r, c >> 3) + (c & 7) * 2;
        *(__half *)(hi + at) = h;
        *(__half *)(lo + at) = __float2half_rn(v - __half2float(h));
    }
}

// ---- products ---------------------------------------------------------------------------------------------------------------------
// CTA = 6 warps: 0 loads, 1 MMA issuer and owner of tensor memory, 2-5 epilogue.  A task is a 128 x 128 tile of A, P or X; k in steps of 64.
// A step's four tiles (hi and lo of both operands) are 64 KB and feed twelve MMAs.  hi hi is summed apart from the other two products:
// the tensor core's sums drift towards zero with their length, and those of small numbers do not notice.  For the same reason a sum over
// more than 1024 k is cut: the epilogue adds the pieces up in registers, in fp32 with rounding.
constexpr int kOThreads = 192;
constexpr int kOStages = 3;
constexpr uint32_t kOStage = 4 * kOrthoTile;
constexpr int kOSegment = 16;                              // steps of a sum
constexpr uint32_t kOStaging = 4 * 8192;                   // an epilogue warp's 32 rows x 64 columns, hi and lo (or fp32)

struct OrthoCtl {
    uint64_t full[kOStages], empty[kOStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
};

// Where an operand of a step lies: one tile (K-major), or the halves of two (MN-major).
struct OrthoOperand {
    long long first, second;
    bool mn;
};

struct OrthoTask {
    const OrthoItem *it;
    uint8_t *m;                  // the matrix's part of the workspace
    int copy;
    int i, j;                    // row and column of the tile of 128 x 128
    int steps;                   // of k
};

__device__ __forceinline__ OrthoTask ortho_task(const OrthoTable &tab, uint8_t *ws, int phase, int t) {
    OrthoTask k;
    const bool update = phase == kOrthoUpdate;
    k.it = &tab.item[find_item(tab, t, [update](const OrthoItem &i) { return update ? i.first_update : i.first_gram; })];
    const OrthoItem &it = *k.it;
    const int d = min(it.rt, it.ct), side = min(it.rows, it.cols);
    int local = t - (update ? it.first_update : it.first_gram);
    if (update) {
        const int per = it.rt * it.ct;
        k.copy = local / per;
        local -= k.copy * per;
        k.i = local / it.ct;
        k.j = local % it.ct;
    } else {
        const int per = d * (d + 1) / 2;
        k.copy = local / per;
        local -= k.copy * per;
        // row i of the lower half starts at i (i + 1) / 2
        int i = (int)((sqrtf(8.f * (float)local + 1.f) - 1.f) * 0.5f);
        while (i * (i + 1) / 2 > local) --i;
        while ((i + 1) * (i + 2) / 2 <= local) ++i;
        k.i = i;
        k.j = local - i * (i + 1) / 2;
    }
    k.m = ws + it.base + k.copy * it.bytes;
    k.steps = ((phase == kOrthoGram ? max(it.rows, it.cols) : side) + 63) / 64;
    return k;
}

__device__ __forceinline__ OrthoOperand symmetric_operand(long long at, int d, int block, int step) {
    const int j = step >> 1;
    if (j <= block) return {at + ((long long)block * 2 * d + step) * kOrthoTile, 0, false};
    const long long first = at + ((long long)j * 2 * d + 2 * block) * kOrthoTile + (step & 1) * (kOrthoTile / 2);
    return {first, first + kOrthoTile, true};
}
__device__ __forceinline__ OrthoOperand rows_operand(long long at, int ct, int block, int step) {          // k along X's rows
    return {at + ((long long)block * 2 * ct + step) * kOrthoTile, 0, false};
}
__device__ __forceinline__ OrthoOperand cols_operand(long long at, int ct, int block, int step) {          // k down X's columns
    const long long first = at + ((long long)(step >> 1) * 2 * ct + 2 * block) * kOrthoTile + (step & 1) * (kOrthoTile / 2);
    return {first, first + kOrthoTile, true};
}

// Operands of step `step` of a task (offsets in the matrix's part; lo lies half_a, half_b behind).
__device__ __forceinline__ void ortho_operands(const OrthoTask &k, int phase, int which, int step, OrthoOperand &a, OrthoOperand &b, long long &half_a,
                                               long long &half_b) {
    const OrthoItem &it = *k.it;
    const OrthoPlace place(it.rt, it.ct);
    const int d = min(it.rt, it.ct);
    const bool tall = it.rows > it.cols;
    const long long x = place.x(which);
    if (phase == kOrthoGram) {
        half_a = half_b = place.x_bytes;
        a = tall ? cols_operand(x, it.ct, k.i, step) : rows_operand(x, it.ct, k.i, step);
        b = tall ? cols_operand(x, it.ct, k.j, step) : rows_operand(x, it.ct, k.j, step);
    } else if (phase == kOrthoSquare) {
        half_a = half_b = place.s_bytes;
        a = symmetric_operand(place.a(), d, k.i, step);
        b = symmetric_operand(place.a(), d, k.j, step);
    } else if (tall) {
        half_a = place.x_bytes;
        half_b = place.s_bytes;
        a = rows_operand(x, it.ct, k.i, step);
        b = symmetric_operand(place.p(), d, k.j, step);
    } else {
        half_a = place.s_bytes;
        half_b = place.x_bytes;
        a = symmetric_operand(place.p(), d, k.i, step);
        b = cols_operand(x, it.ct, k.j, step);
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bulk_store(void *dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}

__device__ __forceinline__ float2 half_pair(uint32_t hi, uint32_t lo) {
    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi)), l = __half22float2(*reinterpret_cast<const __half2 *>(&lo));
    return make_float2(h.x + l.x, h.y + l.y);
}

// One phase of step `index`; the last update of the last step goes out instead of into tiles.
template <class T>
__global__ void __launch_bounds__(kOThreads, 1) ortho_product_kernel(const __grid_constant__ OrthoTable tab, uint8_t *__restrict__ ws, int phase, int index,
                                                                     int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *staging = tiles + kOStages * kOStage;
    OrthoCtl *ctl = (OrthoCtl *)(staging + kOStaging);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;
    const int tasks = phase == kOrthoUpdate ? tab.updates : tab.grams, which = index & 1;
    auto give_up = [&]() { atomicOr(err, ERRW_TIMEOUT); ctl->abort_flag = 1; };

    if (threadIdx.x == 64) {
        for (int s = 0; s < kOStages; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&ctl->acc_full[a], 1); mbar_init(&ctl->acc_empty[a], 4); }
        ctl->abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc(&ctl->tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem_base = ctl->tmem_base;

    if (warp == 0) {
        if (elect_one()) {
            uint32_t it = 0;
            bool ok = true;
            for (int t = blockIdx.x; ok && t < tasks; t += gridDim.x) {
                const OrthoTask k = ortho_task(tab, ws, phase, t);
                for (int s = 0; s < k.steps; ++s, ++it) {
                    const uint32_t slot = it % kOStages;
                    ok = mbar_wait_bounded(&ctl->empty[slot], ((it / kOStages) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    OrthoOperand a, b;
                    long long ha, hb;
                    ortho_operands(k, phase, which, s, a, b, ha, hb);
                    const uint32_t bar = smem_u32(&ctl->full[slot]), dst = smem_u32(tiles) + slot * kOStage;
                    mbar_arrive_expect_tx(bar, kOStage);
                    auto bring = [&](const OrthoOperand &o, long long half, uint32_t to) {
                        if (o.mn) {
                            bulk_load(to, k.m + o.first + half, kOrthoTile / 2, bar);
                            bulk_load(to + kOrthoTile / 2, k.m + o.second + half, kOrthoTile / 2, bar);
                        } else {
                            bulk_load(to, k.m + o.first + half, kOrthoTile, bar);
                        }
                    };
                    bring(a, 0, dst);
                    bring(b, 0, dst + 2 * kOrthoTile);
                    bring(a, ha, dst + kOrthoTile);
                    bring(b, hb, dst + 3 * kOrthoTile);
                }
            }
            if (!ok) {
                give_up();
                for (uint32_t j = it > kOStages ? it - kOStages : 0; j < it; ++j)          // let the copies in flight land
                    mbar_wait_bounded(&ctl->full[j % kOStages], (j / kOStages) & 1u, nullptr, 200000000ull);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t hi = smem_desc_hi_sw128(1024);
            uint32_t it = 0, acc_it = 0;
            bool ok = true;
            for (int t = blockIdx.x; ok && t < tasks; t += gridDim.x) {
                const OrthoTask k = ortho_task(tab, ws, phase, t);
                for (int s = 0; ok && s < k.steps; ++s, ++it) {
                    const uint32_t acc = acc_it & 1u, d = tmem_base + acc * 256u;
                    if (s % kOSegment == 0) {
                        ok = mbar_wait_bounded(&ctl->acc_empty[acc], ((acc_it >> 1) & 1u) ^ 1u, abort_flag);
                        if (!ok) break;
                        tc_fence_after_sync();
                    }
                    const uint32_t slot = it % kOStages;
                    ok = mbar_wait_bounded(&ctl->full[slot], (it / kOStages) & 1u, abort_flag);
                    if (!ok) break;
                    OrthoOperand a, b;
                    long long ha, hb;
                    ortho_operands(k, phase, which, s, a, b, ha, hb);
                    const uint32_t idesc = idesc_h16_f32(128, 128, a.mn, b.mn, 1), base = smem_u32(tiles) + slot * kOStage;
                    const uint32_t a_hi = smem_desc_lo(base, a.mn ? 8192 : 16), a_lo = a_hi + (kOrthoTile >> 4);
                    const uint32_t b_hi = smem_desc_lo(base + 2 * kOrthoTile, b.mn ? 8192 : 16), b_lo = b_hi + (kOrthoTile >> 4);
                    const uint32_t sa = a.mn ? 128u : 2u, sb = b.mn ? 128u : 2u, first = s % kOSegment;
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q) umma_bf16_ss_sel(d, a_hi + q * sa, hi, b_hi + q * sb, hi, idesc, first + q);
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q) {
                        umma_bf16_ss_sel(d + 128, a_hi + q * sa, hi, b_lo + q * sb, hi, idesc, first + q);
                        umma_bf16_ss_halves<true>(d + 128, a_lo + q * sa, hi, b_hi + q * sb, hi, idesc);
                    }
                    umma_commit(&ctl->empty[slot]);
                    if (s + 1 == k.steps || s % kOSegment == kOSegment - 1) { umma_commit(&ctl->acc_full[acc]); ++acc_it; }
                }
            }
            if (!ok) give_up();
        }
    } else {
        const int quarter = warp & 3;
        uint8_t *buf = staging + (warp - 2) * 8192;
        const bool last = phase == kOrthoUpdate && index + 1 == tab.steps;
        uint32_t acc_it = 0;
        bool ok = true;
        for (int t = blockIdx.x; ok && t < tasks; t += gridDim.x) {
            const OrthoTask k = ortho_task(tab, ws, phase, t);
            const OrthoItem &it = *k.it;
            const OrthoPlace place(it.rt, it.ct);
            const int segments = (k.steps + kOSegment - 1) / kOSegment;
            float v[128];
            for (int g = 0; g < segments; ++g, ++acc_it) {
                const uint32_t acc = acc_it & 1u;
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->acc_full[acc], (acc_it >> 1) & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t from = tmem_base + acc * 256u + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t p[32], q[32];
                    tmem_ld_32x32(from + h * 32, p);
                    tmem_ld_32x32(from + 128 + h * 32, q);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float sum = __uint_as_float(p[i]) + __uint_as_float(q[i]);
                        v[h * 32 + i] = g == 0 ? sum : v[h * 32 + i] + sum;
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->acc_empty[acc]);
            }
            if (!ok) break;
            const uint32_t row = quarter * 32 + lane;
            // two tiles of 64 columns; numbers are 2^10 times what they stand for, sums of products 2^20 times
            const long long x_at = ((long long)k.i * 2 * it.ct + 2 * k.j) * kOrthoTile;
            const long long s_at = ((long long)k.i * 2 * min(it.rt, it.ct) + 2 * k.j) * kOrthoTile;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (lane == 0) tma_store_wait_read<0>();
                __syncwarp();
                const uint8_t *old = nullptr;
                long long old_half = 0;
                float f_old = 0.f, f_new = 1.f / kOrthoScale;
                if (phase == kOrthoSquare) {
                    old = k.m + place.a() + s_at + h * kOrthoTile; old_half = place.s_bytes; f_old = kOrthoB; f_new = kOrthoC / kOrthoScale;
                } else if (phase == kOrthoUpdate) {
                    old = k.m + place.x(which) + x_at + h * kOrthoTile; old_half = place.x_bytes; f_old = kOrthoA;
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float *w = &v[h * 64 + c * 8];
                    const uint32_t at = ortho_chunk(row, c);
                    if (old) {
                        const uint4 oh = __ldcg((const uint4 *)(old + at)), ol = __ldcg((const uint4 *)(old + old_half + at));
                        const float2 o[4] = {half_pair(oh.x, ol.x), half_pair(oh.y, ol.y), half_pair(oh.z, ol.z), half_pair(oh.w, ol.w)};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            w[2 * e] = fmaf(f_old, o[e].x, w[2 * e] * f_new);
                            w[2 * e + 1] = fmaf(f_old, o[e].y, w[2 * e + 1] * f_new);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] *= f_new;
                    }
                    if (!last) {
                        uint32_t ph[4], pl[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __half2 hh = __floats2half2_rn(w[2 * e], w[2 * e + 1]);
                            const float2 back = __half22float2(hh);
                            const __half2 hl = __floats2half2_rn(w[2 * e] - back.x, w[2 * e + 1] - back.y);
                            ph[e] = *reinterpret_cast<const uint32_t *>(&hh);
                            pl[e] = *reinterpret_cast<const uint32_t *>(&hl);
                        }
                        const uint32_t to = ortho_chunk(lane, c);          // (a warp's rows start on a multiple of 8)
                        *(uint4 *)(buf + to) = make_uint4(ph[0], ph[1], ph[2], ph[3]);
                        *(uint4 *)(buf + 4096 + to) = make_uint4(pl[0], pl[1], pl[2], pl[3]);
                    } else {
                        // fp32, [32][64], chunks of four in an order that spreads a column over the banks
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            *(float4 *)(buf + lane * 256 + (((2 * c + e) ^ (lane & 15)) << 4)) =
                                make_float4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                    }
                }
                if (!last) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        uint8_t *to;
                        long long half;
                        if (phase == kOrthoUpdate) { to = k.m + place.x(which ^ 1) + x_at; half = place.x_bytes; }
                        else { to = k.m + (phase == kOrthoGram ? place.a() : place.p()) + s_at; half = place.s_bytes; }
                        to += h * kOrthoTile + quarter * 4096;
                        bulk_store(to, buf, 4096);
                        bulk_store(to + half, buf + 4096, 4096);
                        tma_store_commit();
                    }
                } else {
                    __syncwarp();
                    const int r0 = k.i * 128 + quarter * 32, c0 = k.j * 128 + h * 64;
                    const long long base = k.copy * ((long long)it.rows * it.cols);
                    for (int r = 0; r < 32 && r0 + r < it.rows; ++r)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int c = lane + 32 * e;
                            if (c0 + c >= it.cols) continue;
                            const float o = *(const float *)(buf + r * 256 + (((c >> 2) ^ (r & 15)) << 4) + (c & 3) * 4) * (1.f / kOrthoScale);
                            const long long at = base + (long long)(r0 + r) * it.cols + c0 + c;
                            if (tab.muon) {
                                const float w = fmaf(-it.scale, o, tab.keep * it.master[at]);
                                it.master[at] = w;
                                if (it.out) ((T *)it.out)[at] = from_f32<T>(w);
                            } else {
                                ((T *)it.out)[at] = from_f32<T>(o);
                            }
                        }
                    __syncwarp();
                }
            }
        }
        if (!ok && lane == 0) give_up();
        if (lane == 0) tma_store_wait_all<0>();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, 512);
}

template <class T>
cudaError_t launch_ortho_t(const OrthoTable &t, uint8_t *ws, cudaStream_t st) {
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    cudaError_t e = launch_pdl(ortho_norm_kernel<T>, dim3((unsigned)t.sums), dim3(256), 0, st, t, ws);
    if (e == cudaSuccess) e = launch_pdl(ortho_tile_kernel<T>, dim3((unsigned)t.tiles), dim3(256), 0, st, t, ws);
    if (e != cudaSuccess) return e;
    auto kernel = ortho_product_kernel<T>;
    static PerDevice attr, carve;
    constexpr int smem = 1024 + kOStages * kOStage + kOStaging + sizeof(OrthoCtl);
    if (e = max_dynamic_smem_once(kernel, smem, &attr); e != cudaSuccess) return e;
    prefer_max_shared_once(kernel, &carve);
    const int sms = device_sm_count();
    for (int index = 0; index < t.steps; ++index)
        for (int phase = kOrthoGram; phase <= kOrthoUpdate; ++phase) {
            const int tasks = phase == kOrthoUpdate ? t.updates : t.grams;
            e = launch_pdl(kernel, dim3((unsigned)(tasks < sms ? tasks : sms)), dim3(kOThreads), smem, st, t, ws, phase, index, err);
            if (e != cudaSuccess) return e;
        }
    return e;
}

}  // namespace

size_t ortho_matrix_bytes(int rows, int cols) {
    OrthoItem it;
    it.rows = rows; it.cols = cols;
    const OrthoPlace place((rows + 127) / 128, (cols + 127) / 128);
    return (size_t)place.sums() + align_up((size_t)ortho_chunks(it) * sizeof(double), 1024);
}

long long ortho_place(OrthoTable &t, int i, long long end) {
    OrthoItem &it = t.item[i];
    it.rt = (it.rows + 127) / 128;
    it.ct = (it.cols + 127) / 128;
    const int d = it.rt < it.ct ? it.rt : it.ct;
    if (i == 0) t.sums = t.tiles = t.grams = t.updates = 0;
    it.first_sum = t.sums; it.first_tile = t.tiles; it.first_gram = t.grams; it.first_update = t.updates;
    t.sums += it.count * ortho_chunks(it);
    t.tiles += it.count * it.rt * it.ct * 2;
    t.grams += it.count * (d * (d + 1) / 2);
    t.updates += it.count * it.rt * it.ct;
    it.base = end;
    it.bytes = (long long)ortho_matrix_bytes(it.rows, it.cols);
    return end + it.count * it.bytes;
}

cudaError_t launch_ortho(const OrthoTable &t, void *workspace, cudaStream_t st) {
    switch (t.dtype) {
        case CONVBN_F32: return launch_ortho_t<float>(t, (uint8_t *)workspace, st);
        case CONVBN_F16: return launch_ortho_t<__half>(t, (uint8_t *)workspace, st);
        default: return launch_ortho_t<__nv_bfloat16>(t, (uint8_t *)workspace, st);
    }
}

}  // namespace convbn
