// The deployed 1x1 block in 8-bit integers as ONE kernel (convbn_deploy_fwd_quant): rows of X become codes on their way into shared
// memory, the product runs on the tensor cores (tcgen05, 8-bit operands, 32-bit integer sums in tensor memory), scales, shift,
// addend and ReLU are applied to the sums.  X is read once in its storage type, Z written once; codes exist on chip only.
//
// CTA = 18 warps: 0 weight tiles (TMA), 1 MMA issuer and owner of tensor memory, 2-9 epilogue (two groups of four, an accumulator
// each), 10-17 rows to codes.  A unit of work is 128 rows (and a span of channel tiles where there are few rows): the last eight
// warps read its rows whole, a row by 8, 16 or 32 lanes, find the largest magnitude, and write the codes as the K-major A operand
// (128-byte swizzle); the next rows are requested before these are converted.
#include "kernels.h"
#include "quant8.cuh"

namespace convbn {

using namespace ptx;

namespace {

constexpr int kQRows = 128;                      // rows of a unit (UMMA M)
constexpr uint32_t kQBlock = kQRows * 128;       // [128 rows][128 codes] of the A operand
constexpr int kQThreads = 576;
constexpr int kQLoadWarp = 10;                   // first of the eight warps that make codes
constexpr int kQMaxStages = 8;
constexpr uint32_t kQStage = 32 * 128;           // an epilogue warp's box: [32 rows][128 bytes]
constexpr int kQSlots = 4;                       // row scales of so many units

struct QuantFused {
    RowMap rows;
    uint32_t p;
    int k, kb, n, bn;                            // C_in, its blocks of 128, C_out, channels of a tile
    uint32_t units, n_tiles, per_part;           // per_part: channel tiles of a unit
    FastDiv by_parts;                            // units of the same rows
    int abufs, stages, nbuf, resident;           // A buffers, slots of streamed weights, boxes of an epilogue warp
    int vec, dense, relu;                        // rows of X (of Z) start on 16-byte boundaries
};

struct QuantCtl {
    uint64_t full[kQMaxStages], empty[kQMaxStages], wfull, a_full[2], a_empty[2], xs_full[kQSlots], acc_full[2], acc_empty[2], add_full[8];
    uint32_t tmem_base;
    int abort_flag;
};

// tcgen05.mma instruction descriptor of kind::i8: bits 4-5 D format (2 = s32), 7-9 and 10-12 operand formats (1 = s8), 17-22 N >> 3,
// 24-28 M >> 4.
__host__ __device__ constexpr uint32_t idesc_s8(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_s8(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}

// LPR lanes read a row, 8 CPL LPR elements at most.
template <class T, int LPR, int CPL>
__global__ void __launch_bounds__(kQThreads) quant_fused_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_z,
                                                                const __grid_constant__ CUtensorMap tm_add, const QuantFused g,
                                                                const T *__restrict__ x, const float *__restrict__ ws,
                                                                const float *__restrict__ shift, const T *__restrict__ add,
                                                                T *__restrict__ z, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *a_tiles = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t a_bytes = (uint32_t)g.kb * kQBlock, w_bytes = (uint32_t)g.bn * 128;
    uint8_t *w_tiles = a_tiles + (size_t)g.abufs * a_bytes;
    uint8_t *staging = w_tiles + (size_t)(g.resident ? g.n_tiles * g.kb : g.stages) * w_bytes;
    float *params = (float *)(staging + (size_t)8 * g.nbuf * kQStage);          // 8 warps x [scale 64 | shift 64]
    float *xs_s = params + 8 * 128;                                             // [kQSlots][128]
    QuantCtl *ctl = (QuantCtl *)(xs_s + kQSlots * kQRows);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &ctl->abort_flag;

    if (threadIdx.x == 0) {
        prefetch_tensormap(&tm_w);
        for (int s = 0; s < kQMaxStages; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        mbar_init(&ctl->wfull, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl->a_full[s], 8); mbar_init(&ctl->a_empty[s], 1);
            mbar_init(&ctl->acc_full[s], 1); mbar_init(&ctl->acc_empty[s], 4);
        }
        for (int s = 0; s < kQSlots; ++s) mbar_init(&ctl->xs_full[s], 8);
        for (int s = 0; s < 8; ++s) mbar_init(&ctl->add_full[s], 1);
        ctl->abort_flag = 0;
        fence_barrier_init();
    }
    uint32_t tmem_cols = 32;
    while (tmem_cols < 2u * g.bn) tmem_cols *= 2;
    if (warp == 1) {
        tmem_alloc(&ctl->tmem_base, tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem_base = ctl->tmem_base;
    auto give_up = [&]() { atomicOr(err, ERRW_TIMEOUT); ctl->abort_flag = 1; };
    // channel tiles [first, last) of unit u, whose rows start at 128 m
    auto unit = [&](uint32_t u, uint32_t &m, uint32_t &first, uint32_t &last) {
        m = g.by_parts.div(u);
        first = (u - m * g.by_parts.d) * g.per_part;
        last = min(first + g.per_part, g.n_tiles);
    };

    if (warp == 0) {
        if (elect_one()) {
            bool ok = true;
            uint32_t it = 0, m, nt, last;
            if (g.resident) {
                mbar_arrive_expect_tx(&ctl->wfull, g.n_tiles * g.kb * w_bytes);
                for (nt = 0; nt < g.n_tiles; ++nt)
                    for (int kb = 0; kb < g.kb; ++kb)
                        tma_load_2d(w_tiles + (size_t)(nt * g.kb + kb) * w_bytes, &tm_w, &ctl->wfull, kb * 128, (int)nt * g.bn);
            } else {
                for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x)
                    for (unit(u, m, nt, last); ok && nt < last; ++nt)
                        for (int kb = 0; kb < g.kb; ++kb, ++it) {
                            const uint32_t s = it % g.stages, ph = (it / g.stages) & 1u;
                            ok = mbar_wait_bounded(&ctl->empty[s], ph ^ 1u, abort_flag);
                            if (!ok) break;
                            mbar_arrive_expect_tx(&ctl->full[s], w_bytes);
                            tma_load_2d(w_tiles + (size_t)s * w_bytes, &tm_w, &ctl->full[s], kb * 128, (int)nt * g.bn);
                        }
            }
            if (!ok) {
                give_up();
                for (uint32_t j = it > (uint32_t)g.stages ? it - g.stages : 0; j < it; ++j)      // let the copies in flight land
                    mbar_wait_bounded(&ctl->full[j % g.stages], (j / g.stages) & 1u, nullptr, 200000000ull);
            } else if (g.resident) {
                mbar_wait_bounded(&ctl->wfull, 0, nullptr, 200000000ull);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = idesc_s8(kQRows, g.bn), hi = smem_desc_hi_sw128(1024);
            const uint32_t a0 = smem_desc_lo(smem_u32(a_tiles), 16), w0 = smem_desc_lo(smem_u32(w_tiles), 16);
            const int tail = (g.k - (g.kb - 1) * 128 + 31) / 32;              // steps of 32 codes of the last block
            bool ok = !g.resident || mbar_wait_bounded(&ctl->wfull, 0, abort_flag);
            uint32_t i = 0, s = 0, it = 0, m, nt, last;
            for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
                const uint32_t ab = g.abufs == 2 ? (i & 1u) : 0u, use = g.abufs == 2 ? (i >> 1) : i;
                ok = mbar_wait_bounded(&ctl->a_full[ab], use & 1u, abort_flag);
                for (unit(u, m, nt, last); ok && nt < last; ++nt, ++s) {
                    const uint32_t acc = s & 1u, d = tmem_base + acc * (uint32_t)g.bn;
                    ok = mbar_wait_bounded(&ctl->acc_empty[acc], ((s >> 1) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    for (int kb = 0; kb < g.kb; ++kb) {
                        uint32_t slot = nt * g.kb + kb;
                        if (!g.resident) {
                            slot = it % g.stages;
                            ok = mbar_wait_bounded(&ctl->full[slot], (it / g.stages) & 1u, abort_flag);
                            if (!ok) break;
                            ++it;
                        }
                        const uint32_t a_lo = a0 + ((ab * a_bytes + (uint32_t)kb * kQBlock) >> 4), w_lo = w0 + (slot * w_bytes >> 4);
                        const int steps = kb + 1 == g.kb ? tail : 4;
                        for (int q = 0; q < steps; ++q) umma_s8(d, a_lo + 2u * q, hi, w_lo + 2u * q, hi, idesc, (uint32_t)(kb | q));
                        if (!g.resident) umma_commit(&ctl->empty[slot]);
                    }
                    if (ok) umma_commit(&ctl->acc_full[acc]);
                }
                if (ok) umma_commit(&ctl->a_empty[ab]);
            }
            if (!ok) give_up();
        }
    } else if (warp >= kQLoadWarp) {
        // ---- rows to codes: warp qw has rows 16 qw .. 16 qw + 15 of a unit, RPI of them an instruction, RB such sets a batch ----
        constexpr int RPI = 32 / LPR, SETS = 16 / RPI;
        constexpr int ROOM = (sizeof(T) == 2 ? 8 : 4) / CPL, RB = ROOM < SETS ? ROOM : SETS, BATCHES = SETS / RB;
        const int qw = warp - kQLoadWarp, sub = lane & (LPR - 1), row_l = lane / LPR;
        Eight<T> next[RB][CPL];
        auto fetch = [&](uint32_t u, int batch) {
            uint32_t m, a, b;
            unit(u, m, a, b);
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const uint32_t row = m * kQRows + qw * 16 + (batch * RB + j) * RPI + row_l;
                const T *src = x + (row < g.p ? g.rows.at(row) : 0);
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    const int at = (c * LPR + sub) * 8;
                    if (row >= g.p || at >= g.k) next[j][c].zero();
                    else if (g.vec) next[j][c].load(src + at);
                    else next[j][c].load_some(src + at, g.k - at);
                }
            }
        };
        bool ok = true;
        uint32_t i = 0;
        if (blockIdx.x < g.units) fetch(blockIdx.x, 0);
        for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
            const uint32_t ab = g.abufs == 2 ? (i & 1u) : 0u, use = g.abufs == 2 ? (i >> 1) : i;
            uint8_t *tile = a_tiles + (size_t)ab * a_bytes;
            float *xs = xs_s + (i % kQSlots) * kQRows + qw * 16;
#pragma unroll 1
            for (int batch = 0; batch < BATCHES; ++batch) {
                Eight<T> now[RB][CPL];
#pragma unroll
                for (int j = 0; j < RB; ++j)
#pragma unroll
                    for (int c = 0; c < CPL; ++c) now[j][c] = next[j][c];
                if (batch + 1 < BATCHES) fetch(u, batch + 1);
                else if (u + gridDim.x < g.units) fetch(u + gridDim.x, 0);
                uint32_t top[RB];
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    uint32_t t = now[j][0].top();
#pragma unroll
                    for (int c = 1; c < CPL; ++c) t = Eight<T>::max_top(t, now[j][c].top());
                    t = Eight<T>::top_f32(t);
                    if constexpr (LPR == 32) t = __reduce_max_sync(0xffffffffu, t);
                    else
#pragma unroll
                        for (int o = LPR / 2; o > 0; o >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, o));
                    top[j] = t;
                }
                // lane j of a row's lanes works out the scales of its set j
                uint32_t mine = top[0];
#pragma unroll
                for (int j = 1; j < RB; ++j) mine = (sub & (RB - 1)) == j ? top[j] : mine;
                const RowScale rs = row_scale(mine);
                if (batch == 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->a_empty[ab], (use & 1u) ^ 1u, abort_flag));
                    if (!ok) break;
                }
                if (sub < RB) xs[(batch * RB + sub) * RPI + row_l] = rs.scale;
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    const float inv = __shfl_sync(0xffffffffu, rs.inv, (lane & ~(LPR - 1)) + j);
                    const int r = qw * 16 + (batch * RB + j) * RPI + row_l;
#pragma unroll
                    for (int c = 0; c < CPL; ++c) {
                        const int at = (c * LPR + sub) * 8;
                        if (at < g.kb * 128)
                            *(uint2 *)(tile + (size_t)(at >> 7) * kQBlock + r * 128 + ((((at >> 4) ^ r) & 7) << 4) + (at & 8)) = now[j][c].codes(inv);
                    }
                }
            }
            if (!ok) break;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) { mbar_arrive(&ctl->xs_full[i % kQSlots]); mbar_arrive(&ctl->a_full[ab]); }
        }
        if (!ok && lane == 0) give_up();
    } else {
        // ---- epilogue ----
        constexpr int CH = 128 / sizeof(T);                  // columns of a box
        const int quarter = warp & 3, ew = warp - 2;
        const uint32_t egroup = (uint32_t)ew >> 2;
        uint8_t *boxes = staging + (size_t)ew * g.nbuf * kQStage;
        float *par = params + ew * 128;
        uint64_t *add_bar = &ctl->add_full[ew];
        bool ok = true;
        uint32_t i = 0, s = 0, m, nt, last, turn = 0, add_ph = 0;
        const bool boxed = g.dense && add;
        for (uint32_t u = blockIdx.x; ok && u < g.units; u += gridDim.x, ++i) {
            for (unit(u, m, nt, last); ok && nt < last; ++nt, ++s) {
                if ((s & 1u) != egroup) continue;
                const uint32_t row0 = m * kQRows + quarter * 32, row = row0 + lane;
                const int n0 = (int)nt * g.bn, cols = min(g.bn, g.n - n0);
                auto box = [&]() { return boxes + (g.nbuf == 2 ? turn * kQStage : 0u); };
                // the addend's box goes where the results will be; the box's last store has been read
                auto fetch_add = [&](int c0) {
                    if (lane == 0) {
                        if (g.nbuf == 2) tma_store_wait_read<1>(); else tma_store_wait_read<0>();
                        if (boxed) {
                            mbar_arrive_expect_tx(add_bar, kQStage);
                            tma_load_2d(box(), &tm_add, add_bar, n0 + c0, (int)row0);
                        }
                    }
                    __syncwarp();
                };
                if (g.dense) fetch_add(0);
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->xs_full[i % kQSlots], (i / kQSlots) & 1u, abort_flag));
                const float xs = ok ? xs_s[(i % kQSlots) * kQRows + quarter * 32 + lane] : 0.f;
                ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&ctl->acc_full[s & 1u], (s >> 1) & 1u, abort_flag));
                if (!ok) {
                    if (boxed) { if (lane == 0) mbar_wait_bounded(add_bar, add_ph, nullptr, 200000000ull); __syncwarp(); }
                    break;
                }
                tc_fence_after_sync();
                const uint32_t t_row = tmem_base + (s & 1u) * (uint32_t)g.bn + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
                for (int c0 = 0; c0 < cols; c0 += CH) {
                    uint8_t *buf = box(), *brow = buf + lane * 128;
#pragma unroll
                    for (int c = lane; c < CH; c += 32) {
                        const int col = n0 + c0 + c;
                        par[c] = col < g.n ? __ldg(ws + col) : 0.f;
                        par[64 + c] = col < g.n ? __ldg(shift + col) : 0.f;
                    }
                    __syncwarp();
                    if (boxed) {
                        ok = __all_sync(0xffffffffu, mbar_wait_bounded(add_bar, add_ph, abort_flag));
                        add_ph ^= 1u;
                        if (!ok) break;
                    }
#pragma unroll 1
                    for (int h = 0; h < CH; h += 32) {
                        uint32_t v[32];
                        tmem_ld_32x32(t_row + (uint32_t)(c0 + h), v);
                        tmem_ld_wait();
                        float f[32];
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 w4 = *(const float4 *)(par + h + j), b4 = *(const float4 *)(par + 64 + h + j);
                            f[j] = fmaf((float)(int)v[j] * xs, w4.x, b4.x);
                            f[j + 1] = fmaf((float)(int)v[j + 1] * xs, w4.y, b4.y);
                            f[j + 2] = fmaf((float)(int)v[j + 2] * xs, w4.z, b4.z);
                            f[j + 3] = fmaf((float)(int)v[j + 3] * xs, w4.w, b4.w);
                        }
                        if (g.dense) {
                            constexpr int PER = 16 / sizeof(T);
#pragma unroll
                            for (int j = 0; j < 32; j += PER) {
                                uint4 *at = (uint4 *)(brow + ((((h + j) / PER ^ lane) & 7) << 4));
                                uint4 q = boxed ? *at : make_uint4(0u, 0u, 0u, 0u);
                                uint32_t *w = (uint32_t *)&q;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if constexpr (sizeof(T) == 2) {
                                        constexpr bool H = __is_same(T, __half);
                                        float lo = f[j + 2 * e], hi = f[j + 2 * e + 1], al, ah;
                                        if (boxed) { unpack2_t<H>(w[e], al, ah); lo += al; hi += ah; }
                                        if (g.relu) { lo = fmaxf(lo, 0.f); hi = fmaxf(hi, 0.f); }
                                        w[e] = pack2_t<H>(lo, hi);
                                    } else {
                                        float v1 = f[j + e];
                                        if (boxed) v1 += __uint_as_float(w[e]);
                                        w[e] = __float_as_uint(g.relu ? fmaxf(v1, 0.f) : v1);
                                    }
                                }
                                *at = q;
                            }
                        } else if (row < g.p) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                if (c0 + h + j >= cols) continue;
                                const size_t at = (size_t)row * g.n + n0 + c0 + h + j;
                                float v1 = f[j];
                                if (add) v1 += to_f32(add[at]);
                                z[at] = from_f32<T>(g.relu ? fmaxf(v1, 0.f) : v1);
                            }
                        }
                    }
                    if (c0 + CH >= cols) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&ctl->acc_empty[s & 1u]);
                    }
                    if (g.dense) {
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(&tm_z, buf, n0 + c0, (int)row0);
                            tma_store_commit();
                        }
                        turn ^= 1u;
                        if (c0 + CH < cols) fetch_add(c0 + CH);
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
    if (warp == 1) tmem_dealloc(tmem_base, tmem_cols);
}

// Shared memory of a choice of buffers; 0: they do not fit.
size_t fused_smem(const QuantFused &g) {
    const size_t w = (size_t)(g.resident ? (int)g.n_tiles * g.kb : g.stages) * g.bn * 128;
    return 1024 + (size_t)g.abufs * g.kb * kQBlock + w + (size_t)8 * g.nbuf * kQStage + 8 * 512 + kQSlots * kQRows * 4 + sizeof(QuantCtl) + 16;
}

}  // namespace

bool quant_fused_eligible(const Problem &pb) { return pb.c_in <= 1024; }

RowMap quant_row_map(const Problem &pb) {
    RowMap r;
    r.step = pb.c_in;
    r.strided = pb.stride_h != 1 || pb.stride_w != 1;
    r.pixel = (long long)pb.stride_w * pb.c_in;
    r.image = (long long)pb.h_in * pb.w_in * pb.c_in;
    r.line = (long long)pb.stride_h * pb.w_in * pb.c_in;
    r.by_w = FastDiv((uint32_t)pb.w_out);
    r.by_h = FastDiv((uint32_t)pb.h_out);
    return r;
}

cudaError_t launch_quant_fused(const Problem &pb, int dtype, const void *x, const void *wq, const float *ws, const float *shift,
                               const void *add, int relu, void *z, cudaStream_t st) {
    const int es = dtype == CONVBN_F32 ? 4 : 2, sms = device_sm_count();
    QuantFused g;
    g.rows = quant_row_map(pb);
    g.p = (uint32_t)pb.p; g.k = pb.c_in; g.kb = (pb.c_in + 127) / 128; g.n = pb.c_out; g.relu = relu;
    g.vec = (size_t)pb.c_in * es % 16 == 0 && pb.c_in % 8 == 0;
    g.dense = (size_t)pb.c_out * es % 16 == 0;
    const uint32_t m_tiles = (uint32_t)((pb.p + kQRows - 1) / kQRows);
    // Enough rows for every SM: wide tiles.  Fewer: tiles of 64 channels, and the channels cut into parts.
    const bool many = m_tiles * 2 > (uint32_t)sms;
    auto tiles = [&](int widest) {
        g.n_tiles = (uint32_t)((pb.c_out + widest - 1) / widest);
        g.bn = (int)(((pb.c_out + g.n_tiles - 1) / g.n_tiles + 63) / 64 * 64);
        uint32_t parts = many ? 1 : (uint32_t)sms / m_tiles;
        if (parts > g.n_tiles) parts = g.n_tiles;
        g.per_part = (g.n_tiles + parts - 1) / parts;
        parts = (g.n_tiles + g.per_part - 1) / g.per_part;
        g.by_parts = FastDiv(parts);
        g.units = m_tiles * parts;
    };
    // Buffers, the most wanted first: two of the A operand (rows are converted while others are multiplied), the weights resident
    // or at least three slots of them, wide tiles, two boxes per epilogue warp.
    const size_t room = 227 * 1024;
    size_t smem = 0;
    for (g.abufs = 2; g.abufs > 0 && !smem; --g.abufs)
        for (int widest = many ? 256 : 64; widest >= (many && g.abufs == 2 ? 128 : 64) && !smem; widest /= 2) {
            tiles(widest);
            for (int choice = 0; choice < 4 && !smem; ++choice) {
                g.resident = choice < 2;
                g.nbuf = 2 - (choice & 1);
                g.stages = 3;
                if (g.resident && (g.by_parts.d != 1 || m_tiles < (uint32_t)sms)) continue;
                if (fused_smem(g) > room) continue;
                while (!g.resident && g.stages < kQMaxStages) {
                    ++g.stages;
                    if (fused_smem(g) > room) { --g.stages; break; }
                }
                smem = fused_smem(g);
            }
            if (smem) break;
        }
    if (!smem) return cudaErrorInvalidValue;
    ++g.abufs;                                         // (the loop's last step)
    const unsigned grid = g.units < (uint32_t)sms ? g.units : (unsigned)sms;
    CUtensorMap tw, tz, ta;
    if (!make_tmap_matrix_bytes(&tw, wq, pb.c_out, quant_pitch(pb), 1, g.bn)) return cudaErrorInvalidValue;
    tz = ta = tw;
    if (g.dense) {
        if (!make_tmap_matrix_bytes(&tz, z, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
        if (add && !make_tmap_matrix_bytes(&ta, add, pb.p, pb.c_out, es, 32)) return cudaErrorInvalidValue;
    }
    int *err = nullptr;
    if (cudaError_t e = error_word_address(&err); e != cudaSuccess) return e;
    auto go = [&](auto tag, auto lpr, auto cpl) {
        using T = decltype(tag);
        auto kernel = quant_fused_kernel<T, decltype(lpr)::value, decltype(cpl)::value>;
        static PerDevice attr, carve;
        if (cudaError_t e = max_dynamic_smem_once(kernel, 227 * 1024, &attr); e != cudaSuccess) return e;
        prefer_max_shared_once(kernel, &carve);
        return launch_pdl(kernel, dim3(grid), dim3(kQThreads), smem, st, tw, tz, ta, g, (const T *)x, ws, shift, (const T *)add, (T *)z, err);
    };
    auto typed = [&](auto tag) {
        using std::integral_constant;
        if (pb.c_in <= 64) return go(tag, integral_constant<int, 8>(), integral_constant<int, 1>());
        if (pb.c_in <= 128) return go(tag, integral_constant<int, 16>(), integral_constant<int, 1>());
        if (pb.c_in <= 256) return go(tag, integral_constant<int, 32>(), integral_constant<int, 1>());
        if (pb.c_in <= 512) return go(tag, integral_constant<int, 32>(), integral_constant<int, 2>());
        return go(tag, integral_constant<int, 32>(), integral_constant<int, 4>());
    };
    return dtype == CONVBN_F32 ? typed(float()) : (dtype == CONVBN_F16 ? typed(__half()) : typed(__nv_bfloat16()));
}

}  // namespace convbn
